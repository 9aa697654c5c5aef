"""mocap_window_attn against the plain form in 64 bits: windows and sinks around
every tile edge, every head layout, splits, hidden NaN and infinities, graphs and
refusals."""
import math

import pytest
import torch

from helpers import say
from paper_2606_22968_amd import binding
from serve_helpers import B, Attention, check_close, make_store, randn

pytestmark = pytest.mark.gpu

# Probabilities enter P V rounded to bf16, and their rounded sum normalises O.
P_ERROR = B


def attend(store, table, q, prefix, scale, window, sinks, splits=0):
    rows, h_q, d = q.shape
    n_ranges, size = binding.mocap_window_attn_workspace_size(prefix, rows, h_q, store.h_kv, d, window, sinks, splits)
    ws = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda").fill_(0xFF)
    o = torch.full((rows, h_q, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    lse = torch.full((h_q, rows), float("nan"), dtype=torch.float32, device="cuda")
    binding.mocap_window_attn(store, table, q, prefix, scale, window, sinks, o, lse, ws, splits)
    return o, lse, n_ranges


def check(o, lse, ref, label):
    check_close(o, ref.o, ref.o_bound(P_ERROR), f"{label} o")
    check_close(lse, ref.lse, ref.lse_bound(), f"{label} lse")


def run(seed, h_q, h_kv, d, bs, prefix, rows, window, sinks, splits=0, drop=True):
    """With `drop`, positions that no row sees hold NaN keys and values."""
    n = prefix + rows
    store, tables, ks, vs = make_store(seed, [n], bs, h_kv, d)
    low = max(0, prefix - window + 1)
    if drop and low > sinks:
        pos = torch.arange(sinks, low, device="cuda")
        block, slot = tables[0].long()[pos // bs], pos % bs
        store.k_pool[block, :, slot] = float("nan")
        store.v_pool[block, :, :, slot] = float("nan")
    q = randn(seed + 1, rows, h_q, d)
    scale = d ** -0.5
    o, lse, n_ranges = attend(store, tables[0], q.cuda(), prefix, scale, window, sinks, splits)
    ref = Attention(q, ks[0], vs[0], prefix, scale, window, sinks)
    check(o, lse, ref, f"P={prefix} L={rows} W={window} s={sinks} splits={n_ranges}")
    return n_ranges


@pytest.mark.parametrize("h_q,h_kv,d", [(8, 2, 128), (8, 8, 64), (12, 4, 128), (6, 3, 64), (32, 1, 128), (64, 1, 64)])
@pytest.mark.parametrize("prefix,rows,window,sinks", [
    (0, 1, 1, 0), (0, 300, 1, 0), (0, 300, 1, 1), (0, 300, 64, 4), (0, 129, 1000, 4), (500, 1, 64, 0), (500, 1, 63, 3),
    (511, 2, 65, 64), (512, 64, 64, 65), (700, 137, 100, 4), (700, 137, 10, 128), (700, 65, 701, 0), (700, 65, 1 << 40, 7),
    (1000, 30, 128, 1 << 40), (1000, 31, 900, 100), (963, 200, 7, 63)])
def test_windows_and_layouts(gpu, h_q, h_kv, d, prefix, rows, window, sinks):
    say(f"[case] window {h_q}/{h_kv}/{d} P={prefix} L={rows} W={window} sinks={sinks}")
    run(100, h_q, h_kv, d, 64, prefix, rows, window, sinks)


@pytest.mark.parametrize("window", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 191, 192, 193])
@pytest.mark.parametrize("sinks", [0, 1, 63, 64, 65])
def test_window_and_sink_edges(gpu, window, sinks):
    say(f"[case] window edges W={window} sinks={sinks}")
    run(101, 4, 2, 64, 192, 200, 150, window, sinks)


@pytest.mark.parametrize("splits", [0, 1, 2, 3, 5, 17, 1000])
@pytest.mark.parametrize("h_q,h_kv,d", [(8, 2, 128), (3, 3, 64)])
def test_splits(gpu, splits, h_q, h_kv, d):
    say(f"[case] window splits={splits} {h_q}/{h_kv}/{d}")
    got = run(102, h_q, h_kv, d, 128, 2001, 100, 1100, 70, splits)
    assert splits == 0 or got == min(splits, got) and (splits == 1) == (got == 1)


def test_long_chunk_many_workgroups(gpu):
    run(103, 16, 2, 128, 256, 1000, 700, 333, 4)


def test_window_of_everything_equals_chunk_attention(gpu):
    """A window that reaches the first position: the rows of mocap_chunk_attn."""
    store, tables, ks, vs = make_store(104, [900], 64, 2, 128)
    q = randn(105, 200, 8, 128).cuda()
    o, lse, _ = attend(store, tables[0], q, 700, 0.1, 900, 0)
    o2, lse2 = torch.empty_like(o), torch.empty_like(lse)
    _, size = binding.mocap_chunk_attn_workspace_size(700, 200, 8, 2, 128, 0)
    binding.mocap_chunk_attn(store, tables[0], q, 700, 0.1, o2, lse2, torch.empty(max(size, 16), dtype=torch.uint8,
                                                                                  device="cuda"))
    ref = Attention(q.cpu(), ks[0], vs[0], 700, 0.1)
    check(o, lse, ref, "window")
    check(o2, lse2, ref, "chunk")


def test_one_token_equals_decode(gpu):
    """One row: mocap_decode_attn with the same window."""
    store, tables, ks, vs = make_store(106, [3000], 64, 2, 64)
    q = randn(107, 1, 4, 64).cuda()
    o, lse, _ = attend(store, tables[0], q, 2999, 0.125, 500, 4)
    o2, lse2 = torch.empty_like(q), torch.empty((1, 4), dtype=torch.float32, device="cuda")
    size = binding.mocap_decode_attn_workspace_size(1, 4, 2, 64, 3000, 500, 4)
    binding.mocap_decode_attn(store, tables, torch.tensor([3000], dtype=torch.int32).cuda(), q, 3000, 0.125, o2, lse2,
                              torch.empty(max(size, 16), dtype=torch.uint8, device="cuda"), 500, 4)
    ref = Attention(q.cpu(), ks[0], vs[0], 2999, 0.125, 500, 4)
    check(o, lse, ref, "window")
    check(o2, lse2.t(), ref, "decode")


@pytest.mark.parametrize("splits", [1, 3])
@pytest.mark.parametrize("d", [64, 128])
def test_nonfinite_reach_the_rows_that_see_them(gpu, splits, d):
    """Keys and values that are NaN or infinite: every row that sees one, no other."""
    prefix, rows, window, sinks, h_q, h_kv = 600, 300, 150, 5, 4, 2
    n = prefix + rows
    store, tables, ks, vs = make_store(108, [n], 64, h_kv, d)
    plant = [("k", 2, 0), ("v", 4, 1), ("v", 470, 0), ("k", 555, 1), ("v", 650, 1), ("v", 700, 0), ("inf", 800, 1),
             ("k", 899, 0)]
    touched_o = torch.zeros(rows, h_q, d, dtype=torch.bool)
    touched_lse = torch.zeros(h_q, rows, dtype=torch.bool)
    t = prefix + torch.arange(rows)
    for what, j, h in plant:
        sees = (j <= t) & ((j < sinks) | (j > t - window))
        block, slot = tables[0, j // 64].long(), j % 64
        heads = slice(h * 2, h * 2 + 2)
        if what == "k":
            store.k_pool[block, h, slot, 3] = float("nan")
            touched_o[sees, heads] = True
            touched_lse[heads, :] |= sees
        else:
            store.v_pool[block, h, 9, slot] = float("nan") if what == "v" else float("inf")
            touched_o[sees, heads, 9] = True
    q = randn(109, rows, h_q, d)
    o, lse, _ = attend(store, tables[0], q.cuda(), prefix, d ** -0.5, window, sinks, splits)
    assert torch.equal(~torch.isfinite(o.cpu().float()), touched_o)
    assert torch.equal(~torch.isfinite(lse.cpu()), touched_lse)
    ref = Attention(q, ks[0], vs[0], prefix, d ** -0.5, window, sinks)
    fine = ~touched_o
    err = (o.cpu().double() - ref.o).abs()[fine] / ref.o_bound(P_ERROR)[fine]
    assert float(err.max()) <= 1.0


@pytest.mark.parametrize("d", [64, 128])
def test_growing_scores(gpu, d):
    """Scores more than 60 binary orders above the first tile's, in and out of the window."""
    prefix, rows = 500, 100
    store, tables, ks, vs = make_store(110, [600], 64, 1, d)
    ks[0][:, 0, 0] = (torch.linspace(0, 1, 600) ** 2 * 250).to(torch.bfloat16)
    for lb in range(10):
        part = ks[0][lb * 64:(lb + 1) * 64]
        store.k_pool[tables[0, lb].long(), :, :part.shape[0]] = part.transpose(0, 1).cuda()
    q = torch.zeros(rows, 2, d, dtype=torch.bfloat16)
    q[:, 0, 0], q[:, 1, 0] = 2.0, -2.0
    o, lse, _ = attend(store, tables[0], q.cuda(), prefix, 1.0, 300, 3)
    check(o, lse, Attention(q, ks[0], vs[0], prefix, 1.0, 300, 3), "growing")


def test_graph_replays(gpu):
    store, tables, ks, vs = make_store(111, [5000], 256, 2, 128)
    q = randn(112, 64, 8, 128).cuda()
    _, size = binding.mocap_window_attn_workspace_size(4936, 64, 8, 2, 128, 2048, 4)
    assert size > 0
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    o, lse = torch.empty_like(q), torch.empty((8, 64), dtype=torch.float32, device="cuda")

    def call():
        binding.mocap_window_attn(store, tables[0], q, 4936, 0.09, 2048, 4, o, lse, ws)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(4):
        q.copy_(randn(113 + i, 64, 8, 128))
        ws.fill_(0xFF)
        o.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = o.clone(), lse.clone()
        check(*got, Attention(q.cpu(), ks[0], vs[0], 4936, 0.09, 2048, 4), f"replay {i}")
        call()
        torch.cuda.synchronize()
        assert torch.equal(o.view(torch.int16), got[0].view(torch.int16)) and torch.equal(lse, got[1])


def test_neighbouring_outputs_are_left_alone(gpu):
    store, tables, _, _ = make_store(114, [300], 64, 2, 64)
    q = randn(115, 64, 4, 64).cuda()
    o = torch.full((96, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((4 * 64 + 32,), 7.0, device="cuda")
    binding.mocap_window_attn(store, tables[0], q[:33], 200, 0.1, 50, 2, o[:33], lse[:4 * 33].view(4, 33), None, 1)
    torch.cuda.synchronize()
    assert (o[33:] == 7.0).all() and (lse[4 * 33:] == 7.0).all() and torch.isfinite(o.float()).all()


def test_offsets_beyond_32_bits(gpu):
    """A window at the end of more than 2^32 bytes of keys."""
    bs, h_kv, d, h_q = 1600, 8, 128, 16
    blocks = (1 << 32) // (2 * h_kv * bs * d) + 2
    store = binding.KvStore(blocks, bs, h_kv, d)
    n, rows = blocks * bs - 100, 50
    table = torch.arange(blocks - 1, -1, -1, dtype=torch.int32)
    table[-2:] = torch.tensor([blocks - 1, blocks - 2])
    table[0] = 1
    k, v = randn(116, 4 + 600, h_kv, d), randn(117, 4 + 600, h_kv, d)
    table = table.cuda()
    binding.mocap_kv_append(store, table, 0, k[:4].cuda(), v[:4].cuda())
    binding.mocap_kv_append(store, table, n - 600, k[4:].cuda(), v[4:].cuda())
    q = randn(118, rows, h_q, d)
    o, lse, _ = attend(store, table, q.cuda(), n - rows, d ** -0.5, 500, 4)
    # The same keys without the gap; the rows see the last 500 and the four sinks.
    ref = Attention(q, k, v, 604 - rows, d ** -0.5, 500, 4)
    check(o, lse, ref, "far")


def test_refused_calls_write_nothing(gpu):
    store, tables, _, _ = make_store(119, [3000], 64, 2, 64)
    q = randn(120, 16, 4, 64).cuda()
    o, lse = torch.full_like(q, 7.0), torch.full((4, 16), 7.0, device="cuda")
    for bad in (dict(window=0, sinks=1), dict(window=-1, sinks=0), dict(window=10, sinks=-1)):
        with pytest.raises(binding.MocapError) as err:
            binding.mocap_window_attn(store, tables[0], q, 2900, 0.1, bad["window"], bad["sinks"], o, lse, None, 1)
        assert err.value.status == binding.MOCAP_ERR_INVALID_ARG
    with pytest.raises(binding.MocapError) as err:
        binding.mocap_window_attn(store, tables[0], q, 2900, 0.1, 1000, 0, o, lse, None, 3)
    assert err.value.status == binding.MOCAP_ERR_WORKSPACE
    with pytest.raises(binding.MocapError):
        binding.mocap_window_attn(store, tables[0], q, 64 * tables.shape[1], 0.1, 1000, 0, o, lse, None, 1)
    with pytest.raises(ValueError):
        binding.mocap_window_attn(store, tables[0], q, 2900, 0.1, 1000, 0, o, lse.t().contiguous(), None, 1)
    torch.cuda.synchronize()
    assert (o == 7.0).all() and (lse == 7.0).all()


def test_empty_chunk(gpu):
    store = binding.KvStore(2, 64, 2, 64, fill=0.0)
    q = torch.zeros((0, 4, 64), dtype=torch.bfloat16, device="cuda")
    binding.mocap_window_attn(store, torch.zeros(2, dtype=torch.int32, device="cuda"), q, 100, 0.1, 5, 1, q.clone(),
                              torch.zeros((4, 0), device="cuda"))


@pytest.mark.parametrize("splits", [1, 3])
@pytest.mark.parametrize("d", [64, 128])
def test_scores_beyond_fp32(gpu, splits, d):
    """Products within fp32 whose multiple by the scale is not: NaN, as with an infinite score, and not an empty row."""
    prefix, rows, window, sinks, h_q, h_kv = 600, 300, 150, 5, 4, 2
    store, tables, _, _ = make_store(121, [prefix + rows], 64, h_kv, d)
    store.k_pool[:, :, :, 0] = 0.0
    want = torch.zeros(rows, h_q, dtype=torch.bool)
    t = prefix + torch.arange(rows)
    for j in (500, 640, 831):
        store.k_pool[tables[0, j // 64].long(), :, j % 64, 0] = 1e19  # 1e38, and 4e38 with the scale
        want[(j <= t) & (j > t - window), 0::2] = True
    q = randn(122, rows, h_q, d)
    q[:, 0::2, 0], q[:, 1::2, 0] = 1e19, -1.0
    o, lse, _ = attend(store, tables[0], q.cuda(), prefix, 4.0, window, sinks, splits)
    assert torch.equal(torch.isnan(lse.cpu()).t(), want) and torch.isfinite(lse.cpu().t()[~want]).all()
    assert torch.equal(torch.isnan(o.cpu()).all(-1), want) and torch.isfinite(o.cpu()[~want].float()).all()
