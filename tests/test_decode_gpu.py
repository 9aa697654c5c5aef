"""mocap_decode_append and mocap_decode_attn against the plain form in 64 bits:
lengths from none to long ones, every head layout, block sizes, windows and
sinks, splits, hidden NaN, graphs, streams and refusals."""
import math

import pytest
import torch

from helpers import say
from paper_2606_22968_amd import binding
from serve_helpers import Attention, check_close, make_store, randn, take

pytestmark = pytest.mark.gpu

# A probability enters P V as two bf16 values: what is left is below B^2 of it.
P_ERROR = 2.0 ** -16


def workspace(batch, h_q, h_kv, d, max_len, window=0, sinks=0):
    size = binding.mocap_decode_attn_workspace_size(batch, h_q, h_kv, d, max_len, window, sinks)
    return torch.empty(max(size, 16), dtype=torch.uint8, device="cuda").fill_(0xFF)


def attend(store, tables, lens, q, max_len, scale, window=0, sinks=0, ws=None):
    batch, h_q, d = q.shape
    o = torch.full((batch, h_q, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    lse = torch.full((batch, h_q), float("nan"), dtype=torch.float32, device="cuda")
    seq_lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
    ws = workspace(batch, h_q, store.h_kv, d, max_len, window, sinks) if ws is None else ws
    binding.mocap_decode_attn(store, tables, seq_lens, q, max_len, scale, o, lse, ws, window, sinks)
    return o, lse


def check(o, lse, q, ks, vs, lens, scale, window=0, sinks=0, label=""):
    for b, n in enumerate(lens):
        n = max(n, 0)
        ref = Attention(q[b:b + 1].cpu(), ks[b][:n], vs[b][:n], n - 1, scale, window, sinks)
        check_close(o[b:b + 1], ref.o, ref.o_bound(P_ERROR) + 1e-30, f"{label} o[{b}] n={n}")
        check_close(lse[b][:, None], ref.lse, ref.lse_bound(), f"{label} lse[{b}] n={n}")


RAGGED = [1, 0, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300, -3, 511, 512, 513, 700]


@pytest.mark.parametrize("h_q,h_kv,d", [(8, 8, 64), (32, 8, 128), (12, 4, 128), (6, 3, 64), (15, 1, 128), (16, 1, 64),
                                        (17, 1, 128), (32, 1, 128), (33, 1, 64), (64, 1, 64), (40, 1, 128)])
@pytest.mark.parametrize("bs", [64, 192])
def test_ragged_batch(gpu, h_q, h_kv, d, bs):
    say(f"[case] decode ragged {h_q}/{h_kv}/{d} bs={bs}")
    store, tables, ks, vs = make_store(1, RAGGED, bs, h_kv, d)
    q = randn(2, len(RAGGED), h_q, d).cuda()
    o, lse = attend(store, tables, RAGGED, q, 700, d ** -0.5)
    check(o, lse, q, ks, vs, RAGGED, d ** -0.5)
    assert (o[1] == 0).all() and (lse[1] == -math.inf).all()


@pytest.mark.parametrize("h_q,h_kv,d", [(32, 8, 128), (8, 2, 64), (20, 1, 64)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 3), (64, 0), (64, 64), (100, 4), (100, 65), (129, 130),
                                          (700, 4), (701, 4), (5000, 9), (300, 5000)])
def test_windows(gpu, h_q, h_kv, d, window, sinks):
    lens = [1, 0, 5, 64, 65, 100, 101, 129, 200, 333, 448, 700]
    say(f"[case] decode window={window} sinks={sinks} {h_q}/{h_kv}/{d}")
    store, tables, ks, vs = make_store(3, lens, 64, h_kv, d)
    # What no row sees may hold anything.
    for b, n in enumerate(lens):
        for t in range(n):
            if not (t < sinks or t > n - 1 - window):
                block, slot = tables[b, t // 64].long(), t % 64
                store.k_pool[block, :, slot] = float("nan")
                store.v_pool[block, :, :, slot] = float("inf")
    q = randn(4, len(lens), h_q, d).cuda()
    o, lse = attend(store, tables, lens, q, 700, d ** -0.5, window, sinks)
    check(o, lse, q, ks, vs, lens, d ** -0.5, window, sinks)


@pytest.mark.parametrize("lens", [[20000], [9001, 1, 64], [5000, 0, 30000, 257, 12345], [2049] * 70, [1] * 200 + [4000]])
@pytest.mark.parametrize("h_q,h_kv,d,bs", [(4, 1, 128, 256), (8, 2, 64, 1600)])
def test_cut_sequences(gpu, lens, h_q, h_kv, d, bs):
    """Long sequences among short ones: parts, and their join; batches beyond 64."""
    say(f"[case] decode cut batch={len(lens)} {h_q}/{h_kv}/{d}")
    store, tables, ks, vs = make_store(5, lens, bs, h_kv, d)
    q = randn(6, len(lens), h_q, d).cuda()
    o, lse = attend(store, tables, lens, q, max(lens), d ** -0.5)
    few = sorted(set(range(min(3, len(lens)))) | {len(lens) - 1})
    for b in few:
        check(o[b:b + 1], lse[b:b + 1], q[b:b + 1], ks[b:b + 1], vs[b:b + 1], lens[b:b + 1], d ** -0.5)
    # The same sequence alone, planned otherwise: equal within the bounds.
    for b in few:
        o1, lse1 = attend(store, tables[b:b + 1].contiguous(), lens[b:b + 1], q[b:b + 1], max(lens[b], 1), d ** -0.5)
        check(o1, lse1, q[b:b + 1], ks[b:b + 1], vs[b:b + 1], lens[b:b + 1], d ** -0.5)
    # Equal inputs, equal bits.
    o2, lse2 = attend(store, tables, lens, q, max(lens), d ** -0.5)
    assert torch.equal(o.view(torch.int16), o2.view(torch.int16)) and torch.equal(lse, lse2)


def test_lengths_beyond_max_len(gpu):
    """A sequence longer than max_len is taken to end there; tables wider than needed."""
    store, tables, ks, vs = make_store(7, [1000, 700], 64, 2, 64)
    q = randn(8, 2, 4, 64).cuda()
    o, lse = attend(store, tables, [1000, 1 << 30], q, 640, 0.125)
    check(o, lse, q, ks, vs, [640, 640], 0.125)


def test_growing_scores(gpu):
    """Scores that grow by tens of binary orders from key to key, and fall: the running maximum."""
    lens = [300, 300]
    store, tables, ks, vs = make_store(9, lens, 64, 1, 64)
    q = torch.zeros(2, 3, 64, dtype=torch.bfloat16)
    q[:, :, 0] = 8.0
    for b in range(2):
        ks[b][:, 0, 0] = torch.linspace(-200, 200, 300).to(torch.bfloat16) * (1 if b == 0 else -1)
        for lb in range(5):
            part = ks[b][lb * 64:(lb + 1) * 64]
            store.k_pool[tables[b, lb].long(), :, :part.shape[0]] = part.transpose(0, 1).cuda()
    q = q.cuda()
    o, lse = attend(store, tables, lens, q, 300, 1.0)
    check(o, lse, q, ks, vs, lens, 1.0)


def test_nonfinite_inputs(gpu):
    """NaN reaches the rows that see it and no other."""
    lens = [200, 200, 200, 2500, 2500]
    store, tables, ks, vs = make_store(10, lens, 64, 2, 128)
    q = randn(11, 5, 4, 128)
    store.k_pool[tables[0, 1].long(), 0, 5] = float("nan")
    store.v_pool[tables[3, 30].long(), 1, 7, 9] = float("nan")
    q[4, 3] = float("nan")
    q = q.cuda()
    o, lse = attend(store, tables, lens, q, 2500, 128 ** -0.5)
    bad = torch.isnan(o).any(-1).cpu()
    want = torch.zeros(5, 4, dtype=torch.bool)
    want[0, :2] = want[3, 2:] = want[4, 3] = True
    assert torch.equal(bad, want)
    assert torch.isnan(o[0, :2]).all() and torch.isnan(o[4, 3]).all()
    assert torch.isnan(o[3, 2:, 7]).all() and torch.isfinite(o[3, 2:, :7].float()).all()
    want[3, 2:] = False
    assert torch.equal(torch.isnan(lse).cpu(), want)
    for b in (1, 2):
        check(o[b:b + 1], lse[b:b + 1], q[b:b + 1], ks[b:b + 1], vs[b:b + 1], lens[b:b + 1], 128 ** -0.5)


@pytest.mark.parametrize("h_kv,d,bs", [(8, 128, 256), (3, 64, 64), (70, 64, 192)])
def test_append_is_bit_exact(gpu, h_kv, d, bs):
    lens = [1, 0, 64, 65, 192, 193, -5, 300, 5000, 7]
    stride = 5
    batch = len(lens)
    say(f"[case] decode append h_kv={h_kv} d={d} bs={bs}")
    total = batch * stride
    tables = torch.randperm(total, generator=torch.Generator().manual_seed(12)).to(torch.int32).view(batch, stride)
    store = binding.KvStore(total, bs, h_kv, d, fill=float("nan"))
    k, v = randn(13, batch, h_kv, d), randn(14, batch, h_kv, d)
    want_k, want_v = store.k_pool.cpu(), store.v_pool.cpu()
    for b, n in enumerate(lens):
        if 0 < n <= stride * bs:
            block, slot = int(tables[b, (n - 1) // bs]), (n - 1) % bs
            want_k[block, :, slot] = k[b]
            want_v[block, :, :, slot] = v[b]
    binding.mocap_decode_append(store, tables.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), k.cuda(), v.cuda())
    torch.cuda.synchronize()
    assert torch.equal(store.k_pool.cpu().view(torch.int16), want_k.view(torch.int16))
    assert torch.equal(store.v_pool.cpu().view(torch.int16), want_v.view(torch.int16))


def test_append_equals_kv_append(gpu):
    """The batch append writes what mocap_kv_append of one position writes."""
    stores = []
    table = torch.tensor([[2, 0], [3, 1]], dtype=torch.int32).cuda()
    k, v = randn(15, 2, 4, 128).cuda(), randn(16, 2, 4, 128).cuda()
    for batch in (True, False):
        store = binding.KvStore(4, 128, 4, 128, fill=0.0)
        if batch:
            binding.mocap_decode_append(store, table, torch.tensor([130, 77], dtype=torch.int32).cuda(), k, v)
        else:
            for b, n in enumerate((130, 77)):
                binding.mocap_kv_append(store, table[b].clone(), n - 1, k[b:b + 1], v[b:b + 1])
        stores.append(store)
    assert torch.equal(stores[0].k_pool, stores[1].k_pool) and torch.equal(stores[0].v_pool, stores[1].v_pool)
    assert torch.equal(take(stores[0], table[1], 77)[0][76], k[1].cpu())


def test_empty_batch(gpu):
    store = binding.KvStore(2, 64, 2, 64, fill=0.0)
    tables = torch.zeros((0, 3), dtype=torch.int32, device="cuda")
    lens = torch.zeros(0, dtype=torch.int32, device="cuda")
    kv = torch.zeros((0, 2, 64), dtype=torch.bfloat16, device="cuda")
    q = torch.zeros((0, 4, 64), dtype=torch.bfloat16, device="cuda")
    binding.mocap_decode_append(store, tables, lens, kv, kv)
    binding.mocap_decode_attn(store, tables, lens, q, 100, 1.0, q.clone(), torch.zeros((0, 4), device="cuda"))


def test_max_len_zero_gives_empty_rows(gpu):
    store = binding.KvStore(2, 64, 2, 64, fill=float("nan"))
    tables = torch.zeros((3, 1), dtype=torch.int32, device="cuda")
    o, lse = attend(store, tables, [5, 0, 64], randn(17, 3, 4, 64).cuda(), 0, 1.0)
    assert (o == 0).all() and (lse == -math.inf).all()


def test_graph_replays_with_other_lengths(gpu):
    """A captured step (append, attention with parts and join) replayed with
    lengths, queries and tokens changed between the replays."""
    lens_list = [[4000, 33, 900], [4001, 34, 901], [1, 3000, 0], [4096, 4096, 4096]]
    h_q, h_kv, d, bs = 8, 2, 128, 128
    store, tables, ks, vs = make_store(18, [4096] * 3, bs, h_kv, d, fill=0.0)
    seq_lens = torch.zeros(3, dtype=torch.int32, device="cuda")
    q = torch.zeros((3, h_q, d), dtype=torch.bfloat16, device="cuda")
    k, v = (torch.zeros((3, h_kv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    o, lse = torch.empty_like(q), torch.empty((3, h_q), dtype=torch.float32, device="cuda")
    ws = workspace(3, h_q, h_kv, d, 4096)

    def step():
        binding.mocap_decode_append(store, tables, seq_lens, k, v)
        binding.mocap_decode_attn(store, tables, seq_lens, q, 4096, d ** -0.5, o, lse, ws)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i, lens in enumerate(lens_list):
        seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        for t, seed in ((q, 20 + i), (k, 30 + i), (v, 40 + i)):
            t.copy_(randn(seed, *t.shape))
        ws.fill_(0xFF)
        o.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = o.clone(), lse.clone()
        for b, n in enumerate(lens):
            if n > 0:
                ks[b][n - 1], vs[b][n - 1] = k[b].cpu(), v[b].cpu()
        check(*got, q, ks, vs, lens, d ** -0.5, label=f"replay {i}")
        step()
        torch.cuda.synchronize()
        assert torch.equal(o.view(torch.int16), got[0].view(torch.int16)) and torch.equal(lse, got[1])


def test_two_streams_with_workspaces_of_their_own(gpu):
    lens = [6000, 100]
    store, tables, ks, vs = make_store(19, lens, 256, 2, 64)
    qs = [randn(50 + i, 2, 8, 64).cuda() for i in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    seq_lens = torch.tensor(lens, dtype=torch.int32).cuda()
    outs = [(torch.empty_like(q), torch.empty((2, 8), dtype=torch.float32, device="cuda"),
             workspace(2, 8, 2, 64, 6000)) for q in qs]
    torch.cuda.synchronize()
    for _ in range(20):
        for q, stream, (o, lse, ws) in zip(qs, streams, outs):
            binding.mocap_decode_attn(store, tables, seq_lens, q, 6000, 0.125, o, lse, ws, stream=stream)
    torch.cuda.synchronize()
    for q, (o, lse, _) in zip(qs, outs):
        check(o, lse, q, ks, vs, lens, 0.125)


def test_shared_blocks(gpu):
    """Two sequences with a common prefix in the same physical blocks."""
    store, tables, ks, vs = make_store(21, [300, 200], 64, 2, 64)
    tables[1, :2] = tables[0, :2]
    ks[1][:128], vs[1][:128] = ks[0][:128], vs[0][:128]
    q = randn(22, 2, 4, 64).cuda()
    o, lse = attend(store, tables, [300, 200], q, 300, 0.125)
    check(o, lse, q, ks, vs, [300, 200], 0.125)


def test_refused_calls_write_nothing(gpu):
    store, tables, _, _ = make_store(23, [3000, 200], 64, 2, 64)
    q = randn(24, 2, 4, 64).cuda()
    seq_lens = torch.tensor([3000, 200], dtype=torch.int32).cuda()
    o, lse = torch.full_like(q, 7.0), torch.full((2, 4), 7.0, device="cuda")
    small = torch.empty(64, dtype=torch.uint8, device="cuda")
    for kwargs in (dict(workspace=None), dict(workspace=small)):
        with pytest.raises(binding.MocapError) as err:
            binding.mocap_decode_attn(store, tables, seq_lens, q, 3000, 0.1, o, lse, **kwargs)
        assert err.value.status == binding.MOCAP_ERR_WORKSPACE
    ws = workspace(2, 4, 2, 64, 3000)
    for bad in (dict(window=-1), dict(sinks=-1)):
        with pytest.raises(binding.MocapError):
            binding.mocap_decode_attn(store, tables, seq_lens, q, 3000, 0.1, o, lse, ws, **bad)
    with pytest.raises(binding.MocapError):
        binding.mocap_decode_attn(store, tables, seq_lens, q, 64 * tables.shape[1] + 1, 0.1, o, lse, ws)
    with pytest.raises(binding.MocapError):
        binding.mocap_decode_attn(store, tables, seq_lens, q, 3000, 0.0, o, lse, ws)
    for args in ((tables.long(), seq_lens), (tables, seq_lens.long()), (tables[:1], seq_lens), (tables[0], seq_lens)):
        with pytest.raises((TypeError, ValueError)):
            binding.mocap_decode_attn(store, *args, q, 3000, 0.1, o, lse, ws)
    with pytest.raises(ValueError):
        binding.mocap_decode_attn(store, tables, seq_lens, q, 3000, 0.1, o[:1], lse, ws)
    with pytest.raises(ValueError):
        binding.mocap_decode_attn(store, tables, seq_lens, q.transpose(1, 2), 3000, 0.1, o, lse, ws)
    torch.cuda.synchronize()
    assert (o == 7.0).all() and (lse == 7.0).all()


def test_table_checks_refuse_a_bad_entry(gpu):
    store, tables, _, _ = make_store(25, [200, 200], 64, 2, 64)
    tables[1, 2] = 99
    q = randn(26, 2, 4, 64).cuda()
    o, lse = torch.zeros_like(q), torch.zeros((2, 4), device="cuda")
    binding.set_table_checks(True)
    try:
        with pytest.raises(binding.MocapError):
            binding.mocap_decode_attn(store, tables, torch.tensor([200, 150], dtype=torch.int32).cuda(), q, 200, 0.1, o,
                                      lse)
        # The bad entry is not one that this length or window uses.
        binding.mocap_decode_attn(store, tables, torch.tensor([200, 128], dtype=torch.int32).cuda(), q, 200, 0.1, o, lse)
    finally:
        binding.set_table_checks(False)


def test_offsets_beyond_32_bits(gpu):
    """A store of more than 2^32 bytes per pool, read at its far end."""
    bs, h_kv, d = 256, 8, 128
    blocks = (1 << 32) // (2 * h_kv * bs * d) + 3
    store = binding.KvStore(blocks, bs, h_kv, d)
    small, small_tables, ks, vs = make_store(27, [600], bs, h_kv, d)
    tables = torch.tensor([[blocks - 1, blocks - 3, blocks - 2]], dtype=torch.int32).cuda()
    for i in range(3):
        store.k_pool[tables[0, i].long()] = small.k_pool[small_tables[0, i].long()]
        store.v_pool[tables[0, i].long()] = small.v_pool[small_tables[0, i].long()]
    q = randn(28, 1, 16, d).cuda()
    o, lse = attend(store, tables, [600], q, 600, d ** -0.5)
    check(o, lse, q, ks, vs, [600], d ** -0.5)
    k, v = randn(29, 1, h_kv, d).cuda(), randn(30, 1, h_kv, d).cuda()
    binding.mocap_decode_append(store, tables, torch.tensor([257], dtype=torch.int32).cuda(), k, v)
    torch.cuda.synchronize()
    assert torch.equal(store.k_pool[blocks - 3, :, 0], k[0]) and torch.equal(store.v_pool[blocks - 3, :, :, 0], v[0])


def test_table_checks_of_an_append(gpu):
    """The entry of the last position alone: blocks that left a window may be gone."""
    store, tables, _, _ = make_store(31, [200, 200], 64, 1, 64, fill=0.0)
    tables[0, :3] = -1
    k, v = randn(32, 2, 1, 64).cuda(), randn(33, 2, 1, 64).cuda()
    binding.set_table_checks(True)
    try:
        with pytest.raises(binding.MocapError):
            binding.mocap_decode_append(store, tables, torch.tensor([192, 0], dtype=torch.int32).cuda(), k, v)
        torch.cuda.synchronize()
        before = store.k_pool.clone()
        binding.mocap_decode_append(store, tables, torch.tensor([193, 0], dtype=torch.int32).cuda(), k, v)
    finally:
        binding.set_table_checks(False)
    torch.cuda.synchronize()
    assert torch.equal(store.k_pool[tables[0, 3].long(), 0, 0], k[0, 0])
    before[tables[0, 3].long(), 0, 0] = k[0, 0]
    assert torch.equal(store.k_pool, before)


def test_table_checks_of_an_append_beyond_the_tables(gpu):
    """Nothing is written for a sequence that the tables do not hold: no entry of its is looked at."""
    store, tables, _, _ = make_store(34, [192, 192], 64, 1, 64, fill=0.0)
    tables[0] = -1
    k, v = randn(35, 2, 1, 64).cuda(), randn(36, 2, 1, 64).cuda()
    before = store.k_pool.clone()
    binding.set_table_checks(True)
    try:
        binding.mocap_decode_append(store, tables, torch.tensor([193, 192], dtype=torch.int32).cuda(), k, v)
    finally:
        binding.set_table_checks(False)
    torch.cuda.synchronize()
    before[tables[1, 2].long(), 0, 63] = k[1, 0]
    assert torch.equal(store.k_pool, before)
