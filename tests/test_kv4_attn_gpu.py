"""Attention over the 4-bit store against the plain form in 64 bits, on the values that
the store stands for: batches and chunks, every head layout, windows and sinks, splits,
hidden and visible NaN blocks, long stores, graphs, streams and refusals."""
import math

import pytest
import torch

from cache_helpers import Pools4, make_store4
from helpers import say
from paper_2606_22968_amd import binding
from serve_helpers import B, Attention, check_close, randn

pytestmark = pytest.mark.gpu

# Decoding: a probability enters P V as two bf16 values, what is left is below B^2 of it.
# Chunks: rounded to bf16, and their rounded sum normalises O.
DECODE_ERROR, CHUNK_ERROR = 2.0 ** -16, B


def decode(store, tables, lens, q, max_len, scale, window=0, sinks=0):
    batch, h_q, d = q.shape
    o = torch.full((batch, h_q, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    lse = torch.full((batch, h_q), float("nan"), dtype=torch.float32, device="cuda")
    size = binding.mocap_kv4_decode_attn_workspace_size(batch, h_q, store.h_kv, d, max_len, window, sinks)
    ws = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda").fill_(0xFF)
    seq_lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
    binding.mocap_kv4_decode_attn(store, tables, seq_lens, q, max_len, scale, o, lse, ws, window, sinks)
    return o, lse


def check_decode(o, lse, q, ks, vs, lens, scale, window=0, sinks=0):
    for b, n in enumerate(lens):
        n = max(n, 0)
        ref = Attention(q[b:b + 1].cpu(), ks[b][:n], vs[b][:n], n - 1, scale, window, sinks)
        check_close(o[b:b + 1], ref.o, ref.o_bound(DECODE_ERROR) + 1e-30, f"o[{b}] n={n}")
        check_close(lse[b][:, None], ref.lse, ref.lse_bound(), f"lse[{b}] n={n}")


def chunk(store, table, q, prefix, scale, window=0, sinks=0, splits=0):
    rows, h_q, d = q.shape
    n_ranges, size = binding.mocap_kv4_chunk_attn_workspace_size(prefix, rows, h_q, store.h_kv, d, window, sinks, splits)
    ws = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda").fill_(0xFF)
    o = torch.full((rows, h_q, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    lse = torch.full((h_q, rows), float("nan"), dtype=torch.float32, device="cuda")
    binding.mocap_kv4_chunk_attn(store, table, q, prefix, scale, o, lse, ws, window, sinks, splits)
    return o, lse, n_ranges


def run_chunk(seed, h_q, h_kv, d, bs, prefix, rows, window=0, sinks=0, splits=0):
    """Positions that no row sees hold NaN blocks."""
    n = prefix + rows
    pools, store, tables, ks, vs = make_store4(seed, [n], bs, h_kv, d)
    low = max(0, prefix - window + 1) if window else 0
    for t in range(sinks, low):
        block, slot = tables[0, t // bs].long(), t % bs
        store.k_scale[block, :, slot // 64, :, slot % 64] = 255
        store.v_scale[block, :, slot // 64, :, slot % 64] = 255
    q = randn(seed + 1, rows, h_q, d)
    scale = d ** -0.5
    o, lse, n_ranges = chunk(store, tables[0], q.cuda(), prefix, scale, window, sinks, splits)
    ref = Attention(q, ks[0], vs[0], prefix, scale, window, sinks)
    check_close(o, ref.o, ref.o_bound(CHUNK_ERROR), f"o splits={n_ranges}")
    check_close(lse, ref.lse, ref.lse_bound(), "lse")
    return n_ranges


RAGGED = [1, 0, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300, -3, 511, 512, 513, 700]


@pytest.mark.parametrize("h_q,h_kv,d", [(8, 8, 64), (32, 8, 128), (12, 4, 128), (6, 3, 64), (15, 1, 128), (16, 1, 64),
                                        (17, 1, 128), (32, 1, 128), (33, 1, 64), (64, 1, 64), (40, 1, 128)])
@pytest.mark.parametrize("bs", [64, 192])
def test_ragged_batch(gpu, h_q, h_kv, d, bs):
    say(f"[case] kv4 decode ragged {h_q}/{h_kv}/{d} bs={bs}")
    _, store, tables, ks, vs = make_store4(1, RAGGED, bs, h_kv, d)
    q = randn(2, len(RAGGED), h_q, d).cuda()
    o, lse = decode(store, tables, RAGGED, q, 700, d ** -0.5)
    check_decode(o, lse, q, ks, vs, RAGGED, d ** -0.5)
    assert (o[1] == 0).all() and (lse[1] == -math.inf).all()


@pytest.mark.parametrize("h_q,h_kv,d", [(32, 8, 128), (8, 2, 64), (20, 1, 64)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 3), (64, 0), (64, 64), (100, 4), (100, 65), (129, 130),
                                          (700, 4), (701, 4), (5000, 9), (300, 5000)])
def test_decode_windows(gpu, h_q, h_kv, d, window, sinks):
    lens = [1, 0, 5, 64, 65, 100, 101, 129, 200, 333, 448, 700]
    say(f"[case] kv4 decode window={window} sinks={sinks} {h_q}/{h_kv}/{d}")
    _, store, tables, ks, vs = make_store4(3, lens, 64, h_kv, d)
    for b, n in enumerate(lens):
        for t in range(n):
            if not (t < sinks or t > n - 1 - window):
                block, slot = tables[b, t // 64].long(), t % 64
                store.k_scale[block, :, 0, :, slot] = 255
                store.v_scale[block, :, 0, :, slot] = 255
    q = randn(4, len(lens), h_q, d).cuda()
    o, lse = decode(store, tables, lens, q, 700, d ** -0.5, window, sinks)
    check_decode(o, lse, q, ks, vs, lens, d ** -0.5, window, sinks)


@pytest.mark.parametrize("h_q,h_kv,d", [(20, 1, 64), (32, 1, 128), (40, 2, 128)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 1), (100, 65), (700, 4), (701, 4)])
def test_large_batches(gpu, h_q, h_kv, d, window, sinks):
    """So many sequences that groups of more than 16 heads go 32 at a time; most are empty."""
    lens = [1, 0, 5, 64, 65, 100, 129, 333, 448, 700]
    say(f"[case] kv4 decode large batch window={window} sinks={sinks} {h_q}/{h_kv}/{d}")
    _, store, tables, ks, vs = make_store4(8, lens, 64, h_kv, d)
    for b, n in enumerate(lens):
        for t in range(n):
            if window and not (t < sinks or t > n - 1 - window):
                block, slot = tables[b, t // 64].long(), t % 64
                store.k_scale[block, :, 0, :, slot] = 255
                store.v_scale[block, :, 0, :, slot] = 255
    more = lens + [0] * 3002
    tables = torch.cat((tables, torch.zeros((3002, tables.shape[1]), dtype=torch.int32, device="cuda")))
    q = randn(9, len(more), h_q, d).cuda()
    o, lse = decode(store, tables, more, q, 700, d ** -0.5, window, sinks)
    check_decode(o[:len(lens)], lse[:len(lens)], q[:len(lens)], ks, vs, lens, d ** -0.5, window, sinks)
    assert (o[len(lens):] == 0).all() and (lse[len(lens):] == -math.inf).all()


@pytest.mark.parametrize("lens", [[20000], [9001, 1, 64], [5000, 0, 30000, 257, 12345], [2049] * 70, [1] * 200 + [4000]])
@pytest.mark.parametrize("h_q,h_kv,d,bs", [(4, 1, 128, 256), (8, 2, 64, 1600)])
def test_cut_sequences(gpu, lens, h_q, h_kv, d, bs):
    say(f"[case] kv4 decode cut batch={len(lens)} {h_q}/{h_kv}/{d}")
    _, store, tables, ks, vs = make_store4(5, lens, bs, h_kv, d)
    q = randn(6, len(lens), h_q, d).cuda()
    o, lse = decode(store, tables, lens, q, max(lens), d ** -0.5)
    few = sorted(set(range(min(3, len(lens)))) | {len(lens) - 1})
    for b in few:
        check_decode(o[b:b + 1], lse[b:b + 1], q[b:b + 1], ks[b:b + 1], vs[b:b + 1], lens[b:b + 1], d ** -0.5)
    o2, lse2 = decode(store, tables, lens, q, max(lens), d ** -0.5)
    assert torch.equal(o.view(torch.int16), o2.view(torch.int16)) and torch.equal(lse, lse2)


def test_lengths_beyond_max_len(gpu):
    _, store, tables, ks, vs = make_store4(7, [1000, 700], 64, 2, 64)
    q = randn(8, 2, 4, 64).cuda()
    o, lse = decode(store, tables, [1000, 1 << 30], q, 640, 0.125)
    check_decode(o, lse, q, ks, vs, [640, 640], 0.125)


def growing(seed, n, h_kv, d, bs):
    """Keys whose first dim climbs in powers of two: scores that grow by many binary orders, and fall again."""
    pools = Pools4(-(-n // bs), bs, h_kv, d)
    k, v = randn(seed, n, h_kv, d).float(), randn(seed + 1, n, h_kv, d)
    step = torch.arange(n) % 200
    k[:, :, 0] = torch.where(step < 100, step.float(), 200.0 - step)[:, None] * 0.75
    table = torch.arange(-(-n // bs), dtype=torch.int32)
    k, v = pools.put(table, 0, k, v)
    return pools.to_gpu(), table.cuda(), k.to(torch.bfloat16), v.to(torch.bfloat16)


@pytest.mark.parametrize("d", [64, 128])
def test_growing_scores(gpu, d):
    store, table, k, v = growing(9, 700, 1, d, 64)
    q = randn(10, 90, 3, d)
    q[:, :, 0] = 8.0
    o, lse = decode(store, table[None], [700], q[:1].cuda(), 700, 1.0)
    check_decode(o, lse, q[:1], [k], [v], [700], 1.0)
    for splits in (1, 3):
        o, lse, _ = chunk(store, table, q.cuda(), 610, 1.0, splits=splits)
        ref = Attention(q, k, v, 610, 1.0)
        check_close(o, ref.o, ref.o_bound(CHUNK_ERROR), "o")
        check_close(lse, ref.lse, ref.lse_bound(), "lse")


@pytest.mark.parametrize("h_q,h_kv,d", [(8, 2, 128), (8, 8, 64), (12, 4, 128), (6, 3, 64), (32, 1, 128), (64, 1, 64)])
@pytest.mark.parametrize("prefix,rows,window,sinks", [
    (0, 1, 0, 0), (0, 300, 0, 0), (64, 64, 0, 9), (500, 1, 0, 0), (511, 2, 0, 0), (700, 137, 0, 0), (0, 1, 1, 0),
    (0, 300, 1, 1), (0, 129, 1000, 4), (500, 1, 63, 3), (511, 2, 65, 64), (512, 64, 64, 65), (700, 137, 100, 4),
    (700, 65, 1 << 40, 7), (1000, 30, 128, 1 << 40), (963, 200, 7, 63)])
def test_chunks(gpu, h_q, h_kv, d, prefix, rows, window, sinks):
    say(f"[case] kv4 chunk {h_q}/{h_kv}/{d} P={prefix} L={rows} W={window} sinks={sinks}")
    run_chunk(100, h_q, h_kv, d, 64, prefix, rows, window, sinks)


# Chunks of so many rows that a workgroup takes 256 of them (test_cache_abi.py holds that they do; the others here are
# in blocks of 16 or 32 rows): prefix, rows, window, sinks, splits of 128/16 heads.
MANY = [(0, 300, 0, 0, 0), (0, 300, 1, 1, 0), (0, 300, 1 << 40, 7, 0), (250, 300, 0, 0, 1), (250, 300, 100, 3, 0),
        (250, 299, 65, 64, 2), (511, 131, 63, 65, 3), (700, 137, 0, 0, 3), (963, 290, 1000, 1 << 40, 5), (64, 257, 64, 0, 0),
        (1500, 301, 700, 70, 4)]


# In blocks of 32 rows: heads, head_dim, prefix, rows, window, sinks.
IN_32 = [(32, 1, 128, 200, 500, 64, 64), (32, 1, 128, 1000, 200, 900, 65), (64, 1, 64, 0, 300, 0, 0),
         (64, 1, 64, 2001, 100, 1100, 70), (32, 8, 128, 0, 600, 0, 0), (32, 8, 128, 200, 500, 64, 64),
         (128, 16, 128, 700, 137, 0, 0), (128, 16, 64, 700, 160, 100, 4), (128, 16, 64, 512, 150, 64, 65),
         (128, 16, 128, 250, 150, 100, 3)]


@pytest.mark.parametrize("h_q,h_kv,d,prefix,rows,window,sinks", IN_32)
def test_blocks_of_32_rows(gpu, h_q, h_kv, d, prefix, rows, window, sinks):
    say(f"[case] kv4 chunk in blocks of 32 {h_q}/{h_kv}/{d} P={prefix} L={rows} W={window} sinks={sinks}")
    run_chunk(106, h_q, h_kv, d, 192, prefix, rows, window, sinks)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("prefix,rows,window,sinks,splits", MANY)
def test_many_rows(gpu, d, prefix, rows, window, sinks, splits):
    say(f"[case] kv4 chunk of many rows d={d} P={prefix} L={rows} W={window} sinks={sinks} splits={splits}")
    run_chunk(104, 128, 16, d, 192, prefix, rows, window, sinks, splits)


@pytest.mark.parametrize("window", [1, 2, 33, 64, 65, 129, 192])
@pytest.mark.parametrize("sinks", [0, 1, 64, 65])
def test_window_and_sink_edges_of_many_rows(gpu, window, sinks):
    say(f"[case] kv4 chunk edges of many rows W={window} sinks={sinks}")
    run_chunk(105, 128, 16, 64, 192, 200, 250, window, sinks)


@pytest.mark.parametrize("window", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 191, 192, 193])
@pytest.mark.parametrize("sinks", [0, 1, 63, 64, 65])
def test_window_and_sink_edges(gpu, window, sinks):
    say(f"[case] kv4 chunk edges W={window} sinks={sinks}")
    run_chunk(101, 4, 2, 64, 192, 200, 150, window, sinks)


@pytest.mark.parametrize("splits", [0, 1, 2, 3, 5, 17, 1000])
@pytest.mark.parametrize("h_q,h_kv,d", [(8, 2, 128), (3, 3, 64)])
@pytest.mark.parametrize("window", [0, 1100])
def test_splits(gpu, splits, h_q, h_kv, d, window):
    say(f"[case] kv4 chunk splits={splits} {h_q}/{h_kv}/{d}")
    got = run_chunk(102, h_q, h_kv, d, 128, 2001, 100, window, 70 if window else 0, splits)
    assert splits == 0 or (splits == 1) == (got == 1)


def test_long_chunk_many_workgroups(gpu):
    run_chunk(103, 16, 2, 128, 256, 1000, 700)


def test_same_rows_as_the_bf16_store(gpu):
    """The same values in a bf16 store: chunks, and a decode, within both calls' bounds of 64 bits."""
    pools, store, tables, ks, vs = make_store4(110, [900], 64, 2, 128)
    plain = binding.KvStore(16, 64, 2, 128)
    table = torch.arange(16, dtype=torch.int32, device="cuda")
    loaded = [torch.empty((1, 900, 2, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    binding.mocap_kv4_load(store, tables, torch.tensor([900], dtype=torch.int32, device="cuda"), *loaded)
    assert torch.equal(loaded[0][0].cpu(), ks[0]) and torch.equal(loaded[1][0].cpu(), vs[0])
    binding.mocap_kv_append(plain, table, 0, loaded[0][0], loaded[1][0])
    q = randn(111, 200, 8, 128).cuda()
    o, lse, _ = chunk(store, tables[0], q, 700, 0.1)
    o2, lse2 = torch.empty_like(o), torch.empty_like(lse)
    _, size = binding.mocap_chunk_attn_workspace_size(700, 200, 8, 2, 128, 0)
    binding.mocap_chunk_attn(plain, table, q, 700, 0.1, o2, lse2, torch.empty(max(size, 16), dtype=torch.uint8,
                                                                              device="cuda"))
    ref = Attention(q.cpu(), ks[0], vs[0], 700, 0.1)
    for a, b in ((o, lse), (o2, lse2)):
        check_close(a, ref.o, ref.o_bound(CHUNK_ERROR), "o")
        check_close(b, ref.lse, ref.lse_bound(), "lse")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 3)])
def test_nan_blocks(gpu, d, window, sinks):
    """A NaN value block is NaN in its dims for exactly the rows that see it; a NaN key block makes them NaN."""
    n, prefix, rows, h_q, h_kv = 400, 250, 150, 8, 2
    _, store, tables, ks, vs = make_store4(120, [n], 64, h_kv, d)
    marks = [(0, 0, 1), (0, 2, 0), (0, 170, 1), (1, 249, d // 32 - 1), (0, 300, 0), (1, 383, 1), (1, 399, 0), (1, 320, 1)]
    for h, t, b in marks:
        store.v_scale[tables[0, t // 64].long(), h, 0, b, t % 64] = 255
    k_mark = (1, 340)
    store.k_scale[tables[0, 340 // 64].long(), 1, 0, 1, 340 % 64] = 255
    q = randn(121, rows, h_q, d)

    def sees(pos, t):
        return t <= pos and (window == 0 or t < sinks or t > pos - window)

    def expect(pos, head):
        h, want = head // (h_q // h_kv), torch.zeros(d, dtype=torch.bool)
        for h2, t, b in marks:
            if h2 == h and sees(pos, t):
                want[32 * b:32 * b + 32] = True
        whole = h == k_mark[0] and sees(pos, k_mark[1])
        return want | whole, whole

    for splits in (1, 3):
        o, lse, _ = chunk(store, tables[0], q.cuda(), prefix, 0.1, window, sinks, splits)
        ref = Attention(q, ks[0], vs[0], prefix, 0.1, window, sinks)
        bound = ref.o_bound(CHUNK_ERROR)
        for i in range(rows):
            for g in range(h_q):
                want, whole = expect(prefix + i, g)
                got = o[i, g].cpu()
                assert torch.equal(torch.isnan(got), want), (i, g)
                assert bool(torch.isnan(lse[g, i])) == whole
                assert ((got.double() - ref.o[i, g]).abs() <= bound[i, g])[~want].all()
    for pos in (0, 1, 2, 100, 249, 250, 339, 340, 383, 399):
        o, lse = decode(store, tables, [pos + 1], q[:1].cuda(), n, 0.1, window, sinks)
        ref = Attention(q[:1], ks[0][:pos + 1], vs[0][:pos + 1], pos, 0.1, window, sinks)
        bound = ref.o_bound(DECODE_ERROR)
        for g in range(h_q):
            want, whole = expect(pos, g)
            got = o[0, g].cpu()
            assert torch.equal(torch.isnan(got), want), (pos, g)
            assert bool(torch.isnan(lse[0, g])) == whole
            assert ((got.double() - ref.o[0, g]).abs() <= bound[0, g])[~want].all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 3)])
@pytest.mark.parametrize("rows,splits", [(300, (1, 3)), (150, (0, 2))])
def test_nan_blocks_of_more_rows(gpu, d, window, sinks, rows, splits):
    """As test_nan_blocks, where a workgroup takes 256 rows, and blocks of 32."""
    n, h_q, h_kv = 400, 128, 16
    prefix, group = n - rows, h_q // h_kv
    _, store, tables, ks, vs = make_store4(122, [n], 64, h_kv, d)
    pos = prefix + torch.arange(rows)
    want, whole = torch.zeros((rows, h_q, d), dtype=torch.bool), torch.zeros((rows, h_q), dtype=torch.bool)

    def sees(t):
        return (t <= pos) & ((t > pos - window) if window else True) | (t <= pos) & (t < sinks)

    for h, t, b in [(0, 0, 1), (0, 2, 0), (3, 99, 1), (15, 100, d // 32 - 1), (7, 170, 0), (1, 383, 1), (15, 399, 0), (1, 320, 1)]:
        store.v_scale[tables[0, t // 64].long(), h, 0, b, t % 64] = 255
        want[sees(t), group * h:group * (h + 1), 32 * b:32 * b + 32] = True
    for h, t in [(1, 340), (9, 63)]:
        store.k_scale[tables[0, t // 64].long(), h, 0, 1, t % 64] = 255
        whole[sees(t), group * h:group * (h + 1)] = True
    want |= whole[..., None]
    q = randn(123, rows, h_q, d)
    ref = Attention(q, ks[0], vs[0], prefix, 0.1, window, sinks)
    for num in splits:
        o, lse, _ = chunk(store, tables[0], q.cuda(), prefix, 0.1, window, sinks, num)
        got = o.cpu()
        assert torch.equal(torch.isnan(got), want)
        assert torch.equal(torch.isnan(lse.cpu()), whole.T)
        assert ((got.double() - ref.o).abs() <= ref.o_bound(CHUNK_ERROR))[~want].all()


@pytest.mark.parametrize("fill", [0x00, 0x7F, 0xFC, 0xFD, 0xFE, 0xFF])
@pytest.mark.parametrize("d", [64, 128])
def test_whatever_unwritten_memory_holds(gpu, fill, d):
    """Codes and scales of no position, and of positions behind a row, may be anything: scales beyond those that are
    stored make infinities of their codes."""
    lens = [1, 63, 65, 130]
    _, store, tables, ks, vs = make_store4(190, lens, 192, 2, d, fill=fill)
    q = randn(191, len(lens), 8, d).cuda()
    o, lse = decode(store, tables, lens, q, 192, d ** -0.5)
    check_decode(o, lse, q, ks, vs, lens, d ** -0.5)
    for b, n in enumerate(lens):
        for splits in (1, 2):
            rows = randn(192 + b, n, 8, d)
            o, lse, _ = chunk(store, tables[b].contiguous(), rows.cuda(), 0, d ** -0.5, splits=splits)
            ref = Attention(rows, ks[b], vs[b], 0, d ** -0.5)
            check_close(o, ref.o, ref.o_bound(CHUNK_ERROR), f"o n={n}")
            check_close(lse, ref.lse, ref.lse_bound(), f"lse n={n}")
    _, store, tables, ks, vs = make_store4(198, [300], 192, 16, d, fill=fill)
    rows = randn(199, 300, 128, d)
    ref = Attention(rows, ks[0], vs[0], 0, d ** -0.5)
    for splits in (1, 2):
        o, lse, _ = chunk(store, tables[0], rows.cuda(), 0, d ** -0.5, splits=splits)
        check_close(o, ref.o, ref.o_bound(CHUNK_ERROR), "o of many rows")
        check_close(lse, ref.lse, ref.lse_bound(), "lse of many rows")


def test_rows_of_larger_arrays(gpu):
    """Tables, lengths and LSE need their type's alignment only."""
    _, store, tables, ks, vs = make_store4(195, [300, 300], 64, 2, 64)
    def apart(x):
        return torch.cat((x.flatten()[:1], x.flatten()))[1:].view(x.shape)

    q, lens = randn(196, 2, 4, 64).cuda(), torch.tensor([300, 77], dtype=torch.int32, device="cuda")
    o, lse = torch.empty_like(q), apart(torch.zeros((2, 4), device="cuda"))
    binding.mocap_kv4_decode_attn(store, apart(tables), apart(lens), q, 320, 0.125, o, lse,
                                  torch.empty(1 << 20, dtype=torch.uint8, device="cuda"))
    check_decode(o, lse, q, ks, vs, [300, 77], 0.125)
    rows = randn(197, 40, 4, 64)
    o, lse = torch.empty_like(rows, device="cuda"), apart(torch.zeros((4, 40), device="cuda"))
    assert lse.data_ptr() % 16 == 4
    binding.mocap_kv4_chunk_attn(store, apart(tables[1]), rows.cuda(), 260, 0.125, o, lse,
                                 torch.empty(1 << 20, dtype=torch.uint8, device="cuda"))
    ref = Attention(rows, ks[1], vs[1], 260, 0.125)
    check_close(o, ref.o, ref.o_bound(CHUNK_ERROR), "o")
    check_close(lse, ref.lse, ref.lse_bound(), "lse")


def test_extreme_scales(gpu):
    """Scale bytes 2 and 252, and blocks of zeros, next to ordinary ones."""
    n, d = 130, 64
    pools = Pools4(3, 64, 1, d)
    k, v = randn(130, n, 1, d).float(), randn(131, n, 1, d).float()
    k[3], k[70, :, :32], v[5], v[100, :, 32:] = 0.0, 1e-38, 0.0, 1e-38
    v[129, :, :32] *= 1e37
    table = torch.arange(3, dtype=torch.int32)
    k, v = pools.put(table, 0, k, v)
    store, q = pools.to_gpu(), randn(132, 20, 2, d)
    k, v = k.to(torch.bfloat16), v.to(torch.bfloat16)
    o, lse, _ = chunk(store, table.cuda(), q.cuda(), n - 20, 0.1)
    ref = Attention(q, k, v, n - 20, 0.1)
    check_close(o, ref.o, ref.o_bound(CHUNK_ERROR), "o")
    check_close(lse, ref.lse, ref.lse_bound(), "lse")
    o, lse = decode(store, table[None].cuda(), [n], q[-1:].cuda(), n, 0.1)
    check_decode(o, lse, q[-1:], [k], [v], [n], 0.1)


def test_captured_step(gpu):
    """Append, rotation and attention of a batch in one graph, replayed as its sequences grow past a tile and a block,
    with other work between the replays; two graphs with a workspace each, replayed at once."""
    h_q, h_kv, d, bs, batch = 8, 2, 64, 64, 3
    start = [62, 0, 190]
    _, store, tables, ks, vs = make_store4(140, [200] * batch, bs, h_kv, d, fill=0)
    lens = torch.tensor(start, dtype=torch.int32, device="cuda")
    freq = (10000.0 ** (-torch.arange(0, d, 2) / d)).float()
    rope = binding.Rope(freq.cuda())
    size = binding.mocap_kv4_decode_attn_workspace_size(batch, h_q, h_kv, d, 256)
    q, k, v = (torch.zeros((batch, h, d), dtype=torch.bfloat16, device="cuda") for h in (h_q, h_kv, h_kv))
    outs = []
    graphs = []
    q_rot = torch.zeros_like(q)
    for i in range(2):
        o, lse = torch.zeros_like(q), torch.zeros((batch, h_q), device="cuda")
        ws = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            if i == 0:
                binding.mocap_kv4_decode_append(store, tables, lens, k, v, rope, None, q, q_rot)
            binding.mocap_kv4_decode_attn(store, tables, lens, q_rot, 256, 0.125, o, lse, ws)
        graphs.append(graph)
        outs.append((o, lse, ws))
    streams = [torch.cuda.Stream() for _ in range(2)]
    for step in range(5):
        for i, x in enumerate((q, k, v)):
            x.copy_(randn(150 + 3 * step + i, *x.shape))
        torch.cuda.synchronize()
        graphs[0].replay()
        torch.cuda.synchronize()
        first = [x.clone() for x in outs[0][:2]]
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for o, lse, _ in outs:
            assert torch.equal(o, first[0]) and torch.equal(lse, first[1])
        eager_o, eager_lse = decode(store, tables, lens.tolist(), q_rot, 256, 0.125)
        assert torch.equal(eager_o, first[0]) and torch.equal(eager_lse, first[1])
        loaded = [torch.empty((batch, 256, h_kv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        binding.mocap_kv4_load(store, tables, lens, *loaded)
        for b, n in enumerate(lens.tolist()):
            kb, vb = (x[b, 256 - n:].cpu() for x in loaded)
            check_decode(first[0][b:b + 1], first[1][b:b + 1], q_rot[b:b + 1], [kb], [vb], [n], 0.125)
        lens += (lens > 0).to(torch.int32)


def test_chunk_on_another_stream_and_in_a_graph(gpu):
    _, store, tables, ks, vs = make_store4(160, [700], 64, 2, 128)
    q = randn(161, 60, 8, 128).cuda()
    o, lse, n_ranges = chunk(store, tables[0], q, 640, 0.1, splits=3)
    assert n_ranges > 1
    size = binding.mocap_kv4_chunk_attn_workspace_size(640, 60, 8, 2, 128, num_splits=3)[1]
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    o2, lse2 = torch.zeros_like(o), torch.zeros_like(lse)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    binding.mocap_kv4_chunk_attn(store, tables[0], q, 640, 0.1, o2, lse2, ws, num_splits=3, stream=side)
    side.synchronize()
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.mocap_kv4_chunk_attn(store, tables[0], q, 640, 0.1, o2, lse2, ws, num_splits=3)
    for _ in range(3):
        o2.zero_()
        lse2.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, o2) and torch.equal(lse, lse2)


def test_two_calls_at_once(gpu):
    """Chunks and batches of two streams over one store, with workspaces and outputs of their own."""
    n, rows, d = 3000, 60, 64
    _, store, tables, ks, vs = make_store4(165, [n, n - 100], 64, 2, d)
    lens = torch.tensor([n, n - 100], dtype=torch.int32, device="cuda")
    q, q1 = randn(166, 2, rows, 8, d).cuda(), randn(167, 2, 2, 8, d).cuda()
    chunk_size = binding.mocap_kv4_chunk_attn_workspace_size(n - 100 - rows, rows, 8, 2, d, num_splits=4)[1]
    batch_size = binding.mocap_kv4_decode_attn_workspace_size(2, 8, 2, d, n)
    assert chunk_size > 0 and batch_size > 0
    streams, outs = [torch.cuda.Stream() for _ in range(2)], []
    for i in range(2):
        ws = [torch.empty(x, dtype=torch.uint8, device="cuda") for x in (chunk_size, batch_size)]
        o, lse = torch.empty_like(q[i]), torch.empty((8, rows), device="cuda")
        o1, lse1 = torch.empty_like(q1[i]), torch.empty((2, 8), device="cuda")
        outs.append((ws, o, lse, o1, lse1))
    torch.cuda.synchronize()
    for _ in range(20):
        for i, (ws, o, lse, o1, lse1) in enumerate(outs):
            binding.mocap_kv4_chunk_attn(store, tables[i], q[i], n - 100 - rows, 0.125, o, lse, ws[0], num_splits=4,
                                         stream=streams[i])
            binding.mocap_kv4_decode_attn(store, tables, lens, q1[i], n, 0.125, o1, lse1, ws[1], stream=streams[i])
    torch.cuda.synchronize()
    for i, (_, o, lse, o1, lse1) in enumerate(outs):
        alone = chunk(store, tables[i], q[i], n - 100 - rows, 0.125, splits=4)
        assert torch.equal(o, alone[0]) and torch.equal(lse, alone[1])
        alone = decode(store, tables, lens.tolist(), q1[i], n, 0.125)
        assert torch.equal(o1, alone[0]) and torch.equal(lse1, alone[1])
        check_decode(o1, lse1, q1[i], ks, vs, lens.tolist(), 0.125)


def test_store_beyond_32_bits(gpu):
    """Pools of more than 2^32 bytes: the sequence lies in the last blocks."""
    bs, h_kv, d, n = 1600, 8, 128, 3300
    pools, small, tables, ks, vs = make_store4(170, [n], bs, h_kv, d, spare=0)
    blocks = 6000                                                     # 4.9 GB of codes in each pool
    store = binding.Kv4Store(blocks, bs, h_kv, d)
    table = tables[0] + (blocks - 3)
    for name in Pools4.NAMES:
        getattr(store, name)[blocks - 3:] = getattr(small, name)
    assert store.k_pool.numel() > 1 << 32
    q = randn(171, 40, 16, d)
    o, lse, _ = chunk(store, table, q.cuda(), n - 40, d ** -0.5)
    ref = Attention(q, ks[0], vs[0], n - 40, d ** -0.5)
    check_close(o, ref.o, ref.o_bound(CHUNK_ERROR), "o")
    o, lse = decode(store, table[None], [n], q[-1:].cuda(), n, d ** -0.5)
    check_decode(o, lse, q[-1:], ks, vs, [n], d ** -0.5)
    k, v = randn(172, 70, h_kv, d), randn(173, 70, h_kv, d)
    binding.mocap_kv4_append(store, table, n - 40, k.cuda(), v.cuda())
    pools.put(tables[0], n - 40, k, v)
    binding.mocap_kv4_decode_append(store, table[None], torch.tensor([2], dtype=torch.int32, device="cuda"), k[:1].cuda(),
                                    v[:1].cuda())
    pools.put(tables[0], 1, k[:1], v[:1])
    for name in Pools4.NAMES:
        assert torch.equal(getattr(store, name)[blocks - 3:].cpu(), getattr(pools, name)), name
    far, near = ([torch.empty((1, n + 30, h_kv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)] for _ in range(2))
    ends = torch.tensor([n + 30], dtype=torch.int32, device="cuda")
    binding.mocap_kv4_load(store, table[None], ends, *far)
    binding.mocap_kv4_load(pools.to_gpu(), tables, ends, *near)
    for a, b in zip(far, near):
        assert torch.equal(a, b)


def test_refusals(gpu):
    _, store, tables, _, _ = make_store4(180, [200], 64, 2, 64)
    q = randn(181, 1, 4, 64).cuda()
    o, lse = torch.empty_like(q), torch.empty((1, 4), device="cuda")
    lens = torch.tensor([200], dtype=torch.int32, device="cuda")
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    for bad, error in ((dict(o=o[:, :2].contiguous()), ValueError), (dict(lse=lse.double()), TypeError),
                       (dict(q=q.cpu()), ValueError), (dict(window=-1), binding.MocapError),
                       (dict(scale=0.0), binding.MocapError), (dict(max_len=257), binding.MocapError)):
        args = dict(q=q, max_len=200, scale=0.1, o=o, lse=lse, workspace=ws) | bad
        with pytest.raises(error):
            binding.mocap_kv4_decode_attn(store, tables, lens, **args)
    # Four tiles are never cut and need no workspace, a hundred are.
    assert binding.mocap_kv4_decode_attn_workspace_size(1, 4, 2, 64, 200) == 0
    assert binding.mocap_kv4_decode_attn_workspace_size(1, 4, 2, 64, 6400) > 0
    wide = tables.repeat(1, 25)
    for short in (None, ws[:1024]):
        with pytest.raises(binding.MocapError):
            binding.mocap_kv4_decode_attn(store, wide, lens, q, 6400, 0.1, o, lse, short)
    lse_c = torch.empty((4, 1), device="cuda")
    for bad, error in ((dict(lse=lse), ValueError), (dict(prefix_len=256), binding.MocapError),
                       (dict(window=-1), binding.MocapError), (dict(sinks=-1), binding.MocapError),
                       (dict(num_splits=2, workspace=None), binding.MocapError)):
        args = dict(q=q, prefix_len=199, scale=0.1, o=o, lse=lse_c, workspace=ws) | bad
        with pytest.raises(error):
            binding.mocap_kv4_chunk_attn(store, tables[0], **args)
    wrong = binding.Kv4Store(4, 64, 2, 64)
    wrong.k_scale = wrong.k_scale.cpu()
    with pytest.raises(ValueError):
        binding.mocap_kv4_decode_attn(wrong, tables, lens, q, 200, 0.1, o, lse, ws)
