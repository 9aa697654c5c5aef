"""The rotating appends against the plain form in 64 bits: both stores, both orders of
pairs, some or all dims, chunks from any slot, batches with empty rows, strided rows,
far positions, graphs, streams and refusals."""
import pytest
import torch

from cache_helpers import Pools4, inv_freq, quantise, rotate, values
from helpers import say
from paper_2606_22968_amd import binding
from serve_helpers import B, U, check_close, put, randn

pytestmark = pytest.mark.gpu


def rotated_bound(want, size):
    """bf16 rounding of the result, B of it; before that the fp32 cosine and sine, off by at most 4 u (the polynomial's
    steps and the angle's rounding to fp32, u pi / 4), and the products and their sum, 2 u of each: 6 u (|x| + |y|),
    taken as 8."""
    return B * want.abs() * (1 + B) + 8 * U * size + 1e-30


def tokens(seed, n, h_q, h_kv, d, fused):
    """q, k, v of n tokens on the GPU: parts of one tensor's rows, or tensors of their own."""
    if fused:
        rows = randn(seed, n, h_q + 2 * h_kv, d).cuda()
        return rows[:, :h_q], rows[:, h_q:h_q + h_kv], rows[:, h_q + h_kv:]
    return randn(seed, n, h_q, d).cuda(), randn(seed + 1, n, h_kv, d).cuda(), randn(seed + 2, n, h_kv, d).cuda()


def rope_of(rot, interleaved, theta=10000.0):
    if rot == 0:
        return None, None
    freq = inv_freq(rot, theta)
    return binding.Rope(freq.cuda(), interleaved), freq


def same_bits(a, b):
    return torch.equal(a.cpu().view(torch.int16), b.cpu().view(torch.int16))


def chunk(four, h_q, h_kv, d, bs, start, n, rot, interleaved, shift=0, fused=True, seed=1, theta=10000.0):
    blocks = -(-(start + n) // bs) + 2
    table = torch.randperm(blocks, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    q, k, v = tokens(seed + 10, n, h_q, h_kv, d, fused)
    rope, freq = rope_of(rot, interleaved, theta)
    at = start + shift + torch.arange(n)
    q_out = torch.full((n, h_q, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    want_k, k_size = rotate(k.cpu(), at, freq, interleaved)
    want_q, q_size = rotate(q.cpu(), at, freq, interleaved)
    call = dict(position=None if shift == 0 else start + shift, q=q, q_out=q_out)
    if four:
        pools = Pools4(blocks, bs, h_kv, d, fill=0xA5)
        store = pools.to_gpu()
        binding.mocap_kv4_append(store, table.cuda(), start, k, v, rope, **call)
        # In 64 bits the result is within 1e-15 of the exact one, and no value of these inputs is that near a border.
        pools.put(table, start, want_k, v.cpu())
        pools.same_as(store, "4-bit append")
    else:
        store = binding.KvStore(blocks, bs, h_kv, d, fill=-7.0)
        binding.mocap_rope_append(store, table.cuda(), start, k, v, rope, **call)
        k_pool, v_pool = torch.full_like(store.k_pool, -7.0).cpu(), torch.full_like(store.v_pool, -7.0).cpu()
        pos = start + torch.arange(n)
        block, slot = table.long()[pos // bs], pos % bs
        got = store.k_pool.cpu()[block, :, slot]
        check_close(got, want_k, rotated_bound(want_k, k_size), "k")
        assert same_bits(got[..., rot:], k[..., rot:].contiguous())
        put(k_pool, v_pool, table, bs, start, got, v.cpu())     # everything else is as it was
        assert same_bits(store.k_pool, k_pool) and same_bits(store.v_pool, v_pool)
    if h_q:
        check_close(q_out, want_q, rotated_bound(want_q, q_size), "q")
        assert same_bits(q_out[..., rot:].contiguous(), q[..., rot:].contiguous())


LAYOUTS = [(32, 8, 128), (8, 8, 64), (12, 4, 128), (6, 3, 64), (7, 1, 128), (64, 1, 64)]


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("h_q,h_kv,d", LAYOUTS)
@pytest.mark.parametrize("start,n", [(0, 1), (0, 64), (63, 1), (63, 2), (70, 137), (1, 63), (129, 300)])
def test_chunks(gpu, four, h_q, h_kv, d, start, n):
    say(f"[case] rope chunk four={four} {h_q}/{h_kv}/{d} start={start} n={n}")
    chunk(four, h_q, h_kv, d, 192, start, n, d, False, fused=n % 2 == 0)


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rot", [(64, r) for r in range(0, 65, 16)] + [(128, r) for r in range(0, 129, 16)])
def test_rotated_dims(gpu, four, interleaved, d, rot):
    say(f"[case] rope four={four} interleaved={interleaved} {rot} of {d}")
    chunk(four, 4, 2, d, 64, 61, 70, rot, interleaved, shift=5000 if rot else 0)


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("position", [0, 131072, 1 << 24, (1 << 29) + 12345, (1 << 31) - 128 - 20])
def test_far_positions(gpu, four, position):
    """Slots from 5 on, angles of any size (the largest 2^31 radians)."""
    say(f"[case] rope four={four} position={position}")
    chunk(four, 4, 1, 128, 64, 5, 20, 128, False, shift=position - 5, theta=1000000.0)


@pytest.mark.parametrize("four", [False, True])
def test_no_queries_and_no_tokens(gpu, four):
    pools = Pools4(3, 64, 2, 64, fill=7)
    store = pools.to_gpu() if four else binding.KvStore(3, 64, 2, 64, fill=1.0)
    append = binding.mocap_kv4_append if four else binding.mocap_rope_append
    table = torch.tensor([2, 0], dtype=torch.int32, device="cuda")
    rope, _ = rope_of(64, False)
    k, v = randn(1, 20, 2, 64).cuda(), randn(2, 20, 2, 64).cuda()
    append(store, table, 128, k[:0], v[:0], rope)
    if four:
        pools.same_as(store, "no tokens")
    append(store, table, 50, k, v, rope)
    if four:
        pools.put(table, 50, rotate(k.cpu(), 50 + torch.arange(20), inv_freq(64), False)[0], v.cpu())
        pools.same_as(store, "no queries")


@pytest.mark.parametrize("four", [False, True])
def test_in_place_queries(gpu, four):
    q, k, v = tokens(3, 70, 4, 2, 128, False)
    rope, _ = rope_of(128, True)
    table = torch.tensor([1, 0], dtype=torch.int32, device="cuda")
    append = binding.mocap_kv4_append if four else binding.mocap_rope_append
    store = binding.Kv4Store(2, 64, 2, 128, fill=0) if four else binding.KvStore(2, 64, 2, 128, fill=0.0)
    out = torch.empty_like(q)
    append(store, table, 9, k, v, rope, 9, q, out)
    append(store, table, 9, k, v, rope, 9, q, q)
    assert same_bits(out, q)


LENS = [1, 0, 64, 65, -3, 129, 190, 700, 1 << 30, 192]


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("h_q,h_kv,d", LAYOUTS)
@pytest.mark.parametrize("rot,interleaved,given", [("all", False, False), ("half", True, True), (16, False, True)])
def test_batches(gpu, four, h_q, h_kv, d, rot, interleaved, given):
    """Rows without a sequence, and one longer than the tables hold, leave everything as it was."""
    rot = {"all": d, "half": d // 2}.get(rot, rot)
    say(f"[case] rope batch four={four} {h_q}/{h_kv}/{d} rot={rot}")
    bs, batch, stride = 64, len(LENS), 11
    perm = torch.randperm(batch * stride, generator=torch.Generator().manual_seed(5)).to(torch.int32)
    tables = perm.reshape(batch, stride)
    seq_lens = torch.tensor(LENS, dtype=torch.int32)
    positions = torch.tensor([7 * i * i + 3 for i in range(batch)], dtype=torch.int32) if given else None
    q, k, v = tokens(6, batch, h_q, h_kv, d, True)
    rope, freq = rope_of(rot, interleaved)
    pools = Pools4(batch * stride, bs, h_kv, d, fill=0x33)
    store = pools.to_gpu() if four else binding.KvStore(batch * stride, bs, h_kv, d, fill=-7.0)
    q_out = torch.full((batch, h_q, d), 9.0, dtype=torch.bfloat16, device="cuda")
    append = binding.mocap_kv4_decode_append if four else binding.mocap_decode_rope_append
    append(store, tables.cuda(), seq_lens.cuda(), k, v, rope, None if positions is None else positions.cuda(), q, q_out)
    at = (seq_lens - 1) if positions is None else positions
    want_k, k_size = rotate(k.cpu(), at, freq, interleaved)
    want_q, q_size = rotate(q.cpu(), at, freq, interleaved)
    if not four:
        k_pool, v_pool = torch.full_like(store.k_pool, -7.0).cpu(), torch.full_like(store.v_pool, -7.0).cpu()
        got_pool = store.k_pool.cpu()
    for b, n in enumerate(LENS):
        if not 0 < n <= stride * bs:
            assert (q_out[b] == 9.0).all()
            continue
        check_close(q_out[b], want_q[b], rotated_bound(want_q[b], q_size[b]), f"q[{b}]")
        if four:
            pools.put(tables[b], n - 1, want_k[b:b + 1], v[b:b + 1].cpu())
        else:
            got = got_pool[tables[b, (n - 1) // bs].long(), :, (n - 1) % bs][None]
            check_close(got[0], want_k[b], rotated_bound(want_k[b], k_size[b]), f"k[{b}]")
            put(k_pool, v_pool, tables[b], bs, n - 1, got, v[b:b + 1].cpu())
    if four:
        pools.same_as(store, "4-bit batch")
    else:
        assert same_bits(store.k_pool, k_pool) and same_bits(store.v_pool, v_pool)


@pytest.mark.parametrize("four", [False, True])
def test_positions_of_either_sign(gpu, four):
    """A batch's rotation positions are any int32, apart from the slots."""
    at = torch.tensor([-1, -(1 << 31), (1 << 31) - 1, -70000, 0], dtype=torch.int32)
    batch, h_kv, d, bs = at.numel(), 2, 64, 64
    lens = torch.arange(1, batch + 1, dtype=torch.int32)
    tables = torch.arange(batch, dtype=torch.int32)[:, None].contiguous()
    rope, freq = rope_of(d, False)
    q, k, v = tokens(70, batch, 4, h_kv, d, True)
    q_out = torch.empty((batch, 4, d), dtype=torch.bfloat16, device="cuda")
    want_k, k_size = rotate(k.cpu(), at, freq, False)
    want_q, q_size = rotate(q.cpu(), at, freq, False)
    if four:
        pools = Pools4(batch, bs, h_kv, d, fill=0)
        store = pools.to_gpu()
        binding.mocap_kv4_decode_append(store, tables.cuda(), lens.cuda(), k, v, rope, at.cuda(), q, q_out)
        for b in range(batch):
            pools.put(tables[b], int(lens[b]) - 1, want_k[b:b + 1], v[b:b + 1].cpu())
        pools.same_as(store, "either sign")
    else:
        store = binding.KvStore(batch, bs, h_kv, d, fill=0.0)
        binding.mocap_decode_rope_append(store, tables.cuda(), lens.cuda(), k, v, rope, at.cuda(), q, q_out)
        got = store.k_pool.cpu()[torch.arange(batch), :, lens.long() - 1]
        check_close(got, want_k, rotated_bound(want_k, k_size), "k")
    check_close(q_out, want_q, rotated_bound(want_q, q_size), "q")


def test_store_beyond_32_bits(gpu):
    """A bf16 store of more than 2^32 values a pool: the positions lie in the last blocks."""
    bs, h_kv, d, blocks = 1600, 8, 128, 2700
    store = binding.KvStore(blocks, bs, h_kv, d)
    assert store.k_pool.numel() > 1 << 32
    store.k_pool[-2:], store.v_pool[-2:] = 0.0, 0.0
    table = torch.tensor([blocks - 1, blocks - 2], dtype=torch.int32)
    rope, freq = rope_of(d, False)
    k, v = randn(80, 71, h_kv, d), randn(81, 71, h_kv, d)
    binding.mocap_rope_append(store, table.cuda(), bs - 40, k[:70].cuda(), v[:70].cuda(), rope)
    binding.mocap_decode_rope_append(store, table[None].cuda(), torch.tensor([bs + 31], dtype=torch.int32, device="cuda"),
                                     k[70:].cuda(), v[70:].cuda(), rope)
    at = bs - 40 + torch.arange(71)
    want, size = rotate(k, at, freq, False)
    small_k, small_v = store.k_pool[-2:].cpu(), store.v_pool[-2:].cpu()
    near = table - (blocks - 2)
    got = small_k[near.long()[at // bs], :, at % bs]
    check_close(got, want, rotated_bound(want, size), "k")
    k_pool, v_pool = torch.zeros_like(small_k), torch.zeros_like(small_v)
    put(k_pool, v_pool, near, bs, bs - 40, got, v)
    assert same_bits(small_k, k_pool) and same_bits(small_v, v_pool)


def test_rounding_to_four_bits(gpu):
    """Every border between codes and scales, in blocks of their own: exact ties, their neighbours in bf16, powers of
    two, the least and the largest magnitudes, zeros of both signs, NaN and infinities."""
    d, rows = 64, []
    edges = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 3.0, 0.5, 4.0]
    for top in (6.0, 4.0, 3.0, 3.015625, 5.96875, 6.03125):
        near = [torch.tensor(x, dtype=torch.bfloat16) for x in edges]
        bits = torch.stack(near).view(torch.int16)
        row = torch.cat((bits - 1, bits, bits + 1)).view(torch.bfloat16)[:31]
        rows.append(torch.cat((row.clamp(max=top), torch.tensor([top], dtype=torch.bfloat16))))
    rows = torch.stack(rows)
    rows = torch.cat((rows, -rows, rows * 2.0 ** -20, rows * 2.0 ** 60))
    tiny = torch.zeros(32, dtype=torch.bfloat16)
    tiny[:4] = torch.tensor([1e-38, -3e-39, 2.0 ** -126, -0.0], dtype=torch.bfloat16)
    big = torch.full((32,), 3.3e38, dtype=torch.bfloat16)
    big[1], big[2] = -2.5e38, 1.0
    odd = [torch.zeros(32, dtype=torch.bfloat16), tiny, big]
    for bad in (float("nan"), float("inf"), -float("inf")):
        x = torch.ones(32, dtype=torch.bfloat16)
        x[13] = bad
        odd.append(x)
    rows = torch.cat((rows, torch.stack(odd)))
    x = torch.cat((rows, rows.flip(0)), 1)[:, None]                    # [n][1][64]: two blocks a position
    n = x.shape[0]
    pools = Pools4(2, 64, 1, d, fill=0)
    store = pools.to_gpu()
    table = torch.tensor([1], dtype=torch.int32)
    binding.mocap_kv4_append(store, table.cuda(), 0, x.cuda(), x.flip(2).contiguous().cuda())
    pools.put(table, 0, x, x.flip(2))
    pools.same_as(store, "borders")
    k, v = (torch.empty((1, n, 1, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    binding.mocap_kv4_load(store, table[None].cuda(), torch.tensor([n], dtype=torch.int32).cuda(), k, v)
    for got, want in ((k, x), (v, x.flip(2))):
        want = values(*quantise(want))
        assert torch.equal(torch.isnan(got[0].cpu()), torch.isnan(want))
        assert torch.equal(got[0].cpu().double().nan_to_num(), want.nan_to_num())


@pytest.mark.parametrize("h_kv,d,bs", [(2, 128, 64), (3, 64, 192)])
@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 200])
def test_load(gpu, h_kv, d, bs, n):
    """The last n of each sequence: fewer than n, none, tiles' edges, and ends beyond the tables."""
    say(f"[case] load {h_kv}/{d} n={n}")
    ends = [1, 64, 65, 0, 130, 200, -5, 1 << 30, 384]
    pools = Pools4(len(ends) * 6, bs, h_kv, d)
    tables = torch.randperm(len(ends) * 6, generator=torch.Generator().manual_seed(n)).to(torch.int32).reshape(-1, 6)
    stored = []
    for b, end in enumerate(ends):
        m = end if 0 < end <= 6 * bs else 0
        k, v = (randn(20 + b, max(m, 1), h_kv, d)[:m] for _ in range(2))
        stored.append(pools.put(tables[b], 0, k, v) if m else None)
    store = pools.to_gpu()
    k, v = (torch.full((len(ends), n, h_kv, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    binding.mocap_kv4_load(store, tables.cuda(), torch.tensor(ends, dtype=torch.int32).cuda(), k, v)
    for b, both in enumerate(stored):
        for got, want in zip((k, v), both or (torch.zeros((0, h_kv, d), dtype=torch.float64),) * 2):
            padded = torch.zeros((n, h_kv, d), dtype=torch.float64)
            m = min(n, want.shape[0])
            padded[n - m:] = want[want.shape[0] - m:]
            assert torch.equal(got[b].cpu().double(), padded), f"sequence {b}"


def test_captured_steps(gpu):
    """A captured append, replayed as lengths and positions move on, with other work between the replays."""
    lens = torch.tensor([5, 63, 0, 127], dtype=torch.int32, device="cuda")
    positions = torch.tensor([500, 7, 0, 90000], dtype=torch.int32, device="cuda")
    tables = torch.arange(12, dtype=torch.int32, device="cuda").reshape(4, 3)
    rope, freq = rope_of(128, False)
    q, k, v = (x.contiguous() for x in tokens(31, 4, 8, 2, 128, False))
    q_out = torch.zeros_like(q)
    pools = Pools4(12, 64, 2, 128, fill=0)
    store = pools.to_gpu()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.mocap_kv4_decode_append(store, tables, lens, k, v, rope, positions, q, q_out)
    for step in range(4):
        for i, x in enumerate((q, k, v)):
            x.copy_(randn(40 + 3 * step + i, *x.shape))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want_k, _ = rotate(k.cpu(), positions.cpu(), freq, False)
        want_q, size = rotate(q.cpu(), positions.cpu(), freq, False)
        for b, n in enumerate(lens.tolist()):
            if n > 0:
                pools.put(tables[b].cpu(), n - 1, want_k[b:b + 1], v[b:b + 1].cpu())
                check_close(q_out[b], want_q[b], rotated_bound(want_q[b], size[b]), f"q[{b}] step {step}")
        pools.same_as(store, f"step {step}")
        lens += (lens > 0).to(torch.int32)
        positions += 1


def test_another_stream(gpu):
    """Enqueued on the stream that is given, behind its work."""
    side = torch.cuda.Stream()
    k, v = randn(50, 100, 2, 64).cuda(), randn(51, 100, 2, 64).cuda()
    late_k = torch.zeros_like(k)
    pools = Pools4(2, 64, 2, 64, fill=0)
    store = pools.to_gpu()
    table = torch.tensor([1, 0], dtype=torch.int32, device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(20000000)
        late_k.copy_(k)
    binding.mocap_kv4_append(store, table, 3, late_k, v, stream=side)
    side.synchronize()
    pools.put(table, 3, k.cpu(), v.cpu())
    pools.same_as(store, "side stream")


def test_refusals(gpu):
    store4, store = binding.Kv4Store(2, 64, 2, 64, fill=0), binding.KvStore(2, 64, 2, 64, fill=0.0)
    table = torch.tensor([1, 0], dtype=torch.int32, device="cuda")
    lens = torch.tensor([1] * 4, dtype=torch.int32, device="cuda")
    tables = torch.zeros((4, 2), dtype=torch.int32, device="cuda")
    q, k, v = tokens(60, 4, 4, 2, 64, True)
    rope, _ = rope_of(64, False)
    out = torch.empty((4, 4, 64), dtype=torch.bfloat16, device="cuda")
    half = binding.Rope(torch.ones(12, device="cuda"))
    for append, s in ((binding.mocap_kv4_append, store4), (binding.mocap_rope_append, store)):
        append(s, table, 0, k, v, rope, 0, q, out)
        for bad, error in ((dict(k=k.float()), TypeError), (dict(k=k.cpu()), ValueError), (dict(k=k[:3]), ValueError),
                           (dict(k=k.transpose(1, 2)), ValueError), (dict(v=v[:, :1]), ValueError),
                           (dict(q=q[:, :, :32]), ValueError), (dict(q_out=None), TypeError),
                           (dict(q_out=out[:3]), ValueError), (dict(q=None), ValueError),
                           (dict(q=q[:, :3], q_out=out[:, :3].contiguous()), binding.MocapError),
                           (dict(rope=half), binding.MocapError), (dict(position=-1), binding.MocapError),
                           (dict(position=(1 << 31) - 128), binding.MocapError), (dict(start_pos=125), binding.MocapError),
                           (dict(start_pos=-1), binding.MocapError)):
            args = dict(start_pos=0, k=k, v=v, rope=rope, position=0, q=q, q_out=out) | bad
            with pytest.raises(error):
                append(s, table, **args)
    for append, s in ((binding.mocap_kv4_decode_append, store4), (binding.mocap_decode_rope_append, store)):
        append(s, tables, lens * 0, k, v, rope, None, q, out)
        for bad, error in ((dict(k=k[:3], v=v[:3], q=None, q_out=None), ValueError),
                           (dict(positions=lens.long()), TypeError), (dict(positions=lens[:2]), ValueError),
                           (dict(rope=half), binding.MocapError)):
            args = dict(k=k, v=v, rope=rope, positions=None, q=q, q_out=out) | bad
            with pytest.raises(error):
                append(s, tables, lens * 0, **args)
    kl = torch.empty((4, 3, 2, 64), dtype=torch.bfloat16, device="cuda")
    for args in ((kl[:3], kl[:3]), (kl, kl[:, :2].contiguous()), (kl[..., :32].contiguous(),) * 2):
        with pytest.raises(ValueError):
            binding.mocap_kv4_load(store4, tables, lens, *args)
