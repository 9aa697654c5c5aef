"""mocap_key_weights and mocap_decode_key_weights against the plain form in 64
bits: chunks of one row to many, every head layout, accumulation over a prompt,
padded batches, non-finite inputs, graphs and refusals."""
import math

import pytest
import torch

from helpers import say
from paper_2606_22968_amd import binding
from serve_helpers import U, Attention, Weights, check_close, make_store, randn

pytestmark = pytest.mark.gpu


def call(store, table, q, prefix, scale, lse, prev, weights):
    rows, h_q, d = q.shape
    size = binding.mocap_key_weights_workspace_size(prefix, rows, h_q, store.h_kv, d)
    ws = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda").fill_(0xFF)
    binding.mocap_key_weights(store, table, q, prefix, scale, lse, prev, weights, ws)


def base(seed, *shape):
    g = torch.Generator(device="cpu")
    g.manual_seed(seed)
    return torch.rand(shape, generator=g) * 3


HEADS = [(32, 8, 128), (8, 8, 64), (12, 4, 128), (6, 3, 64), (32, 1, 128), (64, 1, 64), (5, 1, 64)]


@pytest.mark.parametrize("h_q,h_kv,d", HEADS)
@pytest.mark.parametrize("prefix,rows", [(0, 1), (0, 33), (1, 1), (63, 1), (64, 2), (100, 31), (511, 65), (0, 513),
                                         (1500, 7), (700, 200)])
def test_chunks(gpu, h_q, h_kv, d, prefix, rows):
    say(f"[case] key weights {h_q}/{h_kv}/{d} P={prefix} L={rows}")
    n = prefix + rows
    store, tables, ks, vs = make_store(200, [n], 64, h_kv, d)
    q, scale = randn(201, rows, h_q, d), d ** -0.5
    lse = Attention(q, ks[0], vs[0], prefix, scale).lse.float()
    prev = base(202, h_kv, n + 5)
    prev[:, prefix:] = float("nan")  # weights of keys that are new: not read
    weights = torch.full((h_kv, n + 5), 7.0, device="cuda")
    call(store, tables[0], q.cuda(), prefix, scale, lse.cuda(), prev.cuda(), weights)
    ref = Weights(q, ks[0], prefix, scale, lse, prev)
    check_close(weights[:, :n], ref.w, ref.bound, "with prev")
    assert (weights[:, n:] == 7.0).all()
    # In place, and without former weights.
    again = prev.cuda()
    call(store, tables[0], q.cuda(), prefix, scale, lse.cuda(), again, again)
    assert torch.equal(again[:, :n], weights[:, :n])
    call(store, tables[0], q.cuda(), prefix, scale, lse.cuda(), None, weights)
    ref = Weights(q, ks[0], prefix, scale, lse)
    check_close(weights[:, :n], ref.w, ref.bound, "alone")
    # Every row gives a weight of 1 in all.
    assert abs(float(weights[:, :n].double().sum()) - rows * h_q) <= float(ref.bound.sum()) + rows * h_q * 1e-5


@pytest.mark.parametrize("h_q,h_kv,d,prefix,rows", [(8, 2, 128, 20000, 40), (4, 4, 64, 30001, 3), (16, 1, 128, 9000, 300),
                                                    (2, 1, 64, 3000, 2000), (64, 1, 64, 100, 900)])
def test_larger(gpu, h_q, h_kv, d, prefix, rows):
    """Every number of wavefronts along the keys, and rows in parts."""
    say(f"[case] key weights larger {h_q}/{h_kv}/{d} P={prefix} L={rows}")
    n = prefix + rows
    store, tables, ks, vs = make_store(203, [n], 192, h_kv, d)
    q, scale = randn(204, rows, h_q, d), d ** -0.5
    # Any LSE will do as an input: near the rows' own.
    lse = math.log(n) + 0.5 + 0.1 * base(205, h_q, rows)
    weights = torch.zeros((h_kv, n), device="cuda")
    call(store, tables[0], q.cuda(), prefix, scale, lse.cuda(), None, weights)
    ref = Weights(q, ks[0], prefix, scale, lse)
    check_close(weights, ref.w, ref.bound, "larger")
    first = weights.clone()
    call(store, tables[0], q.cuda(), prefix, scale, lse.cuda(), None, weights)
    assert torch.equal(first, weights)


def test_accumulates_over_a_prompt(gpu):
    """Chunk after chunk, in place, from an uninitialised buffer: the whole prompt's weights."""
    lengths = [100, 1, 70, 129]
    n, h_q, h_kv, d = 300, 8, 2, 64
    store, tables, ks, vs = make_store(206, [n], 64, h_kv, d)
    q, scale = randn(207, n, h_q, d), 0.125
    lse = Attention(q, ks[0], vs[0], 0, scale).lse.float()
    weights = torch.full((h_kv, n), float("nan"), device="cuda")
    p = 0
    for c in lengths:
        call(store, tables[0], q[p:p + c].cuda(), p, scale, lse[:, p:p + c].contiguous().cuda(), weights, weights)
        p += c
    ref = Weights(q, ks[0], 0, scale, lse)
    check_close(weights, ref.w, ref.bound * 2, "prompt")


def test_special_rows(gpu):
    """Rows without a visible key add nothing; NaN reaches the keys its row or key has."""
    n, rows, prefix = 200, 40, 160
    store, tables, ks, vs = make_store(208, [n], 64, 1, 64)
    q = randn(209, rows, 2, 64)
    lse = Attention(q, ks[0], vs[0], prefix, 0.125).lse.float()
    lse[0, 5], lse[1, 6] = -math.inf, math.inf
    weights = torch.zeros((1, n), device="cuda")
    call(store, tables[0], q.cuda(), prefix, 0.125, lse.cuda(), None, weights)
    ref = Weights(q, ks[0], prefix, 0.125, lse)
    check_close(weights, ref.w, ref.bound, "infinite LSE")
    lse[1, 20] = float("nan")  # the row at position 180
    q[30, 0, 0] = float("nan")  # at position 190
    store.k_pool[tables[0, 3].long(), 0, 3] = float("nan")  # key 195, seen by rows of 195 and later
    call(store, tables[0], q.cuda(), prefix, 0.125, lse.cuda(), None, weights)
    want = torch.zeros(1, n, dtype=torch.bool)
    want[0, :191] = True
    want[0, 195] = True
    assert torch.equal(torch.isnan(weights).cpu(), want)


def test_unwritten_memory_and_hidden_keys(gpu):
    """NaN in the rest of the last block, and a NaN key that only later rows see."""
    store, tables, ks, vs = make_store(210, [130], 64, 2, 128)
    q = randn(211, 30, 4, 128)
    lse = Attention(q, ks[0], vs[0], 100, 0.09).lse.float()
    weights = torch.zeros((2, 130), device="cuda")
    call(store, tables[0], q.cuda(), 100, 0.09, lse.cuda(), None, weights)
    ref = Weights(q, ks[0], 100, 0.09, lse)
    check_close(weights, ref.w, ref.bound, "unwritten")
    assert torch.isfinite(weights).all()


RAGGED = [1, 0, 2, 63, 64, 65, 128, 129, -4, 300, 511, 700]


@pytest.mark.parametrize("h_q,h_kv,d", HEADS + [(17, 1, 128), (40, 1, 64)])
def test_decode_batch(gpu, h_q, h_kv, d):
    say(f"[case] decode key weights {h_q}/{h_kv}/{d}")
    store, tables, ks, vs = make_store(212, RAGGED, 64, h_kv, d)
    q, scale = randn(213, len(RAGGED), h_q, d), d ** -0.5
    lse = torch.full((len(RAGGED), h_q), -math.inf)
    for b, n in enumerate(RAGGED):
        if n > 0:
            lse[b] = Attention(q[b:b + 1], ks[b], vs[b], n - 1, scale).lse[:, 0].float()
    prev = base(214, len(RAGGED), h_kv, 750)
    for b, n in enumerate(RAGGED):
        prev[b, :, max(n - 1, 0):] = float("nan")
    weights = torch.full((len(RAGGED), h_kv, 750), 7.0, device="cuda")
    seq_lens = torch.tensor(RAGGED, dtype=torch.int32).cuda()
    binding.mocap_decode_key_weights(store, tables, seq_lens, q.cuda(), 700, scale, lse.cuda(), prev.cuda(), weights)
    for b, n in enumerate(RAGGED):
        n = max(n, 0)
        assert (weights[b, :, n:] == 7.0).all()
        if n > 0:
            ref = Weights(q[b:b + 1], ks[b], n - 1, scale, lse[b][:, None], prev[b])
            check_close(weights[b, :, :n], ref.w, ref.bound, f"sequence {b}")
    again = prev.cuda()
    binding.mocap_decode_key_weights(store, tables, seq_lens, q.cuda(), None if tables.shape[1] * 64 <= 750 else 700,
                                     scale, lse.cuda(), again, again)
    for b, n in enumerate(RAGGED):
        assert torch.equal(again[b, :, :max(n, 0)], weights[b, :, :max(n, 0)])


def test_decode_equals_chunk_of_one(gpu):
    lens = [9000, 5, 3000]
    store, tables, ks, vs = make_store(215, lens, 256, 2, 128)
    q = randn(216, 3, 8, 128).cuda()
    lse = math.log(9000) + 0.1 * base(217, 3, 8)
    weights = torch.zeros((3, 2, 9000), device="cuda")
    binding.mocap_decode_key_weights(store, tables, torch.tensor(lens, dtype=torch.int32).cuda(), q, 9000, 0.09,
                                     lse.cuda(), None, weights)
    for b, n in enumerate(lens):
        one = torch.zeros((2, n), device="cuda")
        call(store, tables[b], q[b:b + 1], n - 1, 0.09, lse[b][:, None].contiguous().cuda(), None, one)
        ref = Weights(q[b:b + 1].cpu(), ks[b], n - 1, 0.09, lse[b][:, None])
        check_close(weights[b, :, :n], ref.w, ref.bound, f"batch {b}")
        check_close(one, ref.w, ref.bound, f"chunk {b}")


def test_graph_replays(gpu):
    store, tables, ks, vs = make_store(218, [600, 600], 64, 2, 64)
    q = randn(219, 2, 4, 64).cuda()
    lse = torch.full((2, 4), 7.0, device="cuda")
    seq_lens = torch.zeros(2, dtype=torch.int32, device="cuda")
    w2 = torch.zeros((2, 2, 640), device="cuda")
    qc, lc = randn(220, 50, 4, 64).cuda(), torch.full((4, 50), 6.0, device="cuda")
    w1 = torch.zeros((2, 600), device="cuda")
    size = binding.mocap_key_weights_workspace_size(550, 50, 4, 2, 64)
    ws = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")

    def step():
        binding.mocap_key_weights(store, tables[0], qc, 550, 0.125, lc, w1, w1, ws)
        binding.mocap_decode_key_weights(store, tables, seq_lens, q, 600, 0.125, lse, w2, w2)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for lens in ([600, 1], [0, 333], [64, 65], [599, 600]):
        seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        results = []
        for run in (graph.replay, step):
            w1.fill_(0.5)
            w2.fill_(0.25)
            torch.cuda.synchronize()
            run()
            torch.cuda.synchronize()
            results.append((w1.clone(), w2.clone()))
        assert torch.equal(results[0][0], results[1][0]) and torch.equal(results[0][1], results[1][1])
        for b, n in enumerate(lens):
            if n:
                ref = Weights(q[b:b + 1].cpu(), ks[b][:n], n - 1, 0.125, lse[b][:, None].cpu(), torch.full((2, n), 0.25))
                check_close(results[0][1][b, :, :n], ref.w, ref.bound, f"replay {lens}")


def test_refused_calls_write_nothing(gpu):
    store, tables, _, _ = make_store(221, [200], 64, 2, 64)
    q, lse = randn(222, 10, 4, 64).cuda(), torch.zeros((4, 10), device="cuda")
    weights = torch.full((2, 200), 7.0, device="cuda")
    with pytest.raises(binding.MocapError) as err:
        binding.mocap_key_weights(store, tables[0], q, 191, 0.1, lse, None, weights)
    assert err.value.status == binding.MOCAP_ERR_INVALID_ARG  # 201 positions
    with pytest.raises(binding.MocapError):
        binding.mocap_key_weights(store, tables[0], q, 190, -0.1, lse, None, weights)
    flat = torch.zeros(500, device="cuda")
    with pytest.raises(ValueError):  # overlapping, but not the same
        binding.mocap_key_weights(store, tables[0], q, 190, 0.1, lse, flat[4:404].view(2, 200), flat[:400].view(2, 200))
    with pytest.raises(ValueError):
        binding.mocap_key_weights(store, tables[0], q, 190, 0.1, lse, weights[:, :100].contiguous(), weights)
    with pytest.raises(ValueError):
        binding.mocap_key_weights(store, tables[0], q, 190, 0.1, lse.t().contiguous(), None, weights)
    with pytest.raises(ValueError):
        binding.mocap_key_weights(store, tables[0], q, 190, 0.1, lse, None, weights[:1])
    seq_lens = torch.tensor([200], dtype=torch.int32).cuda()
    with pytest.raises(binding.MocapError):
        binding.mocap_decode_key_weights(store, tables, seq_lens, q[:1], 201, 0.1, lse[:, :1].t().contiguous(), None,
                                         weights[None])
    torch.cuda.synchronize()
    assert (weights == 7.0).all()
    empty = torch.zeros((0, 4, 64), dtype=torch.bfloat16, device="cuda")
    binding.mocap_key_weights(store, tables[0], empty, 100, 0.1, torch.zeros((4, 0), device="cuda"), None, weights)
    torch.cuda.synchronize()
    assert (weights == 7.0).all()


def test_more_than_64_blocks_of_new_keys(gpu):
    """A chunk so long that a workgroup looks for its part among more key blocks than a
    wavefront has lanes: some keys of every block against the sum in 64 bits."""
    rows, d, scale = 34000, 64, 0.125
    store, tables, ks, _ = make_store(230, [rows], 256, 1, d)
    q = randn(231, rows, 1, d)
    lse = math.log(rows) + 0.1 * base(232, 1, rows)
    weights = torch.full((1, rows), float("nan"), device="cuda")
    size = binding.mocap_key_weights_workspace_size(0, rows, 1, 1, d)
    assert size > 0
    call(store, tables[0], q.cuda(), 0, scale, lse.cuda(), None, weights)
    keys = torch.arange(0, rows, 211)
    s = q[:, 0].double() @ ks[0][keys, 0].double().t() * scale
    big = q[:, 0].double().abs() @ ks[0][keys, 0].double().abs().t() * scale
    term = torch.exp(s - lse[0].double()[:, None]) * (torch.arange(rows)[:, None] >= keys)
    # The bound of Weights: each term's argument and exponential, then the sum.
    e = (d + 16) * U * big + 4 * U * lse[0].double().abs()[:, None] + 4 * U
    bound = (e * term * (1 + 2 * e)).sum(0) + (rows / 16 + 34) * U * term.sum(0) + 1e-37
    check_close(weights[0].cpu()[keys], term.sum(0), bound, "long chunk")
    assert torch.isfinite(weights).all()
