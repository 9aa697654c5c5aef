"""The calls that follow the prefill as a program would use them: prompts go in
by chunks, one under full attention while its key weights accumulate, one in a
sliding window; the first is cut to a budget; both are decoded as one padded
batch by a graph that is captured once; the first is cut again.  Every output is
checked against the plain forms in 64 bits, over keys and values that the test
follows itself."""
import pytest
import torch

from helpers import say
from paper_2606_22968_amd import binding
from serve_helpers import B, Attention, Weights, check_close, make_store, put, randn, take
from test_evict_gpu import expected

pytestmark = pytest.mark.gpu

# Probabilities enter P V as bf16 in the calls over chunks (both the product and
# the normaliser take the rounded ones), as two bf16 values in the decoding.
P_CHUNK, P_DECODE = B, 2.0 ** -16


def scratch(size):
    return torch.empty(max(size, 16), dtype=torch.uint8, device="cuda").fill_(0xFF)


class Sequence:
    """One sequence's keys and values as the test follows them, and its blocks."""

    def __init__(self, store, blocks):
        self.store, self.table = store, torch.tensor(blocks, dtype=torch.int32).cuda()
        self.k = torch.empty((0, store.h_kv, store.head_dim), dtype=torch.bfloat16)
        self.v = self.k.clone()

    def append(self, k, v):
        prefix = self.k.shape[0]
        binding.mocap_kv_append(self.store, self.table, prefix, k.cuda(), v.cuda())
        self.follow(k, v)
        return prefix

    def follow(self, k, v):
        self.k, self.v = torch.cat([self.k, k]), torch.cat([self.v, v])


def chunk(seq, q, k, v, scale, window, sinks, what):
    """One chunk of a prompt; its LSE."""
    prefix = seq.append(k, v)
    rows, h_q, d = q.shape
    h_kv = seq.store.h_kv
    o = torch.full((rows, h_q, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    lse = torch.full((h_q, rows), float("nan"), device="cuda")
    if window:
        size = binding.mocap_window_attn_workspace_size(prefix, rows, h_q, h_kv, d, window, sinks)[1]
        binding.mocap_window_attn(seq.store, seq.table, q.cuda(), prefix, scale, window, sinks, o, lse, scratch(size))
    else:
        size = binding.mocap_chunk_attn_workspace_size(prefix, rows, h_q, h_kv, d)[1]
        binding.mocap_chunk_attn(seq.store, seq.table, q.cuda(), prefix, scale, o, lse, scratch(size))
    ref = Attention(q, seq.k, seq.v, prefix, scale, window, sinks)
    check_close(o, ref.o, ref.o_bound(P_CHUNK), f"{what} P={prefix} o")
    check_close(lse, ref.lse, ref.lse_bound(), f"{what} P={prefix} lse")
    return prefix, lse


def cut(seq, blocks, keep, sinks, recent, weights):
    """Evicts to other blocks of the same store; the sequence that is left and its weights."""
    store, n = seq.store, seq.k.shape[0]
    left = Sequence(store, blocks)
    kept = torch.full((store.h_kv, keep), -1, dtype=torch.int32, device="cuda")
    kept_weights = torch.full((store.h_kv, keep), float("nan"), device="cuda")
    size = binding.mocap_kv_evict_workspace_size(n, store.h_kv, keep)
    binding.mocap_kv_evict(store, seq.table, store, left.table, n, keep, sinks, recent, weights, kept, kept_weights,
                           scratch(size))
    torch.cuda.synchronize()
    of = weights.cpu()
    left.k = torch.empty((keep, store.h_kv, store.head_dim), dtype=torch.bfloat16)
    left.v = left.k.clone()
    for h in range(store.h_kv):
        want = expected(of[h], n, keep, sinks, recent)
        assert kept[h].tolist() == want, f"head {h}"
        assert torch.equal(kept_weights[h].cpu(), of[h][want])
        left.k[:, h], left.v[:, h] = seq.k[want, h], seq.v[want, h]
    got_k, got_v = take(store, left.table, keep)
    assert torch.equal(got_k, left.k) and torch.equal(got_v, left.v)
    return left, kept_weights


@pytest.mark.parametrize("h_q,h_kv,d,bs", [(8, 2, 64, 64), (8, 8, 128, 128), (16, 1, 128, 192)])
def test_prefill_evict_decode(gpu, h_q, h_kv, d, bs):
    say(f"[case] run {h_q}/{h_kv}/{d} bs={bs}")
    scale, sinks, window, recent, keep = d ** -0.5, 4, 150, 32, 200
    blocks = torch.randperm(64, generator=torch.Generator().manual_seed(bs)).tolist()
    store = binding.KvStore(64, bs, h_kv, d, fill=float("nan"))
    full, slid = Sequence(store, blocks[:16]), Sequence(store, blocks[16:32])

    # Two prompts in chunks; the first one's weights grow in place.
    weights = torch.full((h_kv, 700), float("nan"), device="cuda")
    for i, rows in enumerate((257, 64, 200)):
        q, k, v = randn(400 + i, rows, h_q, d), randn(410 + i, rows, h_kv, d), randn(420 + i, rows, h_kv, d)
        prefix, lse = chunk(full, q, k, v, scale, 0, 0, "full")
        before = weights.cpu()
        size = binding.mocap_key_weights_workspace_size(prefix, rows, h_q, h_kv, d)
        binding.mocap_key_weights(store, full.table, q.cuda(), prefix, scale, lse, weights, weights, scratch(size))
        ref = Weights(q, full.k, prefix, scale, lse.cpu(), before)
        check_close(weights[:, :prefix + rows], ref.w, ref.bound, f"weights P={prefix}")
    for i, rows in enumerate((190, 130)):
        q, k, v = randn(430 + i, rows, h_q, d), randn(440 + i, rows, h_kv, d), randn(450 + i, rows, h_kv, d)
        chunk(slid, q, k, v, scale, window, sinks, "window")

    # The first prompt is cut to its heaviest keys, in other blocks.
    full, kept_weights = cut(full, blocks[32:40], keep, sinks, recent, weights)

    # A batch of both and a row without a sequence: one step, captured.
    tables = torch.zeros((3, 16), dtype=torch.int32, device="cuda")
    tables[0, :8], tables[2] = full.table, slid.table
    live = torch.tensor([1, 0, 1], dtype=torch.int32, device="cuda")
    lens = torch.tensor([keep, 0, slid.k.shape[0]], dtype=torch.int32, device="cuda")
    max_len = 400
    wide = torch.zeros((3, h_kv, max_len), device="cuda")
    wide[0, :, :keep] = kept_weights
    q, o = (torch.zeros((3, h_q, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k, v = (torch.zeros((3, h_kv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    lse = torch.zeros((3, h_q), device="cuda")
    o_slid, lse_slid = torch.zeros_like(o), torch.zeros_like(lse)
    ws = scratch(max(binding.mocap_decode_attn_workspace_size(3, h_q, h_kv, d, max_len),
                     binding.mocap_decode_attn_workspace_size(3, h_q, h_kv, d, max_len, window, sinks)))

    def step():
        lens.add_(live)
        binding.mocap_decode_append(store, tables, lens, k, v)
        binding.mocap_decode_attn(store, tables, lens, q, max_len, scale, o_slid, lse_slid, ws, window, sinks)
        binding.mocap_decode_attn(store, tables, lens, q, max_len, scale, o, lse, ws)
        binding.mocap_decode_key_weights(store, tables, lens, q, max_len, scale, lse, wide, wide)

    at = lens.clone()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step()
    assert torch.equal(lens, at)
    rows = {0: full, 2: slid}
    for i in range(6):
        for t, seed in ((q, 460), (k, 470), (v, 480)):
            t.copy_(randn(seed + i, *t.shape))
        before, pools = wide.cpu(), (store.k_pool.clone(), store.v_pool.clone())
        ws.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for b, seq in rows.items():
            seq.follow(k[b:b + 1].cpu(), v[b:b + 1].cpu())
            n = seq.k.shape[0]
            qb = q[b:b + 1].cpu()
            for what, out, out_lse, w, s in (("all", o, lse, 0, 0), ("window", o_slid, lse_slid, window, sinks)):
                ref = Attention(qb, seq.k, seq.v, n - 1, scale, w, s)
                check_close(out[b:b + 1], ref.o, ref.o_bound(P_DECODE), f"step {i} row {b} {what} o")
                check_close(out_lse[b][:, None], ref.lse, ref.lse_bound(), f"step {i} row {b} {what} lse")
            ref = Weights(qb, seq.k, n - 1, scale, lse[b].cpu()[:, None], before[b])
            check_close(wide[b, :, :n], ref.w, ref.bound, f"step {i} row {b} weights")
            assert torch.equal(wide[b, :, n:].cpu(), before[b, :, n:])
        assert (o[1] == 0).all() and (lse[1] == -float("inf")).all() and torch.equal(wide[1].cpu(), before[1])
        # The pools changed in the two appended slots alone.
        for b, seq in rows.items():
            put(pools[0], pools[1], seq.table, bs, seq.k.shape[0] - 1, k[b:b + 1], v[b:b + 1])
        assert torch.equal(store.k_pool.view(torch.int16), pools[0].view(torch.int16))
        assert torch.equal(store.v_pool.view(torch.int16), pools[1].view(torch.int16))

    # Cut once more, by weights that go on from what was kept.
    cut(full, blocks[40:44], 60, sinks, 6, wide[0])


def test_two_graphs_at_the_same_time(gpu):
    """Two captured steps over one store, each with outputs and a workspace of its
    own, replayed on two streams together."""
    h_q, h_kv, d, bs, n = 16, 2, 64, 128, 9000
    store = binding.KvStore(80, bs, h_kv, d)
    seq = Sequence(store, list(range(80)))
    seq.append(randn(500, n, h_kv, d), randn(501, n, h_kv, d))
    tables, lens = seq.table[None], torch.tensor([n], dtype=torch.int32, device="cuda")
    size = max(binding.mocap_decode_attn_workspace_size(1, h_q, h_kv, d, n),
               binding.mocap_key_weights_workspace_size(n - 300, 300, h_q, h_kv, d),
               binding.mocap_window_attn_workspace_size(n - 300, 300, h_q, h_kv, d, 4000, 4, 3)[1],
               binding.mocap_kv_evict_workspace_size(n, h_kv, 900))
    sides = []
    for i in range(2):
        side = dict(q=randn(502 + i, 300, h_q, d).cuda(), ws=scratch(size), stream=torch.cuda.Stream(),
                    o=torch.zeros((300, h_q, d), dtype=torch.bfloat16, device="cuda"),
                    lse=torch.zeros((h_q, 300), device="cuda"),
                    one=torch.zeros((1, h_q, d), dtype=torch.bfloat16, device="cuda"),
                    one_lse=torch.zeros((1, h_q), device="cuda"), weights=torch.zeros((h_kv, n), device="cuda"),
                    kept=torch.zeros((h_kv, 900), dtype=torch.int32, device="cuda"),
                    dst=binding.KvStore(8, bs, h_kv, d, fill=0.0),
                    table=torch.arange(8, dtype=torch.int32, device="cuda"))
        sides.append(side)

    def step(s):
        binding.mocap_window_attn(store, seq.table, s["q"], n - 300, 0.125, 4000, 4, s["o"], s["lse"], s["ws"], 3)
        binding.mocap_key_weights(store, seq.table, s["q"], n - 300, 0.125, s["lse"], None, s["weights"], s["ws"])
        binding.mocap_decode_attn(store, tables, lens, s["q"][:1], n, 0.125, s["one"], s["one_lse"], s["ws"])
        binding.mocap_kv_evict(store, seq.table, s["dst"], s["table"], n, 900, 4, 64, s["weights"], s["kept"],
                               None, s["ws"])

    outputs = ("o", "lse", "one", "one_lse", "weights", "kept")
    wanted = []
    for s in sides:
        step(s)
        torch.cuda.synchronize()
        wanted.append([s[name].clone() for name in outputs] + [s["dst"].k_pool.clone(), s["dst"].v_pool.clone()])
        s["graph"] = torch.cuda.CUDAGraph()
        with torch.cuda.graph(s["graph"]):
            step(s)
    for _ in range(10):
        for s in sides:
            for name in outputs:
                s[name].zero_()
            s["ws"].fill_(0xFF)
            s["dst"].k_pool.zero_()
            s["dst"].v_pool.zero_()
        torch.cuda.synchronize()
        for s in sides:
            with torch.cuda.stream(s["stream"]):
                s["graph"].replay()
        torch.cuda.synchronize()
        for s, want in zip(sides, wanted):
            got = [s[name] for name in outputs] + [s["dst"].k_pool, s["dst"].v_pool]
            assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_another_device_is_refused(gpu, monkeypatch):
    """Tensors of the first device while the second is current: refused before any launch."""
    store = binding.KvStore(4, 64, 1, 64, fill=0.0)
    table = torch.arange(4, dtype=torch.int32, device="cuda")
    lens = torch.ones(1, dtype=torch.int32, device="cuda")
    row = torch.zeros((1, 1, 64), dtype=torch.bfloat16, device="cuda")
    lse, out = torch.zeros((1, 1), device="cuda"), torch.full((1, 1, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    weights, kept = torch.full((1, 256), 7.0, device="cuda"), torch.full((1, 1), 7, dtype=torch.int32, device="cuda")
    calls = (lambda: binding.mocap_decode_append(store, table[None], lens, row, row),
             lambda: binding.mocap_decode_attn(store, table[None], lens, row, None, 1.0, out, lse),
             lambda: binding.mocap_window_attn(store, table, row, 0, 1.0, 1, 0, out, lse),
             lambda: binding.mocap_key_weights(store, table, row, 0, 1.0, lse, None, weights),
             lambda: binding.mocap_decode_key_weights(store, table[None], lens, row, None, 1.0, lse, None, weights[None]),
             lambda: binding.mocap_kv_evict(store, table[:1], store, table[1:], 1, 1, 0, 0, weights, kept))
    monkeypatch.setattr(binding, "_raw_device", lambda: 1)
    for call in calls:
        with pytest.raises(ValueError, match="current device"):
            call()
    monkeypatch.undo()
    torch.cuda.synchronize()
    assert (out == 7.0).all() and (weights == 7.0).all() and (kept == 7).all()


@pytest.mark.parametrize("h_q,h_kv,d", [(200, 1, 64), (258, 2, 128), (128, 1, 128)])
def test_wide_groups(gpu, h_q, h_kv, d):
    """More query heads on a KV head than any block of rows holds, in every call."""
    say(f"[case] wide groups {h_q}/{h_kv}/{d}")
    lens, scale = [700, 0, 65, 1], d ** -0.5
    store, tables, ks, vs = make_store(520, lens, 64, h_kv, d)
    q = randn(521, 4, h_q, d)
    seq_lens = torch.tensor(lens, dtype=torch.int32).cuda()
    o, lse = torch.zeros((4, h_q, d), dtype=torch.bfloat16, device="cuda"), torch.zeros((4, h_q), device="cuda")
    binding.mocap_decode_attn(store, tables, seq_lens, q.cuda(), 700, scale, o, lse,
                              scratch(binding.mocap_decode_attn_workspace_size(4, h_q, h_kv, d, 700)))
    prev = torch.rand((4, h_kv, 700), generator=torch.Generator().manual_seed(522))
    weights = prev.cuda()
    binding.mocap_decode_key_weights(store, tables, seq_lens, q.cuda(), 700, scale, lse, weights, weights)
    for b, n in enumerate(lens):
        if n == 0:
            assert (o[b] == 0).all() and (lse[b] == -float("inf")).all() and torch.equal(weights[b].cpu(), prev[b])
            continue
        ref = Attention(q[b:b + 1], ks[b], vs[b], n - 1, scale)
        check_close(o[b:b + 1], ref.o, ref.o_bound(P_DECODE), f"row {b} o")
        check_close(lse[b][:, None], ref.lse, ref.lse_bound(), f"row {b} lse")
        ref = Weights(q[b:b + 1], ks[b], n - 1, scale, lse[b].cpu()[:, None], prev[b])
        check_close(weights[b, :, :n], ref.w, ref.bound, f"row {b} weights")
        assert torch.equal(weights[b, :, n:].cpu(), prev[b, :, n:])
    for rows in (1, 7):
        q, prefix = randn(523, rows, h_q, d), 700 - rows
        o = torch.zeros((rows, h_q, d), dtype=torch.bfloat16, device="cuda")
        lse = torch.zeros((h_q, rows), device="cuda")
        size = binding.mocap_window_attn_workspace_size(prefix, rows, h_q, h_kv, d, 300, 4)[1]
        binding.mocap_window_attn(store, tables[0], q.cuda(), prefix, scale, 300, 4, o, lse, scratch(size))
        ref = Attention(q, ks[0], vs[0], prefix, scale, 300, 4)
        check_close(o, ref.o, ref.o_bound(P_CHUNK), f"{rows} rows o")
        check_close(lse, ref.lse, ref.lse_bound(), f"{rows} rows lse")
        sums = torch.zeros((h_kv, 700), device="cuda")
        size = binding.mocap_key_weights_workspace_size(prefix, rows, h_q, h_kv, d)
        binding.mocap_key_weights(store, tables[0], q.cuda(), prefix, scale, lse, None, sums, scratch(size))
        ref = Weights(q, ks[0], prefix, scale, lse.cpu())
        check_close(sums, ref.w, ref.bound, f"{rows} rows weights")
