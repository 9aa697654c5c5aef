"""The rotating appends and the attention of both stores together, as a program uses them: prompts in chunks out of one
projection's rows, an eviction, and captured decoding steps in which the rotation's positions are not the slots."""
import pytest
import torch

from cache_helpers import inv_freq, quantise, rotate, values
from helpers import say
from paper_2606_22968_amd import binding
from serve_helpers import B, Attention, check_close, randn, take

pytestmark = pytest.mark.gpu

CHUNKS = [[100, 64, 37], [1, 130]]


def attend_chunk(four, store, table, q, prefix, scale):
    rows, h_q, d = q.shape
    o, lse = torch.empty_like(q), torch.empty((h_q, rows), device="cuda")
    sizes = binding.mocap_kv4_chunk_attn_workspace_size if four else binding.mocap_chunk_attn_workspace_size
    ws = torch.empty(max(sizes(prefix, rows, h_q, store.h_kv, d)[1], 16), dtype=torch.uint8, device="cuda")
    call = binding.mocap_kv4_chunk_attn if four else binding.mocap_chunk_attn
    call(store, table, q, prefix, scale, o, lse, ws)
    return o, lse


def held(four, store, table, n):
    """Keys and values of positions [0, n), on the CPU in bf16."""
    if not four:
        return take(store, table, n)
    out = [torch.empty((1, n, store.h_kv, store.head_dim), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    binding.mocap_kv4_load(store, table[None], torch.tensor([n], dtype=torch.int32, device="cuda"), *out)
    return out[0][0].cpu(), out[1][0].cpu()


def check_rows(o, lse, q, k, v, prefix, scale, p_error, what):
    ref = Attention(q.cpu(), k, v, prefix, scale)
    check_close(o, ref.o, ref.o_bound(p_error), f"{what} o")
    check_close(lse, ref.lse, ref.lse_bound(), f"{what} lse")


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("h_q,h_kv,d,interleaved", [(8, 2, 128, False), (4, 4, 64, True)])
def test_run(gpu, four, h_q, h_kv, d, interleaved):
    say(f"[case] run four={four} {h_q}/{h_kv}/{d}")
    bs, batch, stride, scale = 64, len(CHUNKS), 8, d ** -0.5  # (mocap_chunk_attn wants its table on 16 bytes)
    store = binding.Kv4Store(20, bs, h_kv, d, fill=0xFF) if four else binding.KvStore(20, bs, h_kv, d, fill=float("nan"))
    tables = torch.randperm(20, generator=torch.Generator().manual_seed(1))[:batch * stride].to(torch.int32)
    tables = tables.reshape(batch, stride).cuda()
    freq = inv_freq(d)
    rope = binding.Rope(freq.cuda(), interleaved)
    append = binding.mocap_kv4_append if four else binding.mocap_rope_append

    # The prompts, chunk by chunk.
    for b, lengths in enumerate(CHUNKS):
        start = 0
        for n in lengths:
            rows = randn(10 * b + start, n, h_q + 2 * h_kv, d).cuda()
            q, k, v = rows[:, :h_q], rows[:, h_q:h_q + h_kv], rows[:, h_q + h_kv:]
            q_out = torch.empty((n, h_q, d), dtype=torch.bfloat16, device="cuda")
            append(store, tables[b], start, k, v, rope, None, q, q_out)
            o, lse = attend_chunk(four, store, tables[b], q_out, start, scale)
            k_held, v_held = held(four, store, tables[b], start + n)
            at = start + torch.arange(n)
            if four:
                assert torch.equal(k_held[start:].double(), values(*quantise(rotate(k.cpu(), at, freq, interleaved)[0])))
                assert torch.equal(v_held[start:].double(), values(*quantise(v.cpu())))
            check_rows(o, lse, q_out, k_held, v_held, start, scale, B, f"prompt {b} chunk at {start}")
            start += n
    lens = [sum(x) for x in CHUNKS]
    true_pos = torch.tensor(lens, dtype=torch.int32)

    # Half of the first sequence is evicted (bf16 store): its slots and positions part.
    if not four:
        keep = 101
        new_table = torch.tensor(sorted(set(range(20)) - set(tables.flatten().tolist()))[:2], dtype=torch.int32).cuda()
        weights = torch.rand((h_kv, lens[0]), generator=torch.Generator().manual_seed(3)).cuda()
        kept = torch.empty((h_kv, keep), dtype=torch.int32, device="cuda")
        size = binding.mocap_kv_evict_workspace_size(lens[0], h_kv, keep)
        binding.mocap_kv_evict(store, tables[0], store, new_table, lens[0], keep, 4, 30, weights, kept, None,
                               torch.empty(max(size, 16), dtype=torch.uint8, device="cuda"))
        tables[0, :2] = new_table
        lens[0] = keep

    # Decoding: one captured step, replayed as the sequences grow.
    seq_lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
    positions = true_pos.cuda() - 1
    fused = torch.zeros((batch, h_q + 2 * h_kv, d), dtype=torch.bfloat16, device="cuda")
    q, k, v = fused[:, :h_q], fused[:, h_q:h_q + h_kv], fused[:, h_q + h_kv:]
    q_out = torch.zeros((batch, h_q, d), dtype=torch.bfloat16, device="cuda")
    o, lse = torch.zeros_like(q_out), torch.zeros((batch, h_q), device="cuda")
    name = "kv4_decode" if four else "decode"
    size = getattr(binding, f"mocap_{name}_attn_workspace_size")(batch, h_q, h_kv, d, stride * bs)
    ws = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")
    step_append = binding.mocap_kv4_decode_append if four else binding.mocap_decode_rope_append
    step_attn = getattr(binding, f"mocap_{name}_attn")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        seq_lens += 1
        positions += 1
        step_append(store, tables, seq_lens, k, v, rope, positions, q, q_out)
        step_attn(store, tables, seq_lens, q_out, stride * bs, scale, o, lse, ws)
    for step in range(4):
        fused.copy_(randn(100 + step, *fused.shape))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        at = true_pos + step
        assert positions.tolist() == at.tolist()
        want_q, size_q = rotate(q.cpu(), at, freq, interleaved)
        check_close(q_out, want_q, B * want_q.abs() * (1 + B) + 2.0 ** -21 * size_q, "q")
        want_k, _ = rotate(k.cpu(), at, freq, interleaved)
        for b in range(batch):
            n = lens[b] + step + 1
            assert int(seq_lens[b]) == n
            k_held, v_held = held(four, store, tables[b], n)
            if four:
                assert torch.equal(k_held[-1:].double(), values(*quantise(want_k[b:b + 1])))
            check_rows(o[b:b + 1], lse[b][:, None], q_out[b:b + 1], k_held, v_held, n - 1, scale, 2.0 ** -16,
                       f"step {step} sequence {b}")


def test_table_checks(gpu):
    """With table checks every call looks at the entries that its positions use, before anything is enqueued, and does the
    same as without."""
    rope = binding.Rope(inv_freq(64).cuda())
    store4, store = binding.Kv4Store(4, 64, 2, 64, fill=0), binding.KvStore(4, 64, 2, 64, fill=0.0)
    good, bad = (torch.tensor([3, 1, x], dtype=torch.int32, device="cuda") for x in (0, 9))   # bad: from position 128
    k, v, q = (randn(120 + i, 20, h, 64).cuda() for i, h in enumerate((2, 2, 4)))
    q_out, o = torch.empty_like(q), torch.empty_like(q)
    lse, lse1 = torch.empty((4, 20), device="cuda"), torch.empty((1, 4), device="cuda")
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")

    def at(n):
        return torch.tensor([n], dtype=torch.int32, device="cuda")

    def calls(table, end):
        yield lambda: binding.mocap_kv4_append(store4, table, end - 20, k, v, rope, None, q, q_out)
        yield lambda: binding.mocap_rope_append(store, table, end - 20, k, v, rope, None, q, q_out)
        yield lambda: binding.mocap_kv4_decode_append(store4, table[None], at(end), k[:1], v[:1], rope, None, q[:1], q_out[:1])
        yield lambda: binding.mocap_decode_rope_append(store, table[None], at(end), k[:1], v[:1], rope, None, q[:1], q_out[:1])
        yield lambda: binding.mocap_kv4_load(store4, table[None], at(end), torch.empty_like(k)[None], torch.empty_like(v)[None])
        yield lambda: binding.mocap_kv4_decode_attn(store4, table[None], at(end), q[:1], 192, 0.1, o[:1], lse1, ws)
        yield lambda: binding.mocap_kv4_chunk_attn(store4, table, q, end - 20, 0.1, o, lse, ws)

    binding.set_table_checks(True)
    try:
        for call in (*calls(good, 150), *calls(bad, 128)):
            call()
        for call in calls(bad, 130):
            with pytest.raises(binding.MocapError):
                call()
    finally:
        binding.set_table_checks(False)
    for call in calls(good, 150):
        call()
    again = torch.empty_like(o)
    binding.set_table_checks(True)
    try:
        binding.mocap_kv4_chunk_attn(store4, good, q, 130, 0.1, again, lse, ws)
    finally:
        binding.set_table_checks(False)
    assert torch.equal(again, o)
