"""The rotating appends at angles of any size: against cosines and sines from whole numbers, up to 2^48 radians, and what
lies beyond."""
import math

import pytest
import torch

from cache_helpers import Pools4, quantise, rotate_exact
from helpers import say
from paper_2606_22968_amd import binding
from serve_helpers import check_close, randn
from test_rope_append_gpu import rotated_bound

pytestmark = pytest.mark.gpu

H_Q, H_KV, D, BS = 4, 2, 64, 64


def append(four, way, at, freq, interleaved, seed):
    """K, V and Q at these positions, in slots 5 on (a chunk) or in a sequence each (a batch).  Returns the store, the
    rotated queries, the table or tables, and the inputs."""
    n = len(at)
    rows = randn(seed, n, H_Q + 2 * H_KV, D).cuda()
    q, k, v = rows[:, :H_Q], rows[:, H_Q:H_Q + H_KV], rows[:, H_Q + H_KV:]
    rope = binding.Rope(freq.cuda(), interleaved)
    out = torch.empty((n, H_Q, D), dtype=torch.bfloat16, device="cuda")
    blocks = n if way == "batch" else 2
    store = binding.Kv4Store(blocks, BS, H_KV, D, fill=0) if four else binding.KvStore(blocks, BS, H_KV, D, fill=0.0)
    tables = torch.arange(blocks, dtype=torch.int32).flip(0)
    if way == "batch":
        tables = tables[:, None].contiguous()
        lens = torch.arange(1, n + 1, dtype=torch.int32, device="cuda")
        call = binding.mocap_kv4_decode_append if four else binding.mocap_decode_rope_append
        call(store, tables.cuda(), lens, k, v, rope, at.to(torch.int32).cuda(), q, out)
    else:
        call = binding.mocap_kv4_append if four else binding.mocap_rope_append
        call(store, tables.cuda(), 5, k, v, rope, int(at[0]), q, out)
    return store, out, tables, q.cpu(), k.cpu(), v.cpu()


def expect4(store, tables, way, n, k, v):
    pools = Pools4(store.num_blocks, BS, H_KV, D, fill=0)
    if way == "batch":
        for b in range(n):
            pools.put(tables[b], b, k[b:b + 1], v[b:b + 1])
    else:
        pools.put(tables, 5, k, v)
    pools.same_as(store, way)


def keys_of(store, tables, way, n):
    pool = store.k_pool.cpu()
    if way == "batch":
        return pool[tables[:, 0].long(), :, torch.arange(n)]
    pos = 5 + torch.arange(n)
    return pool[tables.long()[pos // BS], :, pos % BS]


CHUNKS = [torch.arange(p, p + 20) for p in (0, 3, 1 << 20, (1 << 29) + 7, (1 << 30) + 12345, (1 << 31) - 148)]
BATCHES = [torch.tensor([0, 1, -1, 70003, -(1 << 20), (1 << 29) + 1, 1999999999, -1999999997, (1 << 31) - 1, -(1 << 31)])]


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("way,at", [("chunk", x) for x in CHUNKS] + [("batch", x) for x in BATCHES])
def test_angles_below_their_limit(gpu, four, interleaved, way, at):
    """Frequencies from 2^-20 to 2^17 less a little, of both signs, with full fractions: angles up to 2^48 radians."""
    say(f"[case] rope angles four={four} interleaved={interleaved} {way} from {int(at[0])}")
    g = torch.Generator().manual_seed(7)
    exponents = torch.linspace(-20, 16, D // 2).round()
    freq = (torch.exp2(exponents) * (1 + 0.99 * torch.rand(D // 2, generator=g))).float()
    freq[1::3] *= -1
    assert float(freq.abs().max()) * 2.0 ** 31 < 2.0 ** 48
    store, out, tables, q, k, v = append(four, way, at, freq, interleaved, 300)
    want_q, q_size = rotate_exact(q, at, freq, interleaved)
    want_k, k_size = rotate_exact(k, at, freq, interleaved)
    check_close(out, want_q, rotated_bound(want_q, q_size), "q")
    if four:
        # The fp64 cosines and sines are off by at most 2^-52, products and sums by 2^-53 of each: below 1e-15 |x|.  No
        # value of these inputs is within ten times that of a border (but at position 0, where nothing is rounded).
        k_size[at == 0] = 0.0
        for side in (-1e-14, 1e-14):
            assert all(torch.equal(a, b) for a, b in zip(quantise(want_k), quantise(want_k + side * k_size)))
        expect4(store, tables, way, len(at), want_k, v)
    else:
        check_close(keys_of(store, tables, way, len(at)), want_k, rotated_bound(want_k, k_size), "k")


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("way", ["chunk", "batch"])
def test_angles_beyond_their_limit(gpu, four, way):
    """2^48 radians or more, and frequencies that are no number: NaN in these pairs, and nowhere else."""
    at = torch.arange(1, 21) if way == "chunk" else torch.tensor([0, 1, 5, -7, (1 << 31) - 1, -(1 << 31)])
    freq = torch.full((D // 2,), 0.25)
    freq[0], freq[1], freq[2], freq[3], freq[4] = math.inf, -math.inf, math.nan, 2.0 ** 46, -(2.0 ** 120)
    freq[20], freq[21] = 2.0 ** 17, 3.0 * 2.0 ** 44
    store, out, tables, q, k, v = append(four, way, at, freq, True, 310)
    want_q, q_size = rotate_exact(q, at, freq, True)
    want_k, k_size = rotate_exact(k, at, freq, True)
    gone_q, gone_k = torch.isnan(want_q), torch.isnan(want_k)
    assert 0 < int(gone_q.sum()) < gone_q.numel()
    assert torch.equal(torch.isnan(out.cpu()), gone_q)
    check_close(out.cpu()[~gone_q], want_q[~gone_q], rotated_bound(want_q, q_size)[~gone_q], "q")
    if four:
        expect4(store, tables, way, len(at), want_k, v)
    else:
        got = keys_of(store, tables, way, len(at))
        assert torch.equal(torch.isnan(got), gone_k)
        check_close(got[~gone_k], want_k[~gone_k], rotated_bound(want_k, k_size)[~gone_k], "k")


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rot", [(64, 64), (128, 128), (128, 48)])
@pytest.mark.parametrize("first", [0, 30000, (1 << 31) - 1000])
def test_a_token_is_the_same_both_ways(gpu, four, interleaved, d, rot, first):
    """A prompt's chunk and a batch's tokens at the same positions: the same bits of queries, keys and values."""
    say(f"[case] rope both ways four={four} interleaved={interleaved} {rot} of {d} from {first}")
    n, bs = 640, 64
    rows = randn(320, n, H_Q + 2 * H_KV, d).cuda()
    q, k, v = rows[:, :H_Q], rows[:, H_Q:H_Q + H_KV], rows[:, H_Q + H_KV:]
    rope = binding.Rope((10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)).float().cuda(), interleaved)
    kind = binding.Kv4Store if four else binding.KvStore
    stores = [kind(n // bs, bs, H_KV, d, fill=0) for _ in range(2)]
    outs = [torch.zeros((n, H_Q, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    table = torch.arange(n // bs, dtype=torch.int32, device="cuda")
    (binding.mocap_kv4_append if four else binding.mocap_rope_append)(stores[0], table, 0, k, v, rope, first, q, outs[0])
    lens = torch.arange(1, n + 1, dtype=torch.int32, device="cuda")
    (binding.mocap_kv4_decode_append if four else binding.mocap_decode_rope_append)(
        stores[1], table.repeat(n, 1), lens, k, v, rope, lens + (first - 1), q, outs[1])
    pools = ("k_pool", "v_pool", "k_scale", "v_scale") if four else ("k_pool", "v_pool")
    for name, (a, b) in dict(q=outs, **{x: [getattr(s, x) for s in stores] for x in pools}).items():
        a, b = (x.view(torch.int16) if x.dtype is torch.bfloat16 else x for x in (a, b))
        assert torch.equal(a, b), f"{name}: {int((a != b).sum())} of {a.numel()} differ"
