"""Infinite, NaN and very large queries and keys through the rotating appends: what the formula gives by IEEE's rules, in
exactly the pairs (4 bits: the blocks of 32 dims) that hold them."""
import math

import pytest
import torch

from cache_helpers import rotate_exact
from helpers import say
from serve_helpers import check_close
from test_rope_angles_gpu import BS, D, H_KV, H_Q, binding, expect4, keys_of
from test_rope_append_gpu import rotated_bound

pytestmark = pytest.mark.gpu

PLACES = [(1, 0, 3, math.nan), (2, 1, 35, math.inf), (4, 0, 40, -math.inf), (5, 1, 0, math.inf), (5, 1, 32, math.inf),
          (5, 1, 1, math.inf), (6, 0, 31, 2.5e38), (6, 0, 63, -2.5e38), (7, 1, 17, 3.3e38), (8, 1, 20, 1e-40), (0, 0, 9, math.inf)]


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("way", ["chunk", "batch"])
@pytest.mark.parametrize("rot", [64, 32])
def test_what_is_no_ordinary_number(gpu, four, interleaved, way, rot):
    say(f"[case] rope of non-finite rows four={four} interleaved={interleaved} {way} rot={rot}")
    n = 10
    rows = torch.randn((n, H_Q + 2 * H_KV, D), generator=torch.Generator().manual_seed(330))
    for t, h, e, x in PLACES:
        rows[t, h, e] = rows[t, H_Q + h, e] = x
    rows = rows.to(torch.bfloat16)
    q, k, v = rows[:, :H_Q], rows[:, H_Q:H_Q + H_KV], rows[:, H_Q + H_KV:]
    freq = (10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)).float()
    rope = binding.Rope(freq.cuda(), interleaved)
    at = torch.arange(n)                                                   # sines of 0 at position 0
    out = torch.full((n, H_Q, D), 9.0, dtype=torch.bfloat16, device="cuda")
    blocks = n if way == "batch" else 2
    store = binding.Kv4Store(blocks, BS, H_KV, D, fill=0) if four else binding.KvStore(blocks, BS, H_KV, D, fill=0.0)
    tables = torch.arange(blocks, dtype=torch.int32)
    rows_gpu = rows.cuda()
    args = (rows_gpu[:, H_Q:H_Q + H_KV], rows_gpu[:, H_Q + H_KV:], rope)
    if way == "batch":
        tables = tables[:, None].contiguous()
        call = binding.mocap_kv4_decode_append if four else binding.mocap_decode_rope_append
        call(store, tables.cuda(), torch.arange(1, n + 1, dtype=torch.int32, device="cuda"), *args, None, rows_gpu[:, :H_Q], out)
    else:
        call = binding.mocap_kv4_append if four else binding.mocap_rope_append
        call(store, tables.cuda(), 5, *args, 0, rows_gpu[:, :H_Q], out)
    want_q, q_size = rotate_exact(q, at, freq, interleaved)
    want_k, k_size = rotate_exact(k, at, freq, interleaved)

    def check(got, want, size, what):
        got = got.cpu()
        assert torch.equal(torch.isnan(got), torch.isnan(want)), what
        rounded = want.float().to(torch.bfloat16)                          # (what bf16 does not hold is infinite)
        infinite = torch.isinf(rounded)
        assert torch.equal(got[infinite], rounded[infinite]) and not torch.isinf(got[~infinite]).any(), what
        plain = ~infinite & ~torch.isnan(want)
        check_close(got[plain], want[plain], rotated_bound(want, size)[plain], what)

    assert torch.isnan(want_k).any() and torch.isinf(want_k).any()
    check(out, want_q, q_size, "q")
    if four:
        expect4(store, tables, way, n, want_k, v)
    else:
        check(keys_of(store, tables, way, n), want_k, k_size, "k")
