"""Attention over the 4-bit store at the ends of its format: the least and the largest scales among keys and among
values, and values up to the magnitude at which no sum leaves fp32, in every way that a call goes."""
import pytest
import torch

from cache_helpers import Pools4
from helpers import say
from serve_helpers import Attention, check_close, randn
from test_kv4_attn_gpu import CHUNK_ERROR, DECODE_ERROR, check_decode, chunk, decode, growing

pytestmark = pytest.mark.gpu

# Rows in a block (test_cache_abi.py holds that they are, at these windows): heads, prefix, rows, splits, windows.  (One
# key a row never goes in blocks of 32.)
WAYS = {16: (8, 2, 40, 60, 1, (0, 1)), 32: (128, 16, 250, 150, 1, (0,)), 256: (128, 16, 250, 300, 1, (0, 1))}


def stored(k, v):
    """A store of 64-slot blocks that holds k and v from position 0; its table, and what it stands for."""
    n, h_kv, d = k.shape
    pools = Pools4(-(-n // 64), 64, h_kv, d)
    table = torch.arange(-(-n // 64), dtype=torch.int32)
    k, v = pools.put(table, 0, k, v)
    return pools, pools.to_gpu(), table.cuda(), k.to(torch.bfloat16), v.to(torch.bfloat16)


def check_chunk(store, table, q, k, v, prefix, scale, window, splits, least=0.0):
    o, lse, _ = chunk(store, table, q.cuda(), prefix, scale, window, 0, splits)
    ref = Attention(q, k, v, prefix, scale, window)
    check_close(o, ref.o, ref.o_bound(CHUNK_ERROR) + least, "o")
    check_close(lse, ref.lse, ref.lse_bound(), "lse")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("way", WAYS)
def test_scales_of_values(gpu, d, way):
    """Value blocks with scale bytes 2, 251 and 252: every row sees its own position only, so O is that value; or all keys,
    with one block of 251 and one of 252, whose weights are at most 1 and whose sum fp32 holds."""
    h_q, h_kv, prefix, rows, splits, windows = WAYS[way]
    n, window = prefix + rows, max(windows)
    say(f"[case] kv4 value scales {way} rows a block d={d}")
    k, v = randn(400, n, h_kv, d).float(), randn(401, n, h_kv, d).double()
    v[::3, :, :32] *= 1e-39
    large = [(5, 2.5e38), (9, 0.7e38)] if window == 0 else [(t, 2.5e38 if t % 2 else -0.7e38) for t in range(1, n, 3)]
    for t, top in large:
        v[t, :, 32:] = v[t, :, 32:].clamp(-2.0, 2.0) * (top / 2.0)
        v[t, :, 32] = top
    pools, store, table, k, v = stored(k, v.float().to(torch.bfloat16))
    assert {2, 251, 252} <= set(pools.v_scale[pools.v_scale != 255].tolist())
    q = randn(402, rows, h_q, d)
    check_chunk(store, table, q, k, v, prefix, 0.1, window, splits)
    for end in (n, n - 1, n - 2):
        o, lse = decode(store, table[None], [end], q[-1:].cuda(), n, 0.1, window)
        check_decode(o, lse, q[-1:], [k], [v], [end], 0.1, window)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("way", WAYS)
def test_scales_of_keys(gpu, d, way):
    """Key blocks with scale bytes 251 and 252 under queries near 2^-124, and with byte 2 under large ones."""
    h_q, h_kv, prefix, rows, splits, _ = WAYS[way]
    n = prefix + rows
    say(f"[case] kv4 key scales {way} rows a block d={d}")
    k, v = randn(410, n, h_kv, d).double(), randn(411, n, h_kv, d)
    k[..., :32] = k[..., :32].clamp(-2.0, 2.0) * (2.0 ** 127 / 2.01)
    k[::2, :, :32] *= 0.5
    k[::2, :, 1], k[1::2, :, 0] = 1.2e38, -2.5e38
    k[..., 32:64] *= 2.0 ** -126
    pools, store, table, k, v = stored(k.float().to(torch.bfloat16), v)
    assert {2, 251, 252} <= set(pools.k_scale[pools.k_scale != 255].tolist())
    q = randn(412, rows, h_q, d).float()
    q[..., :32] = torch.where(q[..., :32] < 0, -1.5, 1.0) * 2.0 ** -124
    q[..., 32:64] *= 2.0 ** 118
    q = q.to(torch.bfloat16)
    check_chunk(store, table, q, k, v, prefix, 0.1, 0, splits)
    o, lse = decode(store, table[None], [n], q[-1:].cuda(), n, 0.1)
    check_decode(o, lse, q[-1:], [k], [v], [n], 0.1)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("way", WAYS)
def test_values_up_to_their_limit(gpu, d, way):
    """Values up to 2^40 (chunks) and 2^96 (batches) under scores that climb by 800 binary orders: O is finite."""
    h_q, h_kv, prefix, rows, splits, _ = WAYS[way]
    n = prefix + rows
    say(f"[case] kv4 largest values {way} rows a block d={d}")
    _, _, k, v = growing(420, n, h_kv, d, 64)
    q = randn(421, rows, h_q, d)
    q[..., 0] = 8.0
    for top, batch in ((2.0 ** 40, False), (2.0 ** 96, True)):
        big = (v.double() / v.double().abs().max() * (0.99 * top)).to(torch.bfloat16)
        pools, store, table, k4, v4 = stored(k, big)
        assert 0.7 * top < float(v4.double().abs().max()) <= top
        # Weights below 2^-126, the least normal number of fp32 and bf16, may count as 0; they are so against a reference
        # whose row has a sum of at least 1, so each takes at most 2^-126 of its value from O.
        least = n * 2.0 ** -126 * top
        if batch:
            o, lse = decode(store, table[None], [n], q[-1:].cuda(), n, 1.0)
            ref = Attention(q[-1:], k4, v4, n - 1, 1.0)
            check_close(o, ref.o, ref.o_bound(DECODE_ERROR) + least, "o of a batch")
            check_close(lse[0][:, None], ref.lse, ref.lse_bound(), "lse of a batch")
        else:
            check_chunk(store, table, q, k4, v4, prefix, 1.0, 0, splits, least)
