"""NaN and infinities in mocap_decode_attn: they reach exactly the rows that see
them, whichever of a sequence's parts they lie in."""
import math

import pytest
import torch

from helpers import say
from paper_2606_22968_amd import binding
from serve_helpers import make_store, randn

pytestmark = pytest.mark.gpu

# Parts of four tiles at this load: 2 to 8 of them, and a sequence that is not cut.
LENS = [256 * parts - 3 for parts in range(2, 9)] + [200]
MAX_LEN = 2048
HEADS = [(4, 2, 64), (4, 2, 128), (20, 1, 64), (20, 1, 128)]
WINDOWS = [(0, 0), (1400, 70)]  # both wide enough for parts
DIM = 9


def attend(store, tables, lens, q, scale, window, sinks):
    batch, h_q, d = q.shape
    size = binding.mocap_decode_attn_workspace_size(batch, h_q, store.h_kv, d, MAX_LEN, window, sinks)
    assert size > 0
    ws = torch.empty(size, dtype=torch.uint8, device="cuda").fill_(0xFF)
    o = torch.empty((batch, h_q, d), dtype=torch.bfloat16, device="cuda")
    lse = torch.empty((batch, h_q), dtype=torch.float32, device="cuda")
    binding.mocap_decode_attn(store, tables, lens, q, MAX_LEN, scale, o, lse, ws, window, sinks)
    return o.cpu(), lse.cpu()


def sees(n, j, window, sinks):
    return j < n and (window == 0 or j < sinks or j > n - 1 - window)


def bits(x):
    return x.contiguous().view(torch.int16 if x.dtype == torch.bfloat16 else torch.int32)


def cases(h_q, h_kv, d, seed):
    store, tables, ks, vs = make_store(seed, LENS, 64, h_kv, d)
    q = randn(seed + 1, len(LENS), h_q, d)
    # Even heads have a positive first dim, odd ones a negative one.
    q[:, :, 0] = q[:, :, 0].abs() + 0.5
    q[:, 1::2, 0] *= -1
    return store, tables, torch.tensor(LENS, dtype=torch.int32).cuda(), q.cuda()


@pytest.mark.parametrize("window,sinks", WINDOWS)
@pytest.mark.parametrize("h_q,h_kv,d", HEADS)
@pytest.mark.parametrize("kind", ["nan", "inf"])
def test_a_nonfinite_key_in_every_tile(gpu, kind, h_q, h_kv, d, window, sinks):
    """A key that is NaN, or whose score is +infinity for the even heads and -infinity for the odd ones, in one
    tile of all sequences after the other: NaN in all of O and in the LSE of the heads with a NaN or +infinite
    score, and of those alone."""
    say(f"[case] decode {kind} key {h_q}/{h_kv}/{d} window={window} sinks={sinks}")
    store, tables, lens, q = cases(h_q, h_kv, d, 400)
    group = h_q // h_kv
    o0, lse0 = attend(store, tables, lens, q, d ** -0.5, window, sinks)
    assert torch.isfinite(o0.float()).all() and torch.isfinite(lse0).all()
    for tile in range(MAX_LEN // 64):
        j = tile * 64 + 5
        rows = [b for b, n in enumerate(LENS) if j < n]
        blocks = tables[rows, tile].long()
        before = store.k_pool[blocks, 0, 5].clone()
        if kind == "nan":
            store.k_pool[blocks, 0, 5] = float("nan")
        else:
            store.k_pool[blocks, 0, 5, 0] = math.inf
        o, lse = attend(store, tables, lens, q, d ** -0.5, window, sinks)
        store.k_pool[blocks, 0, 5] = before
        want = torch.zeros(len(LENS), h_q, dtype=torch.bool)
        near = torch.zeros(len(LENS), h_q, dtype=torch.bool)  # heads that see the key
        for b, n in enumerate(LENS):
            if sees(n, j, window, sinks):
                near[b, :group] = True
                want[b, 0:group:1 if kind == "nan" else 2] = True
        assert torch.equal(torch.isnan(lse), want), f"tile {tile}"
        assert torch.equal(torch.isnan(o).all(-1), want) and torch.equal(torch.isnan(o).any(-1), want), f"tile {tile}"
        assert torch.isfinite(lse[~want]).all() and torch.isfinite(o[~want].float()).all()
        assert torch.equal(bits(o[~near]), bits(o0[~near])) and torch.equal(bits(lse[~near]), bits(lse0[~near]))


# Dim -> what two neighbouring keys hold there.
VALUES = {DIM: (math.inf, None), 10: (None, -math.inf), 11: (math.inf, -math.inf), 12: (math.nan, None), 13: (math.inf, math.inf),
          63: (-math.inf, None)}


@pytest.mark.parametrize("window,sinks", WINDOWS)
@pytest.mark.parametrize("h_q,h_kv,d", HEADS)
def test_infinite_values_in_every_tile(gpu, h_q, h_kv, d, window, sinks):
    """O is infinite where one infinity is seen, NaN where both or a NaN are, and the same bits as ever elsewhere."""
    say(f"[case] decode infinite values {h_q}/{h_kv}/{d} window={window} sinks={sinks}")
    store, tables, lens, q = cases(h_q, h_kv, d, 410)
    group = h_q // h_kv
    o0, lse0 = attend(store, tables, lens, q, d ** -0.5, window, sinks)
    before = store.v_pool.clone()
    for tile in range(MAX_LEN // 64):
        first = tile * 64 + 30
        for b, n in enumerate(LENS):
            for i in range(2):
                if first + i < n:
                    for dim, values in VALUES.items():
                        if values[i] is not None:
                            store.v_pool[tables[b, tile].long(), h_kv - 1, dim, 30 + i] = values[i]
        o, lse = attend(store, tables, lens, q, d ** -0.5, window, sinks)
        assert torch.equal(bits(lse), bits(lse0)), f"tile {tile}"
        want, heads = o0.clone().float(), slice(h_q - group, h_q)
        for b, n in enumerate(LENS):
            for dim, values in VALUES.items():
                seen = [v for i, v in enumerate(values) if v is not None and sees(n, first + i, window, sinks)]
                if seen:
                    want[b, heads, dim] = sum(seen)
        same = (o.float() == want) | (torch.isnan(o) & torch.isnan(want))
        assert same.all(), f"tile {tile}: {same.logical_not().nonzero()[:4].tolist()}"
        store.v_pool.copy_(before)


@pytest.mark.parametrize("h_q,h_kv,d", HEADS)
def test_values_of_the_smallest_weights(gpu, h_q, h_kv, d):
    """Infinite and NaN values of keys whose probability is nothing in fp32 reach O all the same."""
    say(f"[case] decode values of the smallest weights {h_q}/{h_kv}/{d}")
    store, tables, ks, vs = make_store(420, [2048], 64, h_kv, d)
    q = torch.zeros(1, h_q, d, dtype=torch.bfloat16)
    q[:, 0::2, 0], q[:, 1::2, 0] = 1.0, -1.0
    # Scores of -150 to 150 and back: exp(-300) is 0 in fp32.
    ramp = torch.linspace(-150, 150, 2048).to(torch.bfloat16).view(32, 64).cuda()
    for tile in range(32):
        store.k_pool[tables[0, tile].long(), :, :, 0] = ramp[tile]
    lens = torch.tensor([2048], dtype=torch.int32).cuda()
    o0, lse0 = attend(store, tables, lens, q.cuda(), 1.0, 0, 0)
    assert torch.isfinite(o0.float()).all()
    for tile in (0, 15, 31):
        pool = store.v_pool[tables[0, tile].long()]
        before = pool.clone()
        pool[:, DIM, 40], pool[:, 10, 41], pool[:, 11, 42] = math.inf, -math.inf, math.nan
        store.v_pool[tables[0, tile].long()] = pool
        o, lse = attend(store, tables, lens, q.cuda(), 1.0, 0, 0)
        store.v_pool[tables[0, tile].long()] = before
        assert torch.equal(bits(lse), bits(lse0))
        assert (o[:, :, DIM] == math.inf).all() and (o[:, :, 10] == -math.inf).all() and torch.isnan(o[:, :, 11]).all()
        o[:, :, DIM:12] = o0[:, :, DIM:12]
        assert torch.equal(bits(o), bits(o0))


@pytest.mark.parametrize("h_q,h_kv,d", HEADS)
def test_scores_beyond_fp32(gpu, h_q, h_kv, d):
    """Products within fp32 whose multiple by the scale is not: NaN, as with an infinite score, and not an empty row."""
    say(f"[case] decode scores beyond fp32 {h_q}/{h_kv}/{d}")
    store, tables, lens, q = cases(h_q, h_kv, d, 430)
    q[:, :, 0] = torch.where(q[:, :, 0] > 0, 1e19, q[:, :, 0])
    for tile in (0, 3, 17, 31):
        rows = [b for b, n in enumerate(LENS) if tile * 64 + 5 < n]
        blocks = tables[rows, tile].long()
        store.k_pool[:, :, :, 0] = 0.0
        store.k_pool[blocks, :, 5, 0] = 1e19  # 1e38, and 4e38 with the scale
        o, lse = attend(store, tables, lens, q, 4.0, 0, 0)
        want = torch.zeros(len(LENS), h_q, dtype=torch.bool)
        want[rows, 0::2] = True
        assert torch.equal(torch.isnan(lse), want) and torch.isfinite(lse[~want]).all(), f"tile {tile}"
        assert torch.equal(torch.isnan(o).all(-1), want) and torch.isfinite(o[~want].float()).all(), f"tile {tile}"
