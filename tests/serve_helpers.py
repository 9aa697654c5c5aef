"""Plain 64-bit forms of the calls that follow the prefill, with the quantities
their error bounds are made of, and builders of paged stores.

Error bounds.  u = 2^-24 is half a step of fp32, B = 2^-8 of bf16.  With
  S = scale * sum_i |q_i k_i|, the largest over a row's visible keys,
a score (fp32 products and sums in any order, then one multiply by a rounded
scale) is off by at most ds = (d + 8) u S, so a probability is off by a factor
within exp(ds) and the 2 u of the exponential, whose argument (of size at most
the largest |score| + |reference|, in base 2) is rounded once: 4 u S.
"""
import math

import torch

from paper_2606_22968_amd import binding

U = 2.0 ** -24
B = 2.0 ** -8


def make_store(seed, lens, bs, h_kv, d, spare=1, fill=float("nan"), device="cuda"):
    """A store whose sequences' blocks lie at permuted places, everything that is
    no position of a sequence `fill`; [batch][stride] tables; K, V per sequence
    [n][h_kv][d] on the CPU."""
    g = torch.Generator(device="cpu")
    g.manual_seed(seed)
    need = [-(-max(n, 0) // bs) for n in lens]
    total = sum(need) + spare
    perm = torch.randperm(total, generator=g).to(torch.int32)
    stride = max(max(need), 1)
    tables = torch.zeros((len(lens), stride), dtype=torch.int32)
    k_pool = torch.full((total, h_kv, bs, d), fill, dtype=torch.bfloat16)
    v_pool = torch.full((total, h_kv, d, bs), fill, dtype=torch.bfloat16)
    ks, vs, at = [], [], 0
    for b, n in enumerate(lens):
        n = max(n, 0)
        k = torch.randn((n, h_kv, d), generator=g).to(torch.bfloat16)
        v = torch.randn((n, h_kv, d), generator=g).to(torch.bfloat16)
        blocks = perm[at:at + need[b]]
        at += need[b]
        tables[b, :need[b]] = blocks
        put(k_pool, v_pool, blocks, bs, 0, k, v)
        ks.append(k)
        vs.append(v)
    store = binding.KvStore(total, bs, h_kv, d, device=device)
    store.k_pool.copy_(k_pool)
    store.v_pool.copy_(v_pool)
    return store, tables.to(device), ks, vs


def put(k_pool, v_pool, table, bs, start, k, v):
    """Positions start .. of CPU pools."""
    pos = torch.arange(start, start + k.shape[0])
    block, slot = table.long()[pos // bs], pos % bs
    k_pool[block, :, slot] = k
    v_pool[block, :, :, slot] = v


def take(store, table, n):
    """Positions [0, n) of a store: K, V [n][h_kv][d] on the CPU."""
    pos = torch.arange(n)
    block, slot = table.cpu().long()[pos // store.block_size], pos % store.block_size
    return store.k_pool.cpu()[block, :, slot], store.v_pool.cpu()[block, :, :, slot]


def randn(seed, *shape):
    g = torch.Generator(device="cpu")
    g.manual_seed(seed)
    return torch.randn(shape, generator=g).to(torch.bfloat16)


def visible(prefix, rows, n, window, sinks):
    """[rows][n]: which keys each row sees."""
    t, j = prefix + torch.arange(rows)[:, None], torch.arange(n)[None, :]
    seen = j <= t
    if window > 0:
        seen &= (j < sinks) | (j > t - window)
    return seen


class Attention:
    """Attention of q [L][h_q][d] over k, v [n][h_kv][d] in 64 bits: o [L][h_q][d],
    lse [h_q][L], and per row S (see above) and the spread sum_j p_j |v_j - o|."""

    def __init__(self, q, k, v, prefix, scale, window=0, sinks=0):
        rows, h_q, d = q.shape
        n, h_kv = k.shape[:2]
        group = h_q // h_kv
        seen = visible(prefix, rows, n, window, sinks)
        self.o = torch.zeros((rows, h_q, d), dtype=torch.float64)
        self.lse = torch.full((h_q, rows), -math.inf, dtype=torch.float64)
        self.spread = torch.zeros((rows, h_q, d), dtype=torch.float64)
        self.top = torch.zeros((rows, h_q, d), dtype=torch.float64)  # sum_j p_j |v_j|
        self.size = torch.zeros((h_q, rows), dtype=torch.float64)
        self.d, self.n = d, n
        if n == 0:
            return
        for g in range(h_q):
            kd, vd, qd = k[:, g // group].double(), v[:, g // group].double(), q[:, g].double()
            s = (qd @ kd.t() * scale).masked_fill(~seen, -math.inf)
            self.lse[g] = torch.logsumexp(s, 1)
            p = torch.exp(s - self.lse[g][:, None]).masked_fill(~seen, 0.0)
            self.o[:, g] = p @ vd
            for r in range(rows):
                self.spread[r, g] = p[r] @ (vd - self.o[r, g]).abs()
            self.top[:, g] = p @ vd.abs()
            self.size[g] = (qd.abs() @ kd.abs().t() * scale).masked_fill(~seen, 0.0).amax(1)

    def o_bound(self, p_error):
        """p_error: rounding of a probability beyond its fp32 arithmetic.  Every
        p_j off by a factor 1 + e_j moves o by at most max|e| sum p |v - o| (and
        by second-order terms: 2 times covers them); the P V product and the
        normalisation add (n + 8) u of sum p |v|, the output's rounding B |o|."""
        e = (self.d + 16) * U * self.size.t()[:, :, None] + 4 * U + p_error
        return e * (1 + 2 * e) * self.spread + (self.n + 8) * U * self.top + B * self.o.abs() * (1 + B)

    def lse_bound(self):
        """ds, the sum's n u, the logarithm's and the final sum's rounding."""
        finite = self.lse.nan_to_num(neginf=0.0)
        return (self.d + 16) * U * self.size + (self.n + 16) * U + 4 * U * finite.abs()


def check_close(got, want, bound, what):
    got = got.cpu().double()
    err = (got - want).abs()
    same = torch.isinf(want) & (got == want)
    ratio = torch.where(same, torch.zeros_like(err), err / bound.clamp_min(1e-30))
    worst = float(ratio.max()) if ratio.numel() else 0.0
    print(f"[bound] {what}: at most {worst:.3f} of the bound", flush=True)
    assert not torch.isnan(got).any(), f"{what}: NaN"
    assert worst <= 1.0, f"{what}: {worst} of the bound at {int(ratio.argmax())}"


class Weights:
    """w [h_kv][n] of mocap_key_weights in 64 bits, and the bound of its fp32 sum."""

    def __init__(self, q, k, prefix, scale, lse, prev=None):
        rows, h_q, d = q.shape
        n, h_kv = k.shape[:2]
        group = h_q // h_kv
        seen = visible(prefix, rows, n, 0, 0)
        self.w = torch.zeros((h_kv, n), dtype=torch.float64)
        self.bound = torch.zeros((h_kv, n), dtype=torch.float64)
        for g in range(h_q):
            h = g // group
            qd, kd = q[:, g].double(), k[:, h].double()
            row_lse = lse[g].double()[:, None]
            term = torch.exp(qd @ kd.t() * scale - row_lse)
            term = torch.where(seen & (row_lse != -math.inf), term, torch.zeros_like(term))
            # The argument: the score's ds, and the roundings of the scale, the
            # base-2 LSE and their difference; then the exponential's.
            size = qd.abs() @ kd.abs().t() * scale
            e = (d + 16) * U * size + 4 * U * row_lse.abs().nan_to_num(posinf=0.0) + 4 * U
            self.w[h] += term.sum(0)
            self.bound[h] += torch.where(term > 0, e * term * (1 + 2 * e), torch.zeros_like(e)).sum(0)
        # A key's terms are added 16 at a time and then along the rows.
        self.bound += (rows * group / 16 + 32) * U * self.w
        if prev is not None:
            self.w[:, :prefix] += prev[:, :prefix].double()
        self.bound += 2 * U * self.w.abs() + 1e-37
