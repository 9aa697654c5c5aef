"""Plain 64-bit forms of the rotation and of the 4-bit store's format, on the CPU,
and builders of 4-bit stores."""
import math

import torch

from paper_2606_22968_amd import binding

MAGS = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def inv_freq(rot, theta=10000.0):
    return (theta ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)).float()


def rotate(x, positions, freq, interleaved):
    """x [n][heads][d] in 64 bits, turned; |first| + |second| of each value's pair beside it."""
    x = x.double()
    half = 0 if freq is None else freq.numel()
    out, size = x.clone(), x.abs()
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        angle = positions.double() * float(freq[i])
        c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
        out[..., a], out[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
        size[..., a] = size[..., b] = x[..., a].abs() + x[..., b].abs()
    return out, size


def quantise(x):
    """Codes [..., d] and scale bytes [..., d / 32] of the format, by search: the least scale that holds the largest
    magnitude, then the nearest code, the even one of two as near."""
    blocks = x.double().unflatten(-1, (-1, 32))
    bad = ~torch.isfinite(blocks).all(-1)
    blocks = torch.where(bad[..., None], torch.zeros_like(blocks), blocks)
    top = blocks.abs().amax(-1)
    e = torch.full_like(top, -125)
    for k in range(-125, 125):
        e = torch.where(top > 6.0 * 2.0 ** k, torch.full_like(e, k + 1), e)
    t = blocks / torch.exp2(e)[..., None]
    order = torch.tensor([0, 2, 4, 6, 1, 3, 5, 7])
    code = order[(t.abs()[..., None] - MAGS[order]).abs().argmin(-1)]
    code = code | torch.signbit(blocks).long() << 3
    code = torch.where(bad[..., None], torch.zeros_like(code), code)
    byte = torch.where(bad, torch.full_like(e, 255), e + 127)
    return code.flatten(-2).to(torch.uint8), byte.to(torch.uint8)


def values(code, byte):
    """What codes and bytes stand for, in 64 bits."""
    code = code.long()
    mag = MAGS[code & 7]
    scale = torch.where(byte == 255, torch.tensor(float("nan"), dtype=torch.float64), torch.exp2(byte.double() - 127))
    return torch.where(code >= 8, -mag, mag) * scale.repeat_interleave(32, -1)


class Pools4:
    """The four pools of a 4-bit store on the CPU, position by position."""

    def __init__(self, blocks, bs, h_kv, d, fill=0xFF):
        self.bs, self.h_kv, self.d = bs, h_kv, d
        self.k_pool = torch.full((blocks, h_kv, bs, d // 2), fill, dtype=torch.uint8)
        self.v_pool = torch.full((blocks, h_kv, bs // 64, d // 2, 64), fill, dtype=torch.uint8)
        self.k_scale = torch.full((blocks, h_kv, bs // 64, d // 32, 64), fill, dtype=torch.uint8)
        self.v_scale = self.k_scale.clone()

    def put(self, table, start, k, v):
        """Quantises k, v [n][h_kv][d] into positions start ..; returns what they then stand for."""
        pos = torch.arange(start, start + k.shape[0])
        block, slot = table.cpu().long()[pos // self.bs], pos % self.bs
        kc, kb = quantise(k)
        vc, vb = quantise(v)
        self.k_pool[block, :, slot] = kc[..., 0::2] | kc[..., 1::2] << 4
        pairs = vc.unflatten(-1, (-1, 2, 16))
        self.v_pool[block, :, slot // 64, :, slot % 64] = (pairs[..., 0, :] | pairs[..., 1, :] << 4).flatten(-2)
        self.k_scale[block, :, slot // 64, :, slot % 64] = kb
        self.v_scale[block, :, slot // 64, :, slot % 64] = vb
        return values(kc, kb), values(vc, vb)

    NAMES = ("k_pool", "v_pool", "k_scale", "v_scale")

    def to_gpu(self):
        store = binding.Kv4Store(self.k_pool.shape[0], self.bs, self.h_kv, self.d)
        for name in self.NAMES:
            getattr(store, name).copy_(getattr(self, name))
        return store

    def same_as(self, store, what):
        for name in self.NAMES:
            got, want = getattr(store, name).cpu(), getattr(self, name)
            assert torch.equal(got, want), f"{what}: {name} differs in {int((got != want).sum())} bytes"


def make_store4(seed, lens, bs, h_kv, d, spare=1, fill=0xFF):
    """A 4-bit store whose sequences' blocks lie at permuted places, every byte that is no position's `fill` (0xFF: NaN);
    [batch][stride] tables; the values that it stands for per sequence [n][h_kv][d], in bf16 (exact), on the CPU."""
    g = torch.Generator(device="cpu")
    g.manual_seed(seed)
    need = [-(-max(n, 0) // bs) for n in lens]
    total = sum(need) + spare
    perm = torch.randperm(total, generator=g).to(torch.int32)
    tables = torch.zeros((len(lens), max(max(need), 1)), dtype=torch.int32)
    pools = Pools4(total, bs, h_kv, d, fill)
    ks, vs, at = [], [], 0
    for b, n in enumerate(lens):
        n = max(n, 0)
        tables[b, :need[b]] = perm[at:at + need[b]]
        at += need[b]
        k, v = (torch.randn((n, h_kv, d), generator=g) for _ in range(2))
        k, v = pools.put(tables[b], 0, k, v) if n else (k, v)
        ks.append(k.to(torch.bfloat16))
        vs.append(v.to(torch.bfloat16))
    return pools, pools.to_gpu(), tables.cuda(), ks, vs


# Angles from whole numbers: pi by Machin's formula, to 2^-400.
_BITS = 400


def _arctan_of_inverse(x):
    term = (1 << _BITS + 20) // x
    total, n, sign = term, 3, -1
    while term:
        term //= x * x
        total += sign * (term // n)
        n, sign = n + 2, -sign
    return total


_PI = (16 * _arctan_of_inverse(5) - 4 * _arctan_of_inverse(239)) >> 20


def exact_turn(position, freq):
    """cos and sin of position * freq (an fp32 value, finite), each within 2^-52 of it at any size."""
    if position < 0:
        c, s = exact_turn(-position, freq)
        return c, -s
    m, e = math.frexp(freq)
    angle, shift = position * int(m * (1 << 24)), _BITS + e - 24
    angle = angle << shift if shift >= 0 else angle >> -shift
    n = (2 * angle + _PI // 2) // _PI                     # quarter turns, rounded
    rest = (2 * angle - n * _PI) / (1 << _BITS + 1)       # within pi / 4
    c, s = math.cos(rest), math.sin(rest)
    return ((c, s), (-s, c), (-c, -s), (s, -c))[n % 4]


def rotate_exact(x, positions, freq, interleaved, limit=2.0 ** 48):
    """As rotate, with exact_turn; angles of `limit` or more, and those that are no number, make NaN pairs."""
    x = x.double()
    half = freq.numel()
    out, size = x.clone(), x.abs()
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        f, turns = float(freq[i]), []
        for p in positions.tolist():
            near = math.isfinite(f) and abs(p * f) < limit
            turns.append(exact_turn(p, f) if near else (math.nan, math.nan))
        c, s = torch.tensor(turns, dtype=torch.float64).T[:, :, None]
        out[..., a], out[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
        size[..., a] = size[..., b] = x[..., a].abs() + x[..., b].abs()
    return out, size
