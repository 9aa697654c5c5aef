"""Performance cases of the operators that write a paged store and of the store
held in 4 bits: the position rotation applied on the way into the store, and
attention over 4-bit keys and values.

Kinds of pass:

  rope_append  ``mocap_rope_append``: a chunk's Q and K rotated, K and V stored in
               bf16.  Returns the rotated Q and the pools.
  rope_decode  ``mocap_decode_rope_append``: the same for one token of each sequence
               of a batch.  Returns the rotated Q and the pools.
  kv4_append   ``mocap_kv4_append`` of a chunk (rotated on the way), then
               ``mocap_kv4_load`` of the positions just stored.  Returns the rotated
               Q, and the keys and values that the 4-bit store now stands for.
  kv4_step     one decoding step over a 4-bit store: ``mocap_kv4_decode_append``,
               ``mocap_kv4_decode_attn`` and ``mocap_kv4_load`` of the new tokens.
               Returns the rotated Q, O, LSE and the new keys and values.
  kv4_decode   ``mocap_kv4_decode_attn`` alone.  Returns O and LSE.
  kv4_chunk    ``mocap_kv4_chunk_attn``: one chunk of a prompt over its prefix and
               itself in a 4-bit store.  Returns O and LSE.

The 4-bit store: 32 consecutive dims of one position and KV head share a scale
2^e, e the smallest with max |x| <= 6 * 2^e, held as the byte e + 127 (from 2 to
252); a value is the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (code 0 to 7, ties to
the even code; bit 3 is the sign), times 2^e.

  k_pool  [blocks][Hkv][bs][d / 2]         byte i: dims 2 i (low nibble) and 2 i + 1
  v_pool  [blocks][Hkv][bs / 64][d / 2][64]  row 16 b + i: dims 32 b + i and 32 b + 16 + i
                                         of 64 consecutive positions
  k_scale, v_scale  [blocks][Hkv][bs / 64][d / 32][64]

Q, K and V hold N(0, 1) in bf16, 4-bit stores N(0, 1) before their rounding; score
scale 1/sqrt(head_dim); every sequence's blocks lie at permuted places of one pool.
"""
import math

import torch

own = False

# (query heads, KV heads, head_dim) of the layers that the library is tested with.
HEADS = ((32, 8, 128), (64, 8, 128), (8, 8, 64), (8, 4, 128), (8, 2, 128), (16, 2, 64), (12, 4, 128),
         (32, 1, 128), (64, 1, 64), (6, 3, 128))


def listed():
    return [
        # An ordinary chunk of a long prompt: Q, K and V are slices of one projection's rows.
        dict(name="rope_8b_2048", kind="rope_append", h_q=32, h_kv=8, d=128, bs=256, prefix=30720, len=2048, rot=128,
             inter=False, theta=500000.0, shift=0, fused=True),
        # The odd remainder of a prompt, small heads, half of their dims rotated in neighbouring pairs, after an
        # eviction: the rotation's positions are not the slots.
        dict(name="rope_tail_d64", kind="rope_append", h_q=16, h_kv=2, d=64, bs=192, prefix=9001, len=137, rot=32,
             inter=True, theta=10000.0, shift=70003, fused=False),
        # One short conversation, plain multi-head layer: bound by latency.
        dict(name="rope_decode_one", kind="rope_decode", h_q=8, h_kv=8, d=64, bs=64, lens="572", rot=64, inter=False,
             theta=10000.0, shift=0, fused=True),
        # A serving batch, two of its rows without a sequence.
        dict(name="rope_decode_batch", kind="rope_decode", h_q=32, h_kv=8, d=128, bs=256,
             lens="1,7,63,64,65,129,0,255,257,400,513,777,1000,1023,300,99,48,100,500,277,301,333,0,97,450,501,255,601,"
                  "650,701,777,192", rot=128, inter=False, theta=500000.0, shift=131072, fused=True),
        # The ordinary chunk into a 4-bit store.
        dict(name="kv4_append_8b_2048", kind="kv4_append", h_q=32, h_kv=8, d=128, bs=256, prefix=30720, len=2048,
             rot=128, inter=False, theta=500000.0, shift=0, fused=True),
        # A long cache moved into 4 bits: keys that are rotated already, from the middle of a block.
        dict(name="kv4_append_offset", kind="kv4_append", h_q=0, h_kv=8, d=128, bs=192, prefix=8191, len=20011, rot=0,
             inter=False, theta=0.0, shift=0, fused=False),
        # One short conversation, a whole step.
        dict(name="kv4_step_one", kind="kv4_step", h_q=8, h_kv=8, d=64, bs=64, lens="572", window=0, sinks=0, rot=64,
             inter=False, theta=10000.0, shift=0, fused=True),
        # A serving batch whose conversations have very different lengths, a whole step.
        dict(name="kv4_step_ragged", kind="kv4_step", h_q=32, h_kv=8, d=128, bs=256,
             lens="1,7,63,64,65,129,200,255,257,400,513,777,1000,1023,1500,1999,2048,2100,2500,2777,3001,3333,4096,"
                  "4097,4500,5001,5555,6001,6500,7001,0,8192", window=0, sinks=0, rot=128, inter=False,
             theta=500000.0, shift=0, fused=True),
        # Long documents under a 70B layer: the largest decode.
        dict(name="kv4_decode_70b_long", kind="kv4_decode", h_q=64, h_kv=8, d=128, bs=256,
             lens="131072,120001,65537,98304", window=0, sinks=0),
        # Streaming sessions: long histories of which a window and a few first tokens are read.
        dict(name="kv4_decode_window", kind="kv4_decode", h_q=32, h_kv=8, d=128, bs=256,
             lens="4097,9001,16384,20011,30720,32768,50001,65536,4000,100,12345,28000,40000,61000,8191,17",
             window=4096, sinks=4),
        # An ordinary chunk of a long prompt: the largest arithmetic.
        dict(name="kv4_chunk_8b_2048", kind="kv4_chunk", h_q=32, h_kv=8, d=128, bs=256, prefix=30720, len=2048,
             window=0, sinks=0),
        # The odd remainder of a prompt, small heads, a short window and a block of sinks.
        dict(name="kv4_chunk_tail_d64", kind="kv4_chunk", h_q=16, h_kv=2, d=64, bs=192, prefix=9001, len=137,
             window=1000, sinks=64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Another case of the listed ranges: chunks of 1 to 8192 rows (4096 for attention) behind 0 to 65536 keys,
    batches of 1 to 64 sequences of 1 to 131072 tokens, windows of 1 to 16384, every head layout, block sizes from 64
    to 1600, rotations of some or all dims in both orders, near and far positions."""
    kind = rng.choice(("rope_append", "rope_decode", "kv4_append", "kv4_step", "kv4_decode", "kv4_chunk"))
    h_q, h_kv, d = rng.choice(HEADS[:2] + HEADS)
    case = dict(kind=kind, h_q=h_q, h_kv=h_kv, d=d, bs=rng.choice((64, 128, 192, 256, 256, 320, 1600)))
    if kind in ("rope_append", "rope_decode", "kv4_append", "kv4_step"):
        rot = rng.choice((d, d, d // 2, 16 * rng.randint(1, d // 16)))
        case.update(rot=rot, inter=rng.random() < 0.4, theta=rng.choice((10000.0, 500000.0, 1000000.0)),
                    shift=rng.choice((0, 0, _log_int(rng, 1, 1000000))), fused=rng.random() < 0.6)
        if kind.startswith("kv4") and rng.random() < 0.15:
            case.update(rot=0, theta=0.0, shift=0)
    if kind in ("rope_append", "kv4_append"):
        prefix = rng.choice((0, 256 * rng.randint(1, 128), _log_int(rng, 1, 32768)))
        return dict(case, prefix=prefix, len=min(_log_int(rng, 1, 8192), 262144 // h_q))
    if kind in ("rope_decode", "kv4_step", "kv4_decode"):
        batch = _log_int(rng, 1, 64)
        top = min(131072, 400000 // batch)
        if kind != "kv4_decode":
            top = min(32768 if kind == "kv4_step" else 4096, 100000 // batch)
        low = rng.choice((1, 64, max(64, top // 4)))
        case.update(lens=",".join(str(_log_int(rng, min(low, top), top)) for _ in range(batch)))
        if kind == "rope_decode":
            return case
        if rng.random() < 0.4:
            return dict(case, window=_log_int(rng, 1, 16384), sinks=rng.choice((0, 1, 4, 64, 100)))
        return dict(case, window=0, sinks=0)
    rows = _log_int(rng, 1, 4096)
    prefix = rng.choice((0, 256 * rng.randint(1, 128), _log_int(rng, 64, 65536)))
    # No more arithmetic than the largest listed case.
    prefix = max(0, min(prefix, int(9.5e11 / (4.0 * d * h_q * rows)) - rows // 2))
    if rng.random() < 0.4:
        return dict(case, prefix=prefix, len=rows, window=_log_int(rng, 1, 8192), sinks=rng.choice((0, 1, 4, 64, 100)))
    return dict(case, prefix=prefix, len=rows, window=0, sinks=0)


# ---- The 4-bit format, in plain operations ----

_VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _quantise(x):
    """Codes [..., d] and scale bytes [..., d / 32] of x [..., d]."""
    blocks = x.reshape(*x.shape[:-1], -1, 32)
    m, e = torch.frexp(blocks.abs().amax(-1))
    # max = m 2^e with 0.5 <= m < 1, and 6 * 2^(e - 3) = 0.75 * 2^e.
    e = torch.where(m > 0.75, e - 2, e - 3)
    e = torch.where(m == 0, -125, e).clamp(-125, 125)
    t = torch.ldexp(blocks, -e[..., None]).abs()
    code = (t > 0.25).to(torch.uint8)
    for border, inside in ((0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += t >= border if inside else t > border
    code |= torch.signbit(blocks).to(torch.uint8) << 3
    return code.reshape(x.shape), (e + 127).to(torch.uint8)


def _value_of(code, scale):
    """What codes [..., d] with scale bytes [..., d / 32] stand for, in 32 bits."""
    lut = torch.tensor(_VALUES + tuple(-v for v in _VALUES), dtype=torch.float32, device=code.device)
    v = lut[code.int()].reshape(*scale.shape, 32)
    return (v * torch.ldexp(torch.ones((), device=code.device), scale.int() - 127)[..., None]).reshape(code.shape)


class _Store:
    """Block pools in the library's layout: K [blocks][Hkv][bs][d], V [blocks][Hkv][d][bs]."""

    def __init__(self, blocks, bs, h_kv, d):
        self.k_pool = torch.zeros((blocks, h_kv, bs, d), dtype=torch.bfloat16, device="cuda")
        self.v_pool = torch.zeros((blocks, h_kv, d, bs), dtype=torch.bfloat16, device="cuda")


class _Store4:
    """4-bit block pools in the library's layout (see above)."""

    def __init__(self, blocks, bs, h_kv, d):
        def pool(*shape):
            return torch.zeros(shape, dtype=torch.uint8, device="cuda")

        self.k_pool, self.v_pool = pool(blocks, h_kv, bs, d // 2), pool(blocks, h_kv, bs // 64, d // 2, 64)
        self.k_scale, self.v_scale = (pool(blocks, h_kv, bs // 64, d // 32, 64) for _ in range(2))


def _k_bytes(code):
    return code[..., 0::2] | code[..., 1::2] << 4


def _k_codes(byte):
    return torch.stack((byte & 15, byte >> 4), -1).flatten(-2)


def _v_bytes(code):
    """[..., d] -> [..., d / 2], byte 16 b + i of dims 32 b + i and 32 b + 16 + i."""
    x = code.reshape(*code.shape[:-1], -1, 2, 16)
    return (x[..., 0, :] | x[..., 1, :] << 4).flatten(-2)


def _v_codes(byte):
    x = byte.reshape(*byte.shape[:-1], -1, 16)
    return torch.stack((x & 15, x >> 4), -2).flatten(-3)


def _put4(store, table, pos, k, v):
    """K, V [n][Hkv][d] at positions pos [n] of a sequence (or of as many sequences: table [n][stride])."""
    bs = store.k_pool.shape[2]
    lb, slot = pos // bs, pos % bs
    block = table.long()[lb] if table.dim() == 1 else table.long().gather(1, lb[:, None])[:, 0]
    tile, at = slot // 64, slot % 64
    code, scale = _quantise(k)
    store.k_pool[block, :, slot] = _k_bytes(code)
    store.k_scale[block, :, tile, :, at] = scale
    code, scale = _quantise(v)
    store.v_pool[block, :, tile, :, at] = _v_bytes(code)
    store.v_scale[block, :, tile, :, at] = scale


def _take4(store, block, slot):
    """K, V [n][Hkv][d] of n slots, in 32 bits."""
    tile, at = slot // 64, slot % 64
    k = _value_of(_k_codes(store.k_pool[block, :, slot]), store.k_scale[block, :, tile, :, at])
    v = _value_of(_v_codes(store.v_pool[block, :, tile, :, at]), store.v_scale[block, :, tile, :, at])
    return k, v


def _gathered4(store, table, h):
    """K, V [..., blocks * bs][d] of one KV head, table [..., blocks], in 32 bits."""
    at = table.long()
    ks = store.k_scale[at, h].transpose(-1, -2).flatten(-3, -2)                # [..., blocks, bs, d / 32]
    vs = store.v_scale[at, h].transpose(-1, -2).flatten(-3, -2)
    k = _value_of(_k_codes(store.k_pool[at, h]), ks)
    v = _value_of(_v_codes(store.v_pool[at, h].transpose(-1, -2).flatten(-3, -2)), vs)
    return k.flatten(-3, -2), v.flatten(-3, -2)


# ---- Inputs ----

def _binding():
    from paper_2606_22968_amd import binding
    return binding


def _store(case, blocks):
    bits4 = case["kind"].startswith("kv4")
    if own:
        kind = _binding().Kv4Store if bits4 else _binding().KvStore
        return kind(blocks, case["bs"], case["h_kv"], case["d"], fill=0)
    return (_Store4 if bits4 else _Store)(blocks, case["bs"], case["h_kv"], case["d"])


def _randn(seed, shape, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda", dtype=dtype)


def _perm(seed, blocks):
    g = torch.Generator(device="cpu")
    g.manual_seed(seed)
    return torch.randperm(blocks, generator=g).to(torch.int32)


def _lens(case):
    return [int(x) for x in case["lens"].split(",")]


def _blocks(case, n):
    return -(-n // case["bs"])


def _scale(case):
    return float(torch.tensor(1.0 / case["d"] ** 0.5, dtype=torch.float32))


def _fill(case, store, seed):
    """Both pools N(0, 1), drawn in pool order."""
    g = torch.Generator(device="cuda")
    g.manual_seed(7919 * seed + 1)
    if not case["kind"].startswith("kv4"):
        store.k_pool.normal_(generator=g)
        store.v_pool.normal_(generator=g)
        return
    blocks, h_kv, bs, d = store.k_pool.shape[0], case["h_kv"], case["bs"], case["d"]
    step = max(1, (1 << 25) // (h_kv * bs * d))
    for b in range(0, blocks, step):
        n = min(step, blocks - b)
        for pool, scales, pack in ((store.k_pool, store.k_scale, _k_bytes), (store.v_pool, store.v_scale, _v_bytes)):
            code, scale = _quantise(torch.randn((n, h_kv, bs, d), generator=g, device="cuda"))
            byte = pack(code)
            pool[b:b + n] = byte if pool is store.k_pool else byte.unflatten(2, (-1, 64)).transpose(-1, -2)
            scales[b:b + n] = scale.unflatten(2, (-1, 64)).transpose(-1, -2)


def _batch_tables(case, seed):
    """[batch][longest] block tables on the CPU, every sequence's blocks its own."""
    lens = _lens(case)
    need = [_blocks(case, n) for n in lens]
    perm = _perm(seed + 1, max(1, sum(need)))
    tables = torch.zeros((len(lens), max(1, max(need))), dtype=torch.int32)
    at = 0
    for b, m in enumerate(need):
        tables[b, :m] = perm[at:at + m]
        at += m
    return tables


def _tokens(case, seed, n):
    """Q, K, V of n tokens: slices of a projection's rows, or tensors of their own."""
    h_q, h_kv, d = case["h_q"], case["h_kv"], case["d"]
    if case["fused"]:
        rows = _randn(seed + 3, (n, (h_q + 2 * h_kv) * d)).unflatten(1, (-1, d))
        return rows[:, :h_q], rows[:, h_q:h_q + h_kv], rows[:, h_q + h_kv:]
    q = _randn(seed + 3, (n, h_q, d)) if h_q else None
    return q, _randn(seed + 8, (n, h_kv, d)), _randn(seed + 9, (n, h_kv, d))


def _inv_freq(case):
    """theta^(-2 i / rot), i < rot / 2, as a layer holds them."""
    if case["rot"] == 0:
        return None
    i = torch.arange(0, case["rot"], 2, dtype=torch.float64)
    return (case["theta"] ** (-i / case["rot"])).float().cuda()


def prepare(case, seed):
    kind, h_kv, h_q, d = case["kind"], case["h_kv"], case["h_q"], case["d"]
    state = dict(case=case, scale=_scale(case))
    if kind in ("rope_append", "rope_decode", "kv4_append", "kv4_step"):
        state["inv_freq"] = _inv_freq(case)
        if own:
            state["rope"] = _binding().Rope(state["inv_freq"], case["inter"]) if case["rot"] else None
    if kind in ("rope_append", "kv4_append", "kv4_chunk"):
        p, n = case["prefix"], case["len"]
        blocks = _blocks(case, p + n)
        store, table = _store(case, blocks), _perm(seed + 1, blocks).cuda()
        state.update(store=store, table=table)
        if kind != "kv4_append":
            _fill(case, store, seed)
        if kind == "kv4_chunk":
            q = _randn(seed + 3, (n, h_q, d))
            state.update(q=q, o=torch.empty_like(q), lse=torch.empty((h_q, n), dtype=torch.float32, device="cuda"))
            if own:
                size = _binding().mocap_kv4_chunk_attn_workspace_size(p, n, h_q, h_kv, d, case["window"],
                                                                      case["sinks"])[1]
                state["workspace"] = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")
            return state
        q, k, v = _tokens(case, seed, n)
        state.update(q=q, k=k, v=v, q_out=None if q is None else torch.empty((n, h_q, d), dtype=torch.bfloat16, device="cuda"))
        if kind == "kv4_append":
            state.update(tables=table[None], ends=torch.tensor([p + n], dtype=torch.int32).cuda(),
                         k_out=torch.empty((1, n, h_kv, d), dtype=torch.bfloat16, device="cuda"),
                         v_out=torch.empty((1, n, h_kv, d), dtype=torch.bfloat16, device="cuda"))
        return state
    lens = _lens(case)
    store = _store(case, max(1, sum(_blocks(case, n) for n in lens)))
    _fill(case, store, seed)
    seq_lens = torch.tensor(lens, dtype=torch.int32)
    state.update(store=store, tables=_batch_tables(case, seed).cuda(), seq_lens=seq_lens.cuda(), max_len=max(lens))
    if kind == "kv4_decode":
        state["q"] = _randn(seed + 3, (len(lens), h_q, d))
    else:
        q, k, v = _tokens(case, seed, len(lens))
        state.update(q=q, k=k, v=v, q_out=torch.zeros((len(lens), h_q, d), dtype=torch.bfloat16, device="cuda"),
                     positions=(seq_lens - 1 + case["shift"]).cuda() if case["shift"] else None)
        if kind == "rope_decode":
            return state
        state.update(k_out=torch.empty((len(lens), 1, h_kv, d), dtype=torch.bfloat16, device="cuda"),
                     v_out=torch.empty((len(lens), 1, h_kv, d), dtype=torch.bfloat16, device="cuda"))
    state.update(o=torch.empty((len(lens), h_q, d), dtype=torch.bfloat16, device="cuda"),
                 lse=torch.empty((len(lens), h_q), dtype=torch.float32, device="cuda"))
    if own:
        size = _binding().mocap_kv4_decode_attn_workspace_size(len(lens), h_q, h_kv, d, max(lens), case["window"],
                                                               case["sinks"])
        state["workspace"] = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")
    return state


# ---- The framework's calls ----

def _run_own(s):
    binding, case = _binding(), s["case"]
    kind = case["kind"]
    if kind == "rope_append":
        binding.mocap_rope_append(s["store"], s["table"], case["prefix"], s["k"], s["v"], s["rope"],
                                  case["prefix"] + case["shift"], s["q"], s["q_out"])
    elif kind == "rope_decode":
        binding.mocap_decode_rope_append(s["store"], s["tables"], s["seq_lens"], s["k"], s["v"], s["rope"],
                                         s["positions"], s["q"], s["q_out"])
    elif kind == "kv4_append":
        binding.mocap_kv4_append(s["store"], s["table"], case["prefix"], s["k"], s["v"], s["rope"],
                                 case["prefix"] + case["shift"], s["q"], s["q_out"])
        binding.mocap_kv4_load(s["store"], s["tables"], s["ends"], s["k_out"], s["v_out"])
    elif kind == "kv4_step":
        binding.mocap_kv4_decode_append(s["store"], s["tables"], s["seq_lens"], s["k"], s["v"], s["rope"],
                                        s["positions"], s["q"], s["q_out"])
        binding.mocap_kv4_decode_attn(s["store"], s["tables"], s["seq_lens"], s["q_out"], s["max_len"], s["scale"],
                                      s["o"], s["lse"], s["workspace"], case["window"], case["sinks"])
        binding.mocap_kv4_load(s["store"], s["tables"], s["seq_lens"], s["k_out"], s["v_out"])
    elif kind == "kv4_decode":
        binding.mocap_kv4_decode_attn(s["store"], s["tables"], s["seq_lens"], s["q"], s["max_len"], s["scale"], s["o"],
                                      s["lse"], s["workspace"], case["window"], case["sinks"])
    else:
        binding.mocap_kv4_chunk_attn(s["store"], s["table"], s["q"], case["prefix"], s["scale"], s["o"], s["lse"],
                                     s["workspace"], case["window"], case["sinks"])


# ---- The plain forms ----

def _rotated(x, positions, inv_freq, inter, keep64=False):
    """x [n][heads][d] at these positions: angles in 64 bits; the products too where a 4-bit rounding follows."""
    x = x.double() if keep64 else x.float()
    if inv_freq is None:
        return x
    angle = positions.double()[:, None] * inv_freq.double()
    cos, sin = torch.cos(angle).to(x.dtype)[:, None], torch.sin(angle).to(x.dtype)[:, None]
    half = inv_freq.numel()
    first, second, rest = x[..., :half], x[..., half:2 * half], x[..., 2 * half:]
    if inter:
        first, second = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
    a, b = first * cos - second * sin, first * sin + second * cos
    turned = torch.stack((a, b), -1).flatten(-2) if inter else torch.cat((a, b), -1)
    return torch.cat((turned, rest), -1)


def _plain_append(s):
    case, store = s["case"], s["store"]
    bs, p, n = case["bs"], case["prefix"], case["len"]
    slots = p + torch.arange(n, device="cuda")
    at, bits4 = slots + case["shift"], case["kind"] == "kv4_append"
    if s["q"] is not None:
        s["q_out"].copy_(_rotated(s["q"], at, s["inv_freq"], case["inter"]).to(torch.bfloat16))
    k = _rotated(s["k"], at, s["inv_freq"], case["inter"], bits4)
    block, slot = s["table"].long()[slots // bs], slots % bs
    if not bits4:
        store.k_pool[block, :, slot] = k.to(torch.bfloat16)
        store.v_pool[block, :, :, slot] = s["v"]
        return
    _put4(store, s["table"], slots, k, s["v"].float())
    k, v = _take4(store, block, slot)
    s["k_out"][0], s["v_out"][0] = k.to(torch.bfloat16), v.to(torch.bfloat16)


def _plain_decode_append(s):
    case, store = s["case"], s["store"]
    bs, bits4 = case["bs"], case["kind"] == "kv4_step"
    rows = torch.nonzero(s["seq_lens"] > 0)[:, 0]
    slots = s["seq_lens"].long()[rows] - 1
    at = slots + case["shift"]
    s["q_out"][rows] = _rotated(s["q"][rows], at, s["inv_freq"], case["inter"]).to(torch.bfloat16)
    k, v = _rotated(s["k"][rows], at, s["inv_freq"], case["inter"], bits4), s["v"][rows]
    tables = s["tables"][rows]
    block, slot = tables.long().gather(1, (slots // bs)[:, None])[:, 0], slots % bs
    if not bits4:
        store.k_pool[block, :, slot] = k.to(torch.bfloat16)
        store.v_pool[block, :, :, slot] = v
        return
    _put4(store, tables, slots, k, v.float())
    k, v = _take4(store, block, slot)
    s["k_out"].zero_()
    s["v_out"].zero_()
    s["k_out"][rows, 0], s["v_out"][rows, 0] = k.to(torch.bfloat16), v.to(torch.bfloat16)


def _plain_decode(s, q):
    case = s["case"]
    h_kv, window, sinks = case["h_kv"], case["window"], case["sinks"]
    group = case["h_q"] // h_kv
    j, n = torch.arange(s["tables"].shape[1] * case["bs"], device="cuda"), s["seq_lens"].long()[:, None]
    hidden = j >= n
    if window:
        hidden |= (j >= sinks) & (j < n - window)
    hidden = hidden[:, None]
    for h in range(h_kv):
        k, v = _gathered4(s["store"], s["tables"], h)                          # [batch][positions][d]
        heads = slice(h * group, (h + 1) * group)
        scores = torch.matmul(q[:, heads].float(), k.transpose(1, 2).contiguous()) * s["scale"]
        scores = scores.masked_fill_(hidden, -math.inf)
        top = scores.amax(2, keepdim=True)
        e = torch.exp(scores - top).nan_to_num_(0.0)                       # (a row without a sequence)
        total = e.sum(2, keepdim=True)
        s["o"][:, heads] = (torch.matmul(e, v) / total).nan_to_num_(0.0).to(torch.bfloat16)
        s["lse"][:, heads] = (top + torch.log(total))[..., 0].nan_to_num_(neginf=-math.inf)


def _plain_chunk(s):
    case = s["case"]
    p, n, window, sinks = case["prefix"], case["len"], case["window"], case["sinks"]
    group, end = case["h_q"] // case["h_kv"], p + n
    j, t = torch.arange(end, device="cuda"), p + torch.arange(n, device="cuda")[:, None]
    hidden = j > t
    if window:
        hidden |= (j <= t - window) & (j >= sinks)
    for h in range(case["h_kv"]):
        k, v = (x[:end] for x in _gathered4(s["store"], s["table"], h))
        kt = k.t().contiguous()
        for g in range(h * group, (h + 1) * group):
            scores = (s["q"][:, g].float() @ kt * s["scale"]).masked_fill_(hidden, -math.inf)
            top = scores.amax(1, keepdim=True)
            e = torch.exp(scores - top)
            total = e.sum(1, keepdim=True)
            s["o"][:, g] = ((e @ v) / total).to(torch.bfloat16)
            s["lse"][g] = (top + torch.log(total))[:, 0]


def _run_plain(s):
    kind = s["case"]["kind"]
    if kind in ("rope_append", "kv4_append"):
        _plain_append(s)
    elif kind == "kv4_chunk":
        _plain_chunk(s)
    else:
        if kind != "kv4_decode":
            _plain_decode_append(s)
        if kind != "rope_decode":
            _plain_decode(s, s["q"] if kind == "kv4_decode" else s["q_out"])


def run(state):
    if own:
        _run_own(state)
    else:
        _run_plain(state)
    kind = state["case"]["kind"]
    if kind.startswith("rope"):
        names = ("q_out",)
    else:
        names = dict(kv4_append=("q_out", "k_out", "v_out"), kv4_step=("q_out", "o", "lse", "k_out", "v_out"),
                     kv4_decode=("o", "lse"), kv4_chunk=("o", "lse"))[kind]
    out = {name: state[name] for name in names if state[name] is not None}
    if kind.startswith("rope"):
        out.update(k_pool=state["store"].k_pool, v_pool=state["store"].v_pool)
    return out


# ---- What a pass cannot do without ----

def _seen(n, window, sinks):
    """Keys that the query of a sequence of n positions sees."""
    return n if not window or n <= window else min(sinks, n - window) + window


def work(case):
    kind, h_q, h_kv, d = case["kind"], case["h_q"], case["h_kv"], case["d"]
    row4 = d // 2 + d // 32  # a key or value in 4 bits
    if kind == "kv4_chunk":
        p, n, window, sinks = case["prefix"], case["len"], case["window"], case["sinks"]
        pairs = sum(_seen(p + i + 1, window, sinks) for i in range(n))
        keys = p + n
        if window and p + 1 > window:
            keys = min(sinks, p + 1 - window) + window + n - 1
        return {"bytes": float(2 * keys * h_kv * row4 + n * h_q * (4 * d + 4)), "flops": 4.0 * d * h_q * pairs}
    total = dict(bytes=0.0, flops=0.0)
    if kind in ("kv4_step", "kv4_decode"):
        lens = _lens(case)
        keys = sum(_seen(n, case["window"], case["sinks"]) for n in lens)
        total["bytes"] += 2 * keys * h_kv * row4 + len(lens) * h_q * (4 * d + 4)
        total["flops"] += 4.0 * d * h_q * keys
        if kind == "kv4_decode":
            return total
    tokens = case["len"] if "len" in case else sum(n > 0 for n in _lens(case))
    total["flops"] += 3.0 * tokens * (h_q + h_kv) * case["rot"]
    # Q in and out, K and V in, the store; what is loaded from it again.
    total["bytes"] += tokens * (h_q * 4 * d + 2 * h_kv * (2 * d + (2 * d if kind.startswith("rope") else row4)))
    if kind in ("kv4_append", "kv4_step"):
        total["bytes"] += tokens * 2 * h_kv * (row4 + 2 * d)
    return total


# ---- The definition in 64 bits, apart from the plain forms ----

def _exact_rotation(x, positions, case):
    """Pairs as complex numbers, turned by exp(i position inv_freq)."""
    x = x.double()
    rot = case["rot"]
    if rot == 0:
        return x
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda").expand(len(positions), rot // 2),
                       positions.double()[:, None] * _inv_freq(case).double())[:, None]
    out = x.clone()
    if case["inter"]:
        z = torch.view_as_complex(x[..., :rot].unflatten(-1, (-1, 2)).contiguous()) * turn
        out[..., :rot] = torch.view_as_real(z).flatten(-2)
    else:
        z = torch.complex(x[..., :rot // 2], x[..., rot // 2:rot]) * turn
        out[..., :rot // 2], out[..., rot // 2:rot] = z.real, z.imag
    return out


def _exact_rounding(x):
    """The nearest value of the 4-bit format to each of x [n][heads][d], in 64 bits."""
    out = torch.empty_like(x, dtype=torch.float64)
    mags = torch.tensor(_VALUES, dtype=torch.float64, device="cuda")
    order = torch.tensor((0, 2, 4, 6, 1, 3, 5, 7), device="cuda")          # even codes first: argmin takes the first
    for r in range(0, x.shape[0], 1024):
        b = x[r:r + 1024].double().unflatten(-1, (-1, 32))
        top = b.abs().amax(-1, keepdim=True)
        e = torch.floor(torch.log2(top.clamp_min(1e-300))) - 4
        for _ in range(4):
            e = torch.where(top > 6 * torch.exp2(e), e + 1, e)
        e = e.clamp(-125, 125)
        t = b / torch.exp2(e)
        near = order[(t.abs()[..., None] - mags[order]).abs().argmin(-1)]
        out[r:r + 1024] = (torch.copysign(mags[near], t) * torch.exp2(e)).flatten(-2)
    return out


def _exact_values(store, table, n, h):
    """K, V [n][d] of one KV head of a 4-bit store in 64 bits, from sign, exponent and fraction of each code."""
    def value(code, scale):
        code = code.long()
        exponent, fraction = code >> 1 & 3, (code & 1).double()
        mag = torch.where(exponent == 0, 0.5 * fraction, (1 + 0.5 * fraction) * torch.exp2(exponent.double() - 1))
        mag = torch.where(code >= 8, -mag, mag)
        return mag * torch.exp2(scale.double() - 127).repeat_interleave(32, -1)

    bs, d = store.k_pool.shape[2], store.k_pool.shape[3] * 2
    j = torch.arange(n, device="cuda")
    block, slot = table.long()[j // bs], j % bs
    ks, vs = (x[block, h, slot // 64, :, slot % 64] for x in (store.k_scale, store.v_scale))
    kb, vb = store.k_pool[block, h, slot], store.v_pool[block, h, slot // 64, :, slot % 64]
    k, v = (torch.empty((n, d), dtype=torch.uint8, device="cuda") for _ in range(2))
    for half in range(2):
        k[:, half::2] = kb >> 4 * half & 15
    for b in range(d // 32):
        for half in range(2):
            v[:, 32 * b + 16 * half:32 * b + 16 * half + 16] = vb[:, 16 * b:16 * b + 16] >> 4 * half & 15
    return value(k, ks), value(v, vs)


def _exact_attention(q, k, v, positions, scale, window, sinks):
    """O [rows][d] and LSE [rows] of rows at these positions, over keys 0 .. n - 1, in 64 bits."""
    j, t = torch.arange(k.shape[0], device="cuda"), positions[:, None]
    sees = j <= t
    if window:
        sees &= (j > t - window) | (j < sinks)
    s = torch.where(sees, q.double() @ k.t().contiguous() * scale, -math.inf)
    lse = torch.logsumexp(s, 1)
    return torch.exp(s - lse[:, None]) @ v, lse



def exact(case, seed):
    kind, h_kv, h_q, d = case["kind"], case["h_kv"], case["h_q"], case["d"]
    s = prepare(case, seed)
    group = h_q // h_kv
    if kind == "kv4_chunk":
        p, n = case["prefix"], case["len"]
        o = torch.empty((n, h_q, d), dtype=torch.float64, device="cuda")
        lse = torch.empty((h_q, n), dtype=torch.float64, device="cuda")
        at = p + torch.arange(n, device="cuda")
        for g in range(h_q):
            k, v = _exact_values(s["store"], s["table"], p + n, g // group)
            for r in range(0, n, 1024):
                o[r:r + 1024, g], lse[g, r:r + 1024] = _exact_attention(s["q"][r:r + 1024, g], k, v, at[r:r + 1024],
                                                                       s["scale"], case["window"], case["sinks"])
        return dict(o=o, lse=lse)
    if kind in ("rope_append", "kv4_append"):
        p, n, bs = case["prefix"], case["len"], case["bs"]
        slots = p + torch.arange(n, device="cuda")
        at = slots + case["shift"]
        out = {} if s["q"] is None else dict(q_out=_exact_rotation(s["q"], at, case))
        k = _exact_rotation(s["k"], at, case)
        if kind == "kv4_append":
            return dict(out, k_out=_exact_rounding(k)[None], v_out=_exact_rounding(s["v"])[None])
        k_pool, v_pool = s["store"].k_pool.double(), s["store"].v_pool.double()
        for i in range(0, n):
            block, slot = s["table"][(p + i) // bs].long(), (p + i) % bs
            k_pool[block, :, slot], v_pool[block, :, :, slot] = k[i], s["v"][i].double()
        return dict(out, k_pool=k_pool, v_pool=v_pool)
    lens = _lens(case)
    if kind in ("rope_decode", "kv4_step"):
        at = torch.tensor(lens, device="cuda") - 1 + case["shift"]
        q, k = _exact_rotation(s["q"], at, case), _exact_rotation(s["k"], at, case)
        q[s["seq_lens"] <= 0] = 0.0
    if kind == "rope_decode":
        k_pool, v_pool = s["store"].k_pool.double(), s["store"].v_pool.double()
        for b, n in enumerate(lens):
            if n > 0:
                block, slot = s["tables"][b, (n - 1) // case["bs"]].long(), (n - 1) % case["bs"]
                k_pool[block, :, slot], v_pool[block, :, :, slot] = k[b], s["v"][b].double()
        return dict(q_out=q, k_pool=k_pool, v_pool=v_pool)
    o = torch.zeros((len(lens), h_q, d), dtype=torch.float64, device="cuda")
    lse = torch.full((len(lens), h_q), -math.inf, dtype=torch.float64, device="cuda")
    out = dict(o=o, lse=lse)
    if kind == "kv4_step":
        k, v = _exact_rounding(k)[:, None], _exact_rounding(s["v"])[:, None]
        k[s["seq_lens"] <= 0] = 0.0
        v[s["seq_lens"] <= 0] = 0.0
        out.update(q_out=q, k_out=k, v_out=v)
        q = q.to(torch.bfloat16)  # the attention's own input is in bf16
    else:
        q = s["q"]
    for b, n in enumerate(lens):
        for h in range(h_kv if n > 0 else 0):
            ks, vs = _exact_values(s["store"], s["tables"][b], n, h)
            if kind == "kv4_step":
                ks[n - 1], vs[n - 1] = k[b, 0, h], v[b, 0, h]
            heads = slice(h * group, (h + 1) * group)
            at = torch.full((group,), n - 1, device="cuda")
            o[b, heads], lse[b, heads] = _exact_attention(q[b, heads], ks, vs, at, s["scale"], case["window"],
                                                          case["sinks"])
    return out
