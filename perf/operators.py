"""Performance cases of the operators that follow the prefill: decoding over the
paged store, attention in a sliding window with sinks, accumulated key weights
and the eviction that goes by them.

Kinds of pass:

  decode         ``mocap_decode_attn``: one new token of each sequence of a batch
                 against its paged keys and values.  Returns O and LSE.
  decode_step    ``mocap_decode_append`` of the new tokens, then the same
                 attention.  Returns O, LSE and the pools.
  window         ``mocap_window_attn``: one chunk whose rows see a window of keys
                 and the first few.  Returns O and LSE.
  weights        ``mocap_key_weights``: the attention weight each key of the store
                 received from a chunk's rows, added to what it had.  Returns the
                 weights.
  decode_weights ``mocap_decode_key_weights``: the same for the new token of each
                 sequence of a batch.  Returns the weights of all sequences.
  evict          ``mocap_kv_evict``: the heaviest keys of each head, compacted into
                 other blocks.  Returns the kept positions, their weights and the
                 destination pools.

Pools hold N(0, 1) in bf16, as do the queries; score scale 1/sqrt(head_dim);
every sequence's blocks lie at permuted places of one pool.
"""
import math

import torch

own = False

# (query heads, KV heads, head_dim) of the layers that the library is tested with.
HEADS = ((32, 8, 128), (64, 8, 128), (8, 8, 64), (8, 4, 128), (8, 2, 128), (16, 2, 64), (12, 4, 128),
         (32, 1, 128), (64, 1, 64), (6, 3, 128))


def listed():
    return [
        # One short conversation, plain multi-head layer: bound by latency.
        dict(name="decode_one_short", kind="decode_step", h_q=8, h_kv=8, d=64, bs=64, lens="572", window=0, sinks=0),
        # A serving batch whose conversations have very different lengths (one to a few thousand tokens).
        dict(name="decode_batch_ragged", kind="decode_step", h_q=32, h_kv=8, d=128, bs=256,
             lens="1,7,63,64,65,129,200,255,257,400,513,777,1000,1023,1500,1999,2048,2100,2500,2777,3001,3333,4096,"
                  "4097,4500,5001,5555,6001,6500,7001,7777,8192", window=0, sinks=0),
        # Long documents under a 70B layer: the largest decode, bound by HBM.
        dict(name="decode_70b_long", kind="decode", h_q=64, h_kv=8, d=128, bs=256, lens="131072,120001,65537,98304",
             window=0, sinks=0),
        # Streaming sessions: long histories of which a window and a few first tokens are read.
        dict(name="decode_window", kind="decode", h_q=32, h_kv=8, d=128, bs=256,
             lens="4097,9001,16384,20011,30720,32768,50001,65536,3000,100,12345,28000,40000,61000,8191,17",
             window=4096, sinks=4),
        # An ordinary chunk of a long prompt with a 4096-token window.
        dict(name="window_8b_2048", kind="window", h_q=32, h_kv=8, d=128, bs=256, prefix=30720, len=2048, window=4096,
             sinks=4),
        # The odd remainder of a prompt, small heads, a short window and a block of sinks.
        dict(name="window_tail_d64", kind="window", h_q=16, h_kv=2, d=64, bs=192, prefix=9001, len=137, window=1000,
             sinks=64),
        # Scores of every key of a long prompt from one chunk of queries: the largest arithmetic.
        dict(name="weights_8b_2048", kind="weights", h_q=32, h_kv=8, d=128, bs=256, prefix=30720, len=2048, prev=True),
        # The last tokens of a prompt as observers of all its keys, before an eviction.
        dict(name="weights_observers", kind="weights", h_q=32, h_kv=8, d=128, bs=256, prefix=65501, len=32, prev=False),
        # One session at a time: latency.
        dict(name="decode_weights_one", kind="decode_weights", h_q=8, h_kv=2, d=128, bs=128, lens="3001", prev=True),
        # A batch of sessions that keep their keys' weights up to date at every token.
        dict(name="decode_weights_batch", kind="decode_weights", h_q=32, h_kv=8, d=128, bs=256,
             lens="32768,20011,16384,30001,12000,8192,27777,32001,64,5000,24001,18000,9001,31000,15000,28001", prev=True),
        # The cache of a short prompt, cut to a third.
        dict(name="evict_short", kind="evict", h_kv=4, d=128, bs=64, n=1571, keep=500, sinks=4, recent=64),
        # The cache of a long prompt, cut to an eighth.
        dict(name="evict_8b_128k", kind="evict", h_kv=8, d=128, bs=256, n=131072, keep=16384, sinks=4, recent=1024),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Another case of the listed ranges: batches of 1 to 64 sequences of 1 to
    131072 tokens; windows of 1 to 16384; chunks of 1 to 4096 rows behind 0 to
    65536 keys; caches of 64 to 262144 positions; every head layout and block
    sizes from 64 to 1600."""
    kind = rng.choice(("decode", "decode_step", "window", "weights", "decode_weights", "evict"))
    h_q, h_kv, d = rng.choice(HEADS[:2] + HEADS)
    case = dict(kind=kind, h_q=h_q, h_kv=h_kv, d=d, bs=rng.choice((64, 128, 192, 256, 256, 320, 1600)))
    if kind in ("decode", "decode_step", "decode_weights"):
        batch = _log_int(rng, 1, 64)
        top = min(131072, 400000 // batch) if kind != "decode_step" else min(32768, 100000 // batch)
        low = rng.choice((1, 64, max(64, top // 4)))
        case.update(lens=",".join(str(_log_int(rng, low, top)) for _ in range(batch)))
        if kind == "decode_weights":
            return dict(case, prev=rng.random() < 0.7)
        if rng.random() < 0.4:
            return dict(case, window=_log_int(rng, 1, 16384), sinks=rng.choice((0, 1, 4, 64, 100)))
        return dict(case, window=0, sinks=0)
    if kind == "evict":
        n = _log_int(rng, 64, 262144)
        keep = max(1, min(n, _log_int(rng, max(1, n // 32), n), 65536))
        sinks = min(rng.choice((0, 4, 64)), keep)
        recent = min(_log_int(rng, 1, max(1, keep)), keep - sinks)
        return dict(case, n=n, keep=keep, sinks=sinks, recent=recent)
    rows = _log_int(rng, 1, 4096)
    prefix = rng.choice((0, 256 * rng.randint(1, 128), _log_int(rng, 64, 65536)))
    # No more arithmetic than the largest listed case.
    if kind == "window":
        window = min(_log_int(rng, 1, 8192), int(3.9e11 / (4.0 * d * h_q * rows)))
        return dict(case, prefix=prefix, len=rows, window=window, sinks=rng.choice((0, 1, 4, 64, 100)))
    prefix = min(prefix, int(3.9e11 / (2.0 * d * h_q * rows)))
    return dict(case, prefix=prefix, len=rows, prev=rng.random() < 0.5)


class _Store:
    """Block pools in the library's layout: K [blocks][Hkv][bs][d], V [blocks][Hkv][d][bs]."""

    def __init__(self, blocks, bs, h_kv, d):
        self.k_pool = torch.zeros((blocks, h_kv, bs, d), dtype=torch.bfloat16, device="cuda")
        self.v_pool = torch.zeros((blocks, h_kv, d, bs), dtype=torch.bfloat16, device="cuda")


def _binding():
    from paper_2606_22968_amd import binding
    return binding


def _store(case, blocks):
    if own:
        return _binding().KvStore(blocks, case["bs"], case["h_kv"], case["d"], fill=0.0)
    return _Store(blocks, case["bs"], case["h_kv"], case["d"])


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


def _fill(store, seed):
    """Both pools N(0, 1), drawn in pool order."""
    for i, pool in enumerate((store.k_pool, store.v_pool)):
        g = torch.Generator(device="cuda")
        g.manual_seed(7919 * seed + i)
        pool.normal_(generator=g)


def _batch_tables(case, seed):
    """[batch][longest] block tables on the CPU, every sequence's blocks its own."""
    lens = _lens(case)
    need = [_blocks(case, n) for n in lens]
    perm = _perm(seed + 1, sum(need))
    tables = torch.zeros((len(lens), max(need)), dtype=torch.int32)
    at = 0
    for b, m in enumerate(need):
        tables[b, :m] = perm[at:at + m]
        at += m
    return tables


def _base_weights(seed, shape):
    """What earlier queries gave the keys: heavy-tailed, as attention weights are."""
    return torch.exp(2.0 * _randn(seed + 5, shape, torch.float32) - 4.0)


def _evict_weights(case, seed):
    """Heavy-tailed weights; a fifth of the keys received none (equal ones)."""
    w = _base_weights(seed, (case["h_kv"], case["n"]))
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + 6)
    w[torch.rand(w.shape, generator=g, device="cuda") < 0.2] = 0.0
    return w


def _gathered(store, table, h, n):
    """K, V [n][d] of one KV head at positions 0 .. n - 1, in 32 bits."""
    at = table.long()
    k = store.k_pool[at, h].float()                                # [blocks][bs][d]
    v = store.v_pool[at, h].float().transpose(1, 2)                # [blocks][bs][d]
    d = k.shape[-1]
    return k.reshape(-1, d)[:n], v.reshape(-1, d)[:n]


def _row_lse(q, store, table, prefix, scale):
    """LSE [Hq][rows] of causal attention, in 32 bits: an input of the weight cases."""
    rows, h_q, _ = q.shape
    h_kv = store.k_pool.shape[1]
    n, group = prefix + rows, h_q // h_kv
    lse = torch.empty((h_q, rows), dtype=torch.float32, device="cuda")
    hidden = torch.arange(n, device="cuda")[None, :] > prefix + torch.arange(rows, device="cuda")[:, None]
    for h in range(h_kv):
        kt = _gathered(store, table, h, n)[0].t().contiguous()
        for g in range(h * group, (h + 1) * group):
            lse[g] = torch.logsumexp((q[:, g].float() @ kt * scale).masked_fill_(hidden, -math.inf), 1)
    return lse


def prepare(case, seed):
    kind, h_kv, d = case["kind"], case["h_kv"], case["d"]
    state = dict(case=case, scale=_scale(case))
    if kind == "evict":
        src = _store(case, _blocks(case, case["n"]))
        _fill(src, seed)
        state.update(src=src, src_table=_perm(seed + 1, _blocks(case, case["n"])).cuda(),
                     dst=_store(case, _blocks(case, case["keep"])),
                     dst_table=_perm(seed + 2, _blocks(case, case["keep"])).cuda(), weights=_evict_weights(case, seed),
                     kept=torch.empty((h_kv, case["keep"]), dtype=torch.int32, device="cuda"),
                     kept_weights=torch.empty((h_kv, case["keep"]), dtype=torch.float32, device="cuda"))
        if own:
            state["workspace"] = torch.empty(
                max(_binding().mocap_kv_evict_workspace_size(case["n"], h_kv, case["keep"]), 16), dtype=torch.uint8,
                device="cuda")
        return state
    h_q = case["h_q"]
    if kind in ("window", "weights"):
        p, n = case["prefix"], case["len"]
        blocks = _blocks(case, p + n)
        store, table = _store(case, blocks), _perm(seed + 1, blocks).cuda()
        _fill(store, seed)
        q = _randn(seed + 3, (n, h_q, d))
        state.update(store=store, table=table, q=q)
        if kind == "window":
            state.update(o=torch.empty_like(q), lse=torch.empty((h_q, n), dtype=torch.float32, device="cuda"))
            size = own and _binding().mocap_window_attn_workspace_size(p, n, h_q, h_kv, d, case["window"],
                                                                       case["sinks"])[1]
        else:
            state.update(lse=_row_lse(q, store, table, p, state["scale"]),
                         prev=_base_weights(seed, (h_kv, p + n)) if case["prev"] else None,
                         weights=torch.empty((h_kv, p + n), dtype=torch.float32, device="cuda"))
            size = own and _binding().mocap_key_weights_workspace_size(p, n, h_q, h_kv, d)
        if own:
            state["workspace"] = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")
        return state
    lens = _lens(case)
    tables = _batch_tables(case, seed)
    store = _store(case, sum(_blocks(case, n) for n in lens))
    _fill(store, seed)
    q = _randn(seed + 3, (len(lens), h_q, d))
    state.update(store=store, lens=lens, tables=tables.cuda(), seq_lens=torch.tensor(lens, dtype=torch.int32).cuda(),
                 max_len=max(lens), q=q)
    if kind == "decode_weights":
        shape = (len(lens), h_kv, max(lens))
        lse = torch.empty((len(lens), h_q), dtype=torch.float32, device="cuda")
        for b, n in enumerate(lens):
            lse[b] = _row_lse(q[b:b + 1], store, state["tables"][b, :_blocks(case, n)], n - 1, state["scale"])[:, 0]
        return dict(state, lse=lse, prev=_base_weights(seed, shape) if case["prev"] else None,
                    weights=torch.zeros(shape, dtype=torch.float32, device="cuda"))
    if kind == "decode_step":
        state.update(k=_randn(seed + 8, (len(lens), h_kv, d)), v=_randn(seed + 9, (len(lens), h_kv, d)))
    state.update(o=torch.empty_like(q), lse=torch.empty((len(lens), h_q), dtype=torch.float32, device="cuda"))
    if own:
        size = _binding().mocap_decode_attn_workspace_size(len(lens), h_q, h_kv, d, max(lens), case["window"],
                                                           case["sinks"])
        state["workspace"] = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")
    return state


def _run_own(s):
    binding, case = _binding(), s["case"]
    kind = case["kind"]
    if kind == "evict":
        binding.mocap_kv_evict(s["src"], s["src_table"], s["dst"], s["dst_table"], case["n"], case["keep"], case["sinks"],
                               case["recent"], s["weights"], s["kept"], s["kept_weights"], s["workspace"])
        return dict(kept=s["kept"], kept_weights=s["kept_weights"], k_pool=s["dst"].k_pool, v_pool=s["dst"].v_pool)
    if kind == "window":
        binding.mocap_window_attn(s["store"], s["table"], s["q"], case["prefix"], s["scale"], case["window"],
                                  case["sinks"], s["o"], s["lse"], s["workspace"])
        return dict(o=s["o"], lse=s["lse"])
    if kind == "weights":
        binding.mocap_key_weights(s["store"], s["table"], s["q"], case["prefix"], s["scale"], s["lse"], s["prev"],
                                  s["weights"], s["workspace"])
        return dict(weights=s["weights"])
    if kind == "decode_weights":
        binding.mocap_decode_key_weights(s["store"], s["tables"], s["seq_lens"], s["q"], s["max_len"], s["scale"],
                                         s["lse"], s["prev"], s["weights"])
        return dict(weights=s["weights"])
    if kind == "decode_step":
        binding.mocap_decode_append(s["store"], s["tables"], s["seq_lens"], s["k"], s["v"])
    binding.mocap_decode_attn(s["store"], s["tables"], s["seq_lens"], s["q"], s["max_len"], s["scale"], s["o"], s["lse"],
                              s["workspace"], case["window"], case["sinks"])
    if kind == "decode_step":
        return dict(o=s["o"], lse=s["lse"], k_pool=s["store"].k_pool, v_pool=s["store"].v_pool)
    return dict(o=s["o"], lse=s["lse"])


def _softmax_rows(scores, v):
    """O and LSE of rows of scores (hidden ones -inf)."""
    top = scores.amax(1, keepdim=True)
    e = torch.exp(scores - top)
    total = e.sum(1, keepdim=True)
    return (e @ v) / total, (top + torch.log(total))[:, 0]


def _plain_decode(s):
    case, store = s["case"], s["store"]
    h_kv, bs, window, sinks = case["h_kv"], case["bs"], case["window"], case["sinks"]
    group = case["h_q"] // h_kv
    if case["kind"] == "decode_step":
        for b, n in enumerate(s["lens"]):
            block, slot = s["tables"][b, (n - 1) // bs].long(), (n - 1) % bs
            store.k_pool[block, :, slot] = s["k"][b]
            store.v_pool[block, :, :, slot] = s["v"][b]
    for b, n in enumerate(s["lens"]):
        table = s["tables"][b, :_blocks(case, n)].long()
        k = store.k_pool[table].float().transpose(0, 1).reshape(h_kv, -1, case["d"])[:, :n]
        v = store.v_pool[table].float().permute(1, 0, 3, 2).reshape(h_kv, -1, case["d"])[:, :n]
        if window and n > window:
            first = n - window
            keep = torch.arange(n, device="cuda")
            keep = (keep < sinks) | (keep >= first)
            k, v = k[:, keep], v[:, keep]
        scores = torch.matmul(s["q"][b].float().reshape(h_kv, group, -1), k.transpose(1, 2).contiguous()) * s["scale"]
        top = scores.amax(2, keepdim=True)
        e = torch.exp(scores - top)
        total = e.sum(2, keepdim=True)
        s["o"][b] = (torch.matmul(e, v.contiguous()) / total).reshape(case["h_q"], -1).to(torch.bfloat16)
        s["lse"][b] = (top + torch.log(total)).reshape(-1)


def _plain_window(s):
    case = s["case"]
    p, n, window, sinks = case["prefix"], case["len"], case["window"], case["sinks"]
    group = case["h_q"] // case["h_kv"]
    rows = 1024
    for h in range(case["h_kv"]):
        k, v = _gathered(s["store"], s["table"], h, p + n)
        for r in range(0, n, rows):
            e = min(n, r + rows)
            low = max(0, p + r - window + 1)
            keys = torch.cat((torch.arange(min(sinks, low), device="cuda"), torch.arange(low, p + e, device="cuda")))
            kt, vs = k[keys].t().contiguous(), v[keys]
            t = p + torch.arange(r, e, device="cuda")[:, None]
            hidden = (keys > t) | ((keys <= t - window) & (keys >= sinks))
            for g in range(h * group, (h + 1) * group):
                scores = (s["q"][r:e, g].float() @ kt * s["scale"]).masked_fill_(hidden, -math.inf)
                o, s["lse"][g, r:e] = _softmax_rows(scores, vs)
                s["o"][r:e, g] = o.to(torch.bfloat16)


def _plain_weights(s):
    case = s["case"]
    p, n = case["prefix"], case["len"]
    group = case["h_q"] // case["h_kv"]
    hidden = torch.arange(n, device="cuda")[None, :] > torch.arange(n, device="cuda")[:, None]
    for h in range(case["h_kv"]):
        kt = _gathered(s["store"], s["table"], h, p + n)[0].t().contiguous()
        # Many small terms: the total is kept in 64 bits.
        total = torch.zeros(p + n, dtype=torch.float64, device="cuda")
        for g in range(h * group, (h + 1) * group):
            w = torch.exp(s["q"][:, g].float() @ kt * s["scale"] - s["lse"][g][:, None])
            w[:, p:].masked_fill_(hidden, 0.0)
            total += w.sum(0)
        if s["prev"] is not None:
            total[:p] += s["prev"][h, :p]
        s["weights"][h] = total.float()


def _plain_decode_weights(s):
    case = s["case"]
    h_kv, group = case["h_kv"], case["h_q"] // case["h_kv"]
    for b, n in enumerate(s["lens"]):
        table = s["tables"][b, :_blocks(case, n)].long()
        k = s["store"].k_pool[table].float().transpose(0, 1).reshape(h_kv, -1, case["d"])[:, :n]
        scores = torch.matmul(s["q"][b].float().reshape(h_kv, group, -1), k.transpose(1, 2).contiguous()) * s["scale"]
        w = torch.exp(scores - s["lse"][b].reshape(h_kv, group, 1)).sum(1)
        if s["prev"] is not None:
            w[:, :n - 1] += s["prev"][b, :, :n - 1]
        s["weights"][b, :, :n] = w


def _plain_evict(s):
    case, src, dst = s["case"], s["src"], s["dst"]
    n, keep, sinks, recent, bs = case["n"], case["keep"], case["sinks"], case["recent"], case["bs"]
    # Largest first, the lower position first among equal ones.
    order = torch.sort(s["weights"][:, sinks:n - recent], dim=1, descending=True, stable=True).indices + sinks
    picked = order[:, :keep - sinks - recent]
    head = torch.arange(sinks, device="cuda").expand(case["h_kv"], -1)
    tail = torch.arange(n - recent, n, device="cuda").expand(case["h_kv"], -1)
    kept = torch.sort(torch.cat((head, picked, tail), 1), dim=1).values
    s["kept"].copy_(kept)
    s["kept_weights"].copy_(torch.gather(s["weights"], 1, kept))
    at = torch.arange(keep, device="cuda")
    to_block, to_slot = s["dst_table"].long()[at // bs], at % bs
    for h in range(case["h_kv"]):
        block, slot = s["src_table"].long()[kept[h] // bs], kept[h] % bs
        dst.k_pool[to_block, h, to_slot] = src.k_pool[block, h, slot]
        dst.v_pool[to_block, h, :, to_slot] = src.v_pool[block, h, :, slot]


def run(state):
    if own:
        return _run_own(state)
    kind = state["case"]["kind"]
    if kind == "evict":
        _plain_evict(state)
        return dict(kept=state["kept"], kept_weights=state["kept_weights"], k_pool=state["dst"].k_pool,
                    v_pool=state["dst"].v_pool)
    if kind in ("weights", "decode_weights"):
        (_plain_weights if kind == "weights" else _plain_decode_weights)(state)
        return dict(weights=state["weights"])
    (_plain_window if kind == "window" else _plain_decode)(state)
    out = dict(o=state["o"], lse=state["lse"])
    if kind == "decode_step":
        out.update(k_pool=state["store"].k_pool, v_pool=state["store"].v_pool)
    return out


def _seen(t, window, sinks):
    """Keys that the row at position t sees."""
    if not window or t < window:
        return t + 1
    return window + min(sinks, t + 1 - window)


def work(case):
    """Keys and values that are looked at read once, queries and statistics read
    or written once; 4 d FLOP per query head and visible (row, key) pair of an
    attention, 2 d of a weight."""
    kind, h_kv, d = case["kind"], case["h_kv"], case["d"]
    if kind == "evict":
        return dict(bytes=4 * case["n"] * h_kv + 8 * case["keep"] * h_kv * d + 8 * case["keep"] * h_kv, flops=0)
    h_q = case["h_q"]
    if kind in ("window", "weights"):
        p, n = case["prefix"], case["len"]
        if kind == "weights":
            return dict(bytes=2 * (p + n) * h_kv * d + 2 * n * h_q * d + 4 * n * h_q
                        + 4 * h_kv * (p + n + (p if case["prev"] else 0)),
                        flops=2 * d * h_q * (n * p + n * (n + 1) // 2))
        low = max(0, p - case["window"] + 1)
        keys = p + n - low + min(case["sinks"], low)
        pairs = sum(_seen(t, case["window"], case["sinks"]) for t in range(p, p + n))
        return dict(bytes=4 * keys * h_kv * d + 4 * n * h_q * d + 4 * n * h_q, flops=4 * d * h_q * pairs)
    lens = _lens(case)
    if kind == "decode_weights":
        keys = sum(lens)
        return dict(bytes=2 * keys * h_kv * d + len(lens) * h_q * (2 * d + 4)
                    + 4 * h_kv * (2 if case["prev"] else 1) * keys, flops=2 * d * h_q * keys)
    keys = sum(_seen(n - 1, case["window"], case["sinks"]) for n in lens)
    total = 4 * keys * h_kv * d + len(lens) * h_q * (4 * d + 4)
    if kind == "decode_step":
        total += 4 * len(lens) * h_kv * d
    return dict(bytes=total, flops=4 * d * h_q * keys)


def _refilled(case, seed, blocks):
    """The pools that prepare() fills from this seed."""
    store = _Store(blocks, case["bs"], case["h_kv"], case["d"])
    _fill(store, seed)
    return store


def _exact_keys(case, store, table, h, pos):
    """K, V [len(pos)][d] of one KV head at given positions, in 64 bits."""
    block, slot = table[pos // case["bs"]].long(), pos % case["bs"]
    return store.k_pool[block, h, slot].double(), store.v_pool[block, h, :, slot].double()


def _exact_decode(case, seed):
    lens, tables = _lens(case), _batch_tables(case, seed).cuda()
    store = _refilled(case, seed, sum(_blocks(case, n) for n in lens))
    q = _randn(seed + 3, (len(lens), case["h_q"], case["d"]))
    group, bs = case["h_q"] // case["h_kv"], case["bs"]
    out = {}
    if case["kind"] == "decode_step":
        k, v = (_randn(seed + i, (len(lens), case["h_kv"], case["d"])) for i in (8, 9))
        last = torch.tensor(lens, device="cuda") - 1
        block = tables[torch.arange(len(lens), device="cuda"), last // bs].long()
        store.k_pool[block, :, last % bs] = k
        store.v_pool[block, :, :, last % bs] = v
        out.update(k_pool=store.k_pool.double(), v_pool=store.v_pool.double())
    if case["kind"] == "decode_weights":
        prev = _base_weights(seed, (len(lens), case["h_kv"], max(lens))) if case["prev"] else None
        w = torch.zeros((len(lens), case["h_kv"], max(lens)), dtype=torch.float64, device="cuda")
        for b, n in enumerate(lens):
            row_lse = _row_lse(q[b:b + 1], store, tables[b, :_blocks(case, n)], n - 1, _scale(case))[:, 0].double()
            for h in range(case["h_kv"]):
                k = _exact_keys(case, store, tables[b], h, torch.arange(n, device="cuda"))[0]
                for g in range(h * group, (h + 1) * group):
                    w[b, h, :n] += torch.exp((k @ q[b, g].double()) * _scale(case) - row_lse[g])
            if prev is not None:
                w[b, :, :n - 1] += prev[b, :, :n - 1]
        return dict(weights=w)
    o = torch.empty((len(lens), case["h_q"], case["d"]), dtype=torch.float64, device="cuda")
    lse = torch.empty((len(lens), case["h_q"]), dtype=torch.float64, device="cuda")
    for b, n in enumerate(lens):
        pos = torch.arange(n, device="cuda")
        if case["window"]:
            pos = pos[(pos < case["sinks"]) | (pos > n - 1 - case["window"])]
        for h in range(case["h_kv"]):
            k, v = _exact_keys(case, store, tables[b], h, pos)
            for g in range(h * group, (h + 1) * group):
                scores = (k @ q[b, g].double()) * _scale(case)
                lse[b, g] = torch.logsumexp(scores, 0)
                o[b, g] = torch.exp(scores - lse[b, g]) @ v
    return dict(out, o=o, lse=lse)


def _exact_chunk(case, seed):
    p, n, bs = case["prefix"], case["len"], case["bs"]
    table = _perm(seed + 1, _blocks(case, p + n)).cuda()
    store = _refilled(case, seed, table.numel())
    q = _randn(seed + 3, (n, case["h_q"], case["d"]))
    group, scale = case["h_q"] // case["h_kv"], _scale(case)
    at = torch.arange(p + n, device="cuda")
    if case["kind"] == "weights":
        row_lse = _row_lse(q, store, table, p, scale).double()
        w = torch.zeros((case["h_kv"], p + n), dtype=torch.float64, device="cuda")
        for h in range(case["h_kv"]):
            k = _exact_keys(case, store, table, h, at)[0]
            for g in range(h * group, (h + 1) * group):
                for r in range(0, n, 512):
                    e = min(n, r + 512)
                    part = torch.exp((k @ q[r:e, g].double().t().contiguous()) * scale - row_lse[g, r:e])
                    part[at[:, None] > p + torch.arange(r, e, device="cuda")[None, :]] = 0.0
                    w[h] += part.sum(1)
        if case["prev"]:
            w[:, :p] += _base_weights(seed, (case["h_kv"], p + n))[:, :p]
        return dict(weights=w)
    o = torch.empty((n, case["h_q"], case["d"]), dtype=torch.float64, device="cuda")
    lse = torch.empty((case["h_q"], n), dtype=torch.float64, device="cuda")
    for r in range(0, n, 512):
        e = min(n, r + 512)
        row = p + torch.arange(r, e, device="cuda")
        pos = at[(at < p + e) & ((at < case["sinks"]) | (at > p + r - case["window"]))]
        seen = (pos[None, :] <= row[:, None]) & ((pos[None, :] < case["sinks"]) |
                                                 (row[:, None] - pos[None, :] < case["window"]))
        for h in range(case["h_kv"]):
            k, v = _exact_keys(case, store, table, h, pos)
            for g in range(h * group, (h + 1) * group):
                scores = torch.where(seen, (q[r:e, g].double() @ k.t().contiguous()) * scale, -math.inf)
                lse[g, r:e] = torch.logsumexp(scores, 1)
                o[r:e, g] = torch.exp(scores - lse[g, r:e, None]) @ v
    return dict(o=o, lse=lse)


def _exact_evict(case, seed):
    n, keep, bs = case["n"], case["keep"], case["bs"]
    table, to = _perm(seed + 1, _blocks(case, n)).cuda(), _perm(seed + 2, _blocks(case, keep)).cuda()
    store = _refilled(case, seed, table.numel())
    w = _evict_weights(case, seed).double()
    # Positions that are always kept rank above every weight; the rank of a
    # position is the number of those before it in the order of eviction.
    rank = w.clone()
    rank[:, :case["sinks"]] = math.inf
    rank[:, n - case["recent"]:] = math.inf
    kept = torch.empty((case["h_kv"], keep), dtype=torch.int64, device="cuda")
    for h in range(case["h_kv"]):
        values = torch.sort(rank[h], descending=True).values
        border = values[keep - 1]
        above = rank[h] > border
        equal = torch.nonzero(rank[h] == border)[:, 0][:keep - int(above.sum())]
        above[equal] = True
        kept[h] = torch.nonzero(above)[:, 0]
    k_pool = torch.zeros((to.numel(), case["h_kv"], bs, case["d"]), dtype=torch.float64, device="cuda")
    v_pool = torch.zeros((to.numel(), case["h_kv"], case["d"], bs), dtype=torch.float64, device="cuda")
    at = torch.arange(keep, device="cuda")
    for h in range(case["h_kv"]):
        k, v = _exact_keys(case, store, table, h, kept[h])
        k_pool[to[at // bs].long(), h, at % bs] = k
        v_pool[to[at // bs].long(), h, :, at % bs] = v
    return dict(kept=kept, kept_weights=torch.gather(w, 1, kept), k_pool=k_pool, v_pool=v_pool)


def exact(case, seed):
    """What run() returns, from the definitions in float64 torch."""
    if case["kind"] == "evict":
        return _exact_evict(case, seed)
    if case["kind"] in ("window", "weights"):
        return _exact_chunk(case, seed)
    return _exact_decode(case, seed)
