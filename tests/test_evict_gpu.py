"""mocap_kv_evict against the definition: which positions stay, in order, bit for
bit, wherever the blocks lie; ties, zeros, infinities and NaN; and what is not
written."""
import math

import pytest
import torch

from helpers import say
from paper_2606_22968_amd import binding
from serve_helpers import make_store, take

pytestmark = pytest.mark.gpu


def expected(weights, n, keep, sinks, recent):
    """Kept positions of one head, from the definition: an ordinary sort by
    (weight descending, position ascending), NaN first, -0 as 0."""
    w = [float(x) for x in weights[:n]]
    middle = sorted(range(sinks, n - recent), key=lambda i: (not math.isnan(w[i]), 0.0 if math.isnan(w[i]) else -w[i], i))
    return sorted(list(range(sinks)) + middle[:keep - sinks - recent] + list(range(n - recent, n)))


def evict(src, src_table, weights, n, keep, sinks, recent, dst=None, dst_bs=None, spare=2, kept_weights=True):
    dst_bs = dst_bs or src.block_size
    blocks = -(-keep // dst_bs)
    if dst is None:
        dst = binding.KvStore(blocks + spare, dst_bs, src.h_kv, src.head_dim, fill=7.0)
    table = torch.randperm(blocks + spare, generator=torch.Generator().manual_seed(keep))[:blocks].to(torch.int32).cuda()
    kept = torch.full((src.h_kv, keep), -1, dtype=torch.int32, device="cuda")
    kw = torch.full((src.h_kv, keep), -1.0, device="cuda") if kept_weights else None
    size = binding.mocap_kv_evict_workspace_size(n, src.h_kv, keep)
    ws = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda").fill_(0xFF)
    binding.mocap_kv_evict(src, src_table, dst, table, n, keep, sinks, recent, weights, kept, kw, ws)
    torch.cuda.synchronize()
    return dst, table, kept.cpu(), kw


def check(src, ks, vs, weights, n, keep, sinks, recent, dst, table, kept, kw):
    pos = torch.arange(keep)
    got_k, got_v = take(dst, table, keep)
    for h in range(src.h_kv):
        want = expected(weights[h].cpu(), n, keep, sinks, recent)
        assert kept[h].tolist() == want, f"head {h}"
        assert torch.equal(got_k[:, h].view(torch.int16), ks[want, h].view(torch.int16))
        assert torch.equal(got_v[:, h].view(torch.int16), vs[want, h].view(torch.int16))
        if kw is not None:
            assert torch.equal(kw[h].cpu().view(torch.int32), weights[h].cpu()[want].view(torch.int32))
    # Everything else of dst is as it was.
    written = torch.zeros(dst.num_blocks, dst.block_size, dtype=torch.bool)
    written[table.cpu().long()[pos // dst.block_size], pos % dst.block_size] = True
    assert (dst.k_pool.cpu().transpose(1, 2)[~written] == 7.0).all()
    assert (dst.v_pool.cpu().permute(0, 3, 1, 2)[~written] == 7.0).all()


def weights_of(kind, h_kv, n, seed):
    g = torch.Generator(device="cpu")
    g.manual_seed(seed)
    w = torch.exp(3 * torch.randn((h_kv, n + 3), generator=g))
    if kind == "ties":
        w = torch.randint(0, 4, (h_kv, n + 3), generator=g).float()
    elif kind == "equal":
        w = torch.full((h_kv, n + 3), 0.5)
    elif kind == "special":
        r = torch.randint(0, 8, (h_kv, n + 3), generator=g)
        for value, x in enumerate((float("nan"), math.inf, -math.inf, -0.0, 0.0, 1e-45, -1.5)):
            w[r == value] = x
    elif kind == "close":  # keys that differ in their last bits
        w = (torch.randint(0, 1000, (h_kv, n + 3), generator=g, dtype=torch.int32) + 0x3F800000).view(torch.float32)
    return w.cuda()


@pytest.mark.parametrize("kind", ["heavy", "ties", "equal", "special", "close"])
@pytest.mark.parametrize("h_kv,d,bs,n,keep,sinks,recent", [
    (2, 128, 64, 1, 1, 0, 0), (2, 128, 64, 1, 1, 1, 0), (3, 64, 64, 65, 64, 4, 8), (1, 64, 192, 700, 100, 0, 0),
    (4, 128, 64, 1571, 500, 4, 64), (2, 64, 128, 1000, 1000, 4, 64), (2, 64, 128, 1000, 999, 0, 0),
    (2, 64, 64, 1000, 68, 4, 64), (2, 128, 64, 1024, 1, 0, 0), (2, 64, 64, 3000, 129, 0, 129), (8, 128, 256, 5000, 1025, 64, 1)])
def test_selection_and_copy(gpu, kind, h_kv, d, bs, n, keep, sinks, recent):
    say(f"[case] evict {kind} h_kv={h_kv} d={d} bs={bs} n={n} keep={keep} sinks={sinks} recent={recent}")
    src, tables, ks, vs = make_store(300, [n], bs, h_kv, d)
    weights = weights_of(kind, h_kv, n, 301)
    out = evict(src, tables[0], weights, n, keep, sinks, recent)
    check(src, ks[0], vs[0], weights, n, keep, sinks, recent, *out)


@pytest.mark.parametrize("n", [1023, 1025, 8191, 8193, 32767, 32769, 65537, 100001])
@pytest.mark.parametrize("kind", ["heavy", "ties", "special", "close"])
def test_long_sequences(gpu, n, kind):
    say(f"[case] evict long n={n} {kind}")
    src, tables, ks, vs = make_store(302, [n], 256, 2, 64)
    weights = weights_of(kind, 2, n, 303)
    keep = n // 7 + 1
    out = evict(src, tables[0], weights, n, keep, 4, 33)
    check(src, ks[0], vs[0], weights, n, keep, 4, 33, *out)


@pytest.mark.parametrize("dst_bs", [64, 192, 1600])
def test_another_block_size(gpu, dst_bs):
    src, tables, ks, vs = make_store(304, [900], 128, 2, 64)
    weights = weights_of("heavy", 2, 900, 305)
    out = evict(src, tables[0], weights, 900, 300, 4, 10, dst_bs=dst_bs, kept_weights=False)
    check(src, ks[0], vs[0], weights, 900, 300, 4, 10, *out)


def test_within_one_store(gpu):
    """Into free blocks of the same pool."""
    src, tables, ks, vs = make_store(306, [900], 64, 2, 64, spare=6, fill=7.0)
    used = set(tables[0].tolist())
    free = torch.tensor([b for b in range(src.num_blocks) if b not in used], dtype=torch.int32)
    weights = weights_of("heavy", 2, 900, 307)
    before_k = src.k_pool.clone()
    kept = torch.empty((2, 300), dtype=torch.int32, device="cuda")
    binding.mocap_kv_evict(src, tables[0], src, free.cuda(), 900, 300, 4, 10, weights, kept)
    torch.cuda.synchronize()
    k, v = take(src, free, 300)
    for h in range(2):
        want = expected(weights[h].cpu(), 900, 300, 4, 10)
        assert kept[h].tolist() == want
        assert torch.equal(k[:, h], ks[0][want, h]) and torch.equal(v[:, h], vs[0][want, h])
    assert torch.equal(src.k_pool[tables[0].long()], before_k[tables[0].long()])


def test_nothing_to_keep(gpu):
    src = binding.KvStore(2, 64, 2, 64, fill=7.0)
    dst = binding.KvStore(2, 64, 2, 64, fill=7.0)
    table = torch.zeros(1, dtype=torch.int32, device="cuda")
    binding.mocap_kv_evict(src, table, dst, table, 0, 0, 0, 0, torch.zeros((2, 4), device="cuda"),
                           torch.zeros((2, 0), dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert (dst.k_pool == 7.0).all()


def test_graph_replays(gpu):
    n, keep = 40000, 5000
    src, tables, ks, vs = make_store(308, [n], 256, 2, 64)
    dst = binding.KvStore(20, 256, 2, 64, fill=7.0)
    table = torch.arange(19, -1, -1, dtype=torch.int32).cuda()
    weights = weights_of("heavy", 2, n, 309)
    kept = torch.empty((2, keep), dtype=torch.int32, device="cuda")
    kw = torch.empty((2, keep), device="cuda")
    ws = torch.empty(max(binding.mocap_kv_evict_workspace_size(n, 2, keep), 16), dtype=torch.uint8, device="cuda")

    def call():
        binding.mocap_kv_evict(src, tables[0], dst, table, n, keep, 4, 100, weights, kept, kw, ws)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i, kind in enumerate(("ties", "heavy", "special", "equal")):
        weights.copy_(weights_of(kind, 2, n, 310 + i))
        dst.k_pool.fill_(7.0)
        dst.v_pool.fill_(7.0)
        ws.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        check(src, ks[0], vs[0], weights, n, keep, 4, 100, dst, table, kept.cpu(), kw)
        call()
        torch.cuda.synchronize()
        check(src, ks[0], vs[0], weights, n, keep, 4, 100, dst, table, kept.cpu(), kw)


def test_refused_calls_write_nothing(gpu):
    src, tables, _, _ = make_store(311, [500], 64, 2, 64)
    dst = binding.KvStore(8, 64, 2, 64, fill=7.0)
    table = torch.arange(8, dtype=torch.int32).cuda()
    weights = weights_of("heavy", 2, 500, 312)

    def call(n=500, keep=100, sinks=4, recent=10, src_table=tables[0], dst_table=table, to=dst, w=weights, kept=None):
        kept = torch.full((2, max(keep, 0)), -1, dtype=torch.int32, device="cuda") if kept is None else kept
        binding.mocap_kv_evict(src, src_table, to, dst_table, n, keep, sinks, recent, w, kept)

    other = binding.KvStore(8, 64, 2, 128, fill=7.0)
    for bad in (dict(keep=501), dict(keep=0), dict(n=-1), dict(sinks=91), dict(sinks=-1), dict(recent=-1),
                dict(n=513), dict(dst_table=table[:1]), dict(src_table=tables[0][:7]), dict(to=other),
                dict(to=src, dst_table=tables[0])):
        with pytest.raises(binding.MocapError) as err:
            call(**bad)
        assert err.value.status == binding.MOCAP_ERR_INVALID_ARG, bad
    with pytest.raises(ValueError):
        call(kept=torch.zeros((2, 99), dtype=torch.int32, device="cuda"))
    with pytest.raises(TypeError):
        call(kept=torch.zeros((2, 100), dtype=torch.int64, device="cuda"))
    with pytest.raises(TypeError):
        call(w=weights.double())
    with pytest.raises(ValueError):
        call(w=weights[:1])
    torch.cuda.synchronize()
    assert (dst.k_pool == 7.0).all() and (dst.v_pool == 7.0).all()


def test_table_checks_refuse_a_shared_block(gpu):
    """Into the same pool: a block of the source is no block of the result."""
    src, tables, _, _ = make_store(330, [300], 64, 1, 64, spare=4)
    weights = weights_of("heavy", 1, 300, 331)
    kept = torch.full((1, 70), 7, dtype=torch.int32, device="cuda")
    free = [b for b in range(src.num_blocks) if b not in tables[0].tolist()]
    binding.set_table_checks(True)
    try:
        for other in (int(tables[0, 0]), int(tables[0, 4])):
            table = torch.tensor([free[0], other], dtype=torch.int32).cuda()
            with pytest.raises(ValueError, match="block"):
                binding.mocap_kv_evict(src, tables[0], src, table, 300, 70, 0, 0, weights, kept)
        torch.cuda.synchronize()
        assert (kept == 7).all()
        table = torch.tensor(free[:2], dtype=torch.int32).cuda()
        binding.mocap_kv_evict(src, tables[0], src, table, 300, 70, 0, 0, weights, kept)
    finally:
        binding.set_table_checks(False)
    torch.cuda.synchronize()
    assert kept[0].tolist() == expected(weights[0].cpu(), 300, 70, 0, 0)


def test_weights_written_to_meanwhile(gpu):
    """Weights that another stream writes to while positions are chosen: which ones stay is then open, but nothing
    is written outside the candidates' places of `kept` and `kept_weights`, and a later call is right."""
    n, keep, sinks, recent, h_kv = 200000, 1000, 4, 64, 2
    src, tables, ks, vs = make_store(340, [n], 256, h_kv, 64)
    dst = binding.KvStore(6, 256, h_kv, 64, fill=7.0)
    table = torch.tensor([3, 1, 4, 0], dtype=torch.int32).cuda()
    few, many = torch.zeros(h_kv, n, device="cuda"), torch.full((h_kv, n), 2.0, device="cuda")
    few[:, 5:2000] = 1.0
    weights = few.clone()
    # All that a head's candidates could be written to, had nothing stopped them.
    kept_room = torch.full((h_kv * keep + n,), -7, dtype=torch.int32, device="cuda")
    kw_room = torch.full((h_kv * keep + n,), -7.0, device="cuda")
    kept, kw = kept_room[:h_kv * keep].view(h_kv, keep), kw_room[:h_kv * keep].view(h_kv, keep)
    ws = torch.empty(binding.mocap_kv_evict_workspace_size(n, h_kv, keep), dtype=torch.uint8, device="cuda")
    chooser, writer = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(100):
        binding.mocap_kv_evict(src, tables[0], dst, table, n, keep, sinks, recent, weights, kept, kw, ws, stream=chooser)
        with torch.cuda.stream(writer):
            for _ in range(4):
                weights.copy_(many)
                weights.copy_(few)
        with torch.cuda.stream(chooser):
            # (One by one on the stream: the next call overwrites them.)
            ends = kept[:, :sinks].clone(), kept[:, keep - recent:].clone()
        chooser.synchronize()
        assert (ends[0].cpu() == torch.arange(sinks, dtype=torch.int32)).all()
        assert (ends[1].cpu() == torch.arange(n - recent, n, dtype=torch.int32)).all()
    torch.cuda.synchronize()
    assert (kept_room[h_kv * keep:] == -7).all() and (kw_room[h_kv * keep:] == -7.0).all()
    weights.copy_(few)
    binding.mocap_kv_evict(src, tables[0], dst, table, n, keep, sinks, recent, weights, kept, kw, ws)
    torch.cuda.synchronize()
    check(src, ks[0], vs[0], weights, n, keep, sinks, recent, dst, table, kept.cpu(), kw)


def test_kept_on_the_weights_is_refused(gpu):
    """Positions would be stored over weights that are still to be read."""
    src, tables, _, _ = make_store(350, [500], 64, 2, 64)
    dst = binding.KvStore(2, 64, 2, 64, fill=7.0)
    table = torch.tensor([1, 0], dtype=torch.int32).cuda()
    room = torch.rand(2 * 500 + 2 * 100, device="cuda")
    before = room.clone()
    weights, apart = room[:1000].view(2, 500), torch.zeros((2, 100), device="cuda")
    for first in (0, 801, 999):
        kept = room[first:first + 200].view(torch.int32).view(2, 100)
        with pytest.raises(ValueError, match="overlap"):
            binding.mocap_kv_evict(src, tables[0], dst, table, 500, 100, 4, 10, weights, kept, apart)
    kept = torch.full((300,), -7, dtype=torch.int32, device="cuda")
    as_floats = kept.view(torch.float32)
    for at, kw_at in ((0, 100), (100, 0), (0, 0)):
        with pytest.raises(ValueError, match="overlap"):
            binding.mocap_kv_evict(src, tables[0], dst, table, 500, 100, 4, 10, weights, kept[at:at + 200].view(2, 100),
                                   as_floats[kw_at:kw_at + 200].view(2, 100))
    torch.cuda.synchronize()
    assert torch.equal(room, before) and (kept == -7).all() and (dst.k_pool == 7.0).all()
    # Right behind the weights.
    kept = room[1000:].view(torch.int32).view(2, 100)
    binding.mocap_kv_evict(src, tables[0], dst, table, 500, 100, 4, 10, weights, kept, apart)
    torch.cuda.synchronize()
    for h in range(2):
        assert kept[h].tolist() == expected(weights[h].cpu(), 500, 100, 4, 10)


@pytest.mark.parametrize("kind", ["heavy", "ties", "special"])
@pytest.mark.parametrize("sinks,recent", [(0, 0), (4, 33)])
@pytest.mark.parametrize("candidates", [1, 1024, 4095, 4096, 4097, 16383, 16384, 16385])
def test_candidates_at_the_dispatch_borders(gpu, candidates, sinks, recent, kind):
    """Four or sixteen candidates a thread of one workgroup, or chunks."""
    say(f"[case] evict candidates={candidates} sinks={sinks} recent={recent} {kind}")
    n = candidates + sinks + recent
    src, tables, ks, vs = make_store(360, [n], 256, 2, 64)
    weights = weights_of(kind, 2, n, 361)
    keep = sinks + recent + max(1, candidates // 5)
    out = evict(src, tables[0], weights, n, keep, sinks, recent)
    check(src, ks[0], vs[0], weights, n, keep, sinks, recent, *out)


@pytest.mark.parametrize("n,sinks,recent,chosen", [
    (20000, 4, 16000, 100),   # few candidates of many positions: a workspace that is not used
    (20000, 10000, 9000, 1), (20000, 4, 18000, 0), (40000, 3, 64, 0), (40000, 20000, 3616, 0), (40000, 20000, 3616, 16384),
    (40000, 20000, 3615, 16384), (40000, 64, 0, 39936)])
@pytest.mark.parametrize("kind", ["heavy", "special", "equal"])
def test_many_positions_kept_whatever_they_weigh(gpu, n, sinks, recent, chosen, kind):
    """Many sinks and recent positions, and few, no or all candidates chosen."""
    say(f"[case] evict n={n} sinks={sinks} recent={recent} chosen={chosen} {kind}")
    src, tables, ks, vs = make_store(362, [n], 256, 1, 64)
    weights = weights_of(kind, 1, n, 363)
    keep = sinks + recent + chosen
    out = evict(src, tables[0], weights, n, keep, sinks, recent)
    check(src, ks[0], vs[0], weights, n, keep, sinks, recent, *out)
