"""The C ABI of mocap_serve.h on the host: exported symbols, refusals before
anything is enqueued (the pointers are fake), how batches, windows and rows are
cut, and the kernels' registers.  No GPU."""
import ctypes
import math
import os
import random
import re
import subprocess

import pytest

from paper_2606_22968_amd import binding, build
from test_kernel_resources import resource_report

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE, MIS, INVALID, UNSUPPORTED, WORKSPACE = 0x10000, 0x10002, 1, 2, 3
BIG = 1 << 40


def recording_build(mocap_lib, folder, *flags):
    if not os.path.exists(build.HIPCC):
        pytest.skip("hipcc not available")
    out = str(folder / "libserve_record.so")
    sources = [os.path.join(build.CSRC, "serve_api.cpp"), os.path.join(ROOT, "tests", "serve_record.cpp")]
    cmd = [build.HIPCC, *build.FLAGS, *flags, "-x", "hip", *sources, "-shared", "-Wl,-Bsymbolic", "-o", out]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    lib = ctypes.CDLL(out)
    for name in mocap_lib.SERVE_EXPORTED:
        f, real = getattr(lib, name), getattr(mocap_lib.load_library(), name)
        f.restype, f.argtypes = real.restype, real.argtypes
    return lib


@pytest.fixture(scope="module")
def host(mocap_lib, tmp_path_factory):
    return recording_build(mocap_lib, tmp_path_factory.mktemp("serve"))


def store(num_blocks=64, block_size=256, h_kv=8, head_dim=128, k=FAKE, v=FAKE):
    return binding.mocap_kv_store(k, v, num_blocks, block_size, h_kv, head_dim)


def ref(kv):
    return None if kv == "null" else ctypes.byref(store() if kv is None else kv)


def append(lib, kv=None, tables=FAKE, stride=16, lens=FAKE, batch=4, k=FAKE, v=FAKE):
    return lib.mocap_decode_append(ref(kv), tables, stride, lens, batch, k, v, None)


def decode(lib, kv=None, tables=FAKE, stride=16, lens=FAKE, batch=4, max_len=4096, q=FAKE, h_q=32, h_kv=8, d=128,
           scale=0.1, window=0, sinks=0, o=FAKE, lse=FAKE, ws=FAKE, ws_bytes=BIG):
    return lib.mocap_decode_attn(ref(kv), tables, stride, lens, batch, max_len, q, h_q, h_kv, d, scale, window, sinks, o,
                                 lse, ws, ws_bytes, None)


def window(lib, kv=None, table=FAKE, n_table=16, q=FAKE, P=1000, L=100, h_q=32, h_kv=8, d=128, scale=0.1, window=500,
           sinks=4, o=FAKE, lse=FAKE, ws=FAKE, ws_bytes=BIG, splits=0):
    return lib.mocap_window_attn(ref(kv), table, n_table, q, P, L, h_q, h_kv, d, scale, window, sinks, o, lse, ws,
                                 ws_bytes, splits, None)


def weights(lib, kv=None, table=FAKE, n_table=16, q=FAKE, P=1000, L=100, h_q=32, h_kv=8, d=128, scale=0.1, lse=FAKE,
            prev=None, w=FAKE, stride=1100, ws=FAKE, ws_bytes=BIG):
    return lib.mocap_key_weights(ref(kv), table, n_table, q, P, L, h_q, h_kv, d, scale, lse, prev, w, stride, ws,
                                 ws_bytes, None)


def decode_weights(lib, kv=None, tables=FAKE, stride=16, lens=FAKE, batch=4, max_len=4096, q=FAKE, h_q=32, h_kv=8,
                   d=128, scale=0.1, lse=FAKE, prev=None, w=FAKE, w_stride=4096):
    return lib.mocap_decode_key_weights(ref(kv), tables, stride, lens, batch, max_len, q, h_q, h_kv, d, scale, lse, prev,
                                        w, w_stride, None)


def evict(lib, src=None, src_table=FAKE, n_src=16, dst=None, dst_table=FAKE + 64, n_dst=16, n=4096, keep=1000, sinks=4,
          recent=64, w=FAKE, stride=4096, kept=FAKE, kw=None, ws=FAKE, ws_bytes=BIG):
    return lib.mocap_kv_evict(ref(src), src_table, n_src, ref(dst), dst_table, n_dst, n, keep, sinks, recent, w, stride,
                              kept, kw, ws, ws_bytes, None)


CALLS = dict(append=append, decode=decode, window=window, weights=weights, decode_weights=decode_weights, evict=evict)


def declared():
    text = open(os.path.join(ROOT, "include", "mocap_serve.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(mocap_[a-z_0-9]+)\s*\(", text)))


def test_every_declared_symbol_is_exported(mocap_lib):
    assert declared() == sorted(mocap_lib.SERVE_EXPORTED)
    for path in (build.LIB, build.DEBUG_LIB):
        assert os.path.exists(path)
        for name in declared():
            assert hasattr(ctypes.CDLL(path), name), name


@pytest.mark.parametrize("name", sorted(CALLS))
def test_good_calls_launch(host, name):
    before = host.record_launches()
    assert CALLS[name](host) == 0
    assert host.record_launches() > before


COMMON = [dict(kv="null"), dict(kv=store(k=0)), dict(kv=store(v=0)), dict(kv=store(k=MIS)), dict(kv=store(num_blocks=0))]
BATCH = COMMON + [dict(tables=0), dict(tables=MIS), dict(lens=0), dict(lens=MIS), dict(batch=-1), dict(stride=-1)]
HEADS = [dict(h_q=0), dict(h_q=30), dict(h_kv=4), dict(h_kv=0), dict(d=64), dict(scale=0.0), dict(scale=-1.0),
         dict(scale=math.nan), dict(scale=math.inf), dict(q=0), dict(q=MIS)]
CHUNK = COMMON + HEADS + [dict(table=0), dict(table=MIS), dict(P=-1), dict(L=-1), dict(n_table=4), dict(n_table=-1),
                          dict(P=(1 << 31) - 128, n_table=1 << 30), dict(lse=0), dict(lse=MIS)]
REFUSED = {
    "append": BATCH + [dict(k=0), dict(v=0), dict(k=MIS), dict(v=FAKE + 8)],
    "decode": BATCH + HEADS + [dict(max_len=-1), dict(max_len=4097), dict(max_len=1 << 31, stride=1 << 30), dict(o=0),
                               dict(o=FAKE + 8), dict(lse=0), dict(lse=MIS), dict(window=-1), dict(sinks=-1)],
    "window": CHUNK + [dict(window=0), dict(window=-5), dict(sinks=-1), dict(splits=-1), dict(o=0), dict(o=FAKE + 8)],
    "weights": CHUNK + [dict(w=0), dict(w=MIS), dict(prev=MIS), dict(stride=1099)],
    "decode_weights": BATCH + HEADS + [dict(max_len=-1), dict(max_len=4097), dict(w=0), dict(w=MIS), dict(prev=MIS),
                                       dict(lse=0), dict(w_stride=4095)],
    "evict": [dict(src="null"), dict(dst="null"), dict(src=store(k=0)), dict(dst=store(v=MIS)), dict(src_table=0),
              dict(dst_table=0), dict(n_src=15), dict(n_dst=3), dict(n=-1), dict(keep=0), dict(keep=-1), dict(keep=4097),
              dict(sinks=-1), dict(recent=-1), dict(sinks=937), dict(sinks=(1 << 31) - 1, recent=(1 << 31) - 1),
              dict(w=0), dict(w=MIS), dict(stride=4095), dict(kept=0), dict(kept=MIS), dict(kw=MIS),
              dict(dst=store(h_kv=4)), dict(dst=store(head_dim=64)), dict(dst_table=FAKE),
              dict(n=(1 << 31), n_src=1 << 30, stride=BIG)],
}


@pytest.mark.parametrize("name,kwargs", [(n, k) for n in sorted(REFUSED) for k in REFUSED[n]])
def test_malformed_calls_are_refused(host, name, kwargs):
    before = host.record_launches()
    assert CALLS[name](host, **kwargs) == INVALID
    assert host.record_launches() == before


@pytest.mark.parametrize("name", sorted(CALLS))
def test_stores_the_kernels_do_not_have(host, name):
    for kv in (store(head_dim=96), store(block_size=100), store(block_size=32)):
        for arg in (("src", "dst") if name == "evict" else ("kv",)):
            assert CALLS[name](host, **{arg: kv}) == UNSUPPORTED


def test_workspaces(host):
    for ws, size in ((0, BIG), (FAKE + 8, BIG), (FAKE, 100)):
        assert decode(host, max_len=4096, ws=ws, ws_bytes=size) == WORKSPACE
        assert window(host, splits=3, ws=ws, ws_bytes=size) == WORKSPACE
    assert window(host, splits=1, ws=0, ws_bytes=0) == 0
    assert decode(host, max_len=64, ws=0, ws_bytes=0) == 0
    size = ctypes.c_size_t(0)
    assert host.mocap_decode_attn_workspace_size(4, 4096, 32, 8, 128, 0, 0, ctypes.byref(size)) == 0
    assert decode(host, ws_bytes=size.value) == 0 and decode(host, ws_bytes=size.value - 1) == WORKSPACE
    n = ctypes.c_int32(0)
    assert host.mocap_window_attn_workspace_size(1000, 100, 32, 8, 128, 500, 4, 3, ctypes.byref(n), ctypes.byref(size)) == 0
    assert n.value == 3
    assert window(host, splits=3, ws_bytes=size.value) == 0 and window(host, splits=3, ws_bytes=size.value - 1) == WORKSPACE


@pytest.mark.parametrize("args", [(-1, 100, 32, 8, 128, 0, 0), (1, -1, 32, 8, 128, 0, 0), (1, 100, 30, 8, 128, 0, 0),
                                  (1, 100, 32, 8, 128, -1, 0), (1, 100, 32, 8, 128, 0, -1), (1, 1 << 31, 32, 8, 128, 0, 0)])
def test_decode_workspace_size_refuses(host, args):
    size = ctypes.c_size_t(0)
    assert host.mocap_decode_attn_workspace_size(*args, ctypes.byref(size)) == INVALID
    assert host.mocap_decode_attn_workspace_size(1, 100, 32, 8, 128, 0, 0, None) == INVALID
    assert host.mocap_decode_attn_workspace_size(1, 100, 32, 8, 96, 0, 0, ctypes.byref(size)) == UNSUPPORTED


def test_other_sizes_refuse(host):
    size = ctypes.c_size_t(0)
    out = ctypes.byref(size)
    assert host.mocap_window_attn_workspace_size(-1, 1, 8, 8, 64, 1, 0, 0, None, out) == INVALID
    assert host.mocap_window_attn_workspace_size(0, 1, 8, 8, 64, 0, 0, 0, None, out) == INVALID
    assert host.mocap_window_attn_workspace_size(0, 1, 8, 8, 64, 1, -1, 0, None, out) == INVALID
    assert host.mocap_window_attn_workspace_size(0, 1, 8, 8, 64, 1, 0, -1, None, out) == INVALID
    assert host.mocap_window_attn_workspace_size(0, 1, 8, 8, 64, 1, 0, 0, None, None) == INVALID
    assert host.mocap_window_attn_workspace_size(0, 1, 8, 8, 65, 1, 0, 0, None, out) == UNSUPPORTED
    assert host.mocap_key_weights_workspace_size(0, -1, 8, 8, 64, out) == INVALID
    assert host.mocap_key_weights_workspace_size(0, 1, 8, 8, 64, None) == INVALID
    assert host.mocap_kv_evict_workspace_size(10, 8, 11, out) == INVALID
    assert host.mocap_kv_evict_workspace_size(10, 8, 0, out) == INVALID
    assert host.mocap_kv_evict_workspace_size(10, 0, 1, out) == INVALID
    assert host.mocap_kv_evict_workspace_size(10, 8, 1, None) == INVALID
    assert host.mocap_kv_evict_workspace_size(0, 8, 0, out) == 0
    assert host.mocap_kv_evict_workspace_size(10, 70000, 1, out) == UNSUPPORTED


def test_sizes_too_large_for_a_grid(host):
    huge = (1 << 31) - 1
    assert append(host, batch=huge) == UNSUPPORTED
    assert decode(host, batch=huge) == UNSUPPORTED
    assert decode_weights(host, batch=huge) == UNSUPPORTED
    kv = store(block_size=64 << 20)
    assert window(host, kv=kv, P=0, L=(1 << 31) - 200, n_table=64, ws_bytes=BIG) == UNSUPPORTED
    assert weights(host, kv=kv, P=0, L=(1 << 31) - 200, n_table=64, stride=BIG) == UNSUPPORTED


def test_empty_calls_launch_nothing(host):
    before = host.record_launches()
    assert append(host, batch=0, tables=0, lens=0, k=0, v=0) == 0
    assert decode(host, batch=0, tables=0, lens=0, q=0, o=0, lse=0) == 0
    assert window(host, L=0, q=0, o=0, lse=0) == 0
    assert weights(host, L=0, q=0, lse=0, w=0) == 0
    assert decode_weights(host, batch=0, q=0, lse=0, w=0) == 0
    assert evict(host, n=0, keep=0, sinks=0, recent=0, w=0, kept=0) == 0
    assert host.record_launches() == before


def tiles_of(n, window, sinks):
    """Tiles with a visible key, counted one key at a time."""
    low = max(0, n - window) if window else 0
    return len({j // 64 for j in range(n) if j >= low or j < sinks})


def test_items_hold_any_lengths(host):
    """The grid's items are enough whatever the lengths turn out to be, and a
    split that the plan rules out never happens."""
    rng = random.Random(5)
    for _ in range(400):
        batch = rng.choice((1, 2, 3, 17, 64, 65, 200, 600))
        h_kv = rng.choice((1, 2, 8))
        group = rng.choice((1, 4, 16, 20, 64))
        max_len = rng.choice((0, 1, 64, 512, 513, 3000, 20000))
        win, sinks = rng.choice(((0, 0), (1, 0), (100, 4), (1000, 70), (5000, 500)))
        kv = store(h_kv=h_kv)
        assert decode(host, kv=kv, stride=100, batch=batch, max_len=max_len, h_q=h_kv * group, h_kv=h_kv, window=win,
                      sinks=sinks) == 0
        out = (ctypes.c_int * 8)()
        host.record_batch(out)
        target, fill, min_tiles, least, items, w, s, _ = out
        assert (w, s) == ((0, 0) if win == 0 or win >= max_len else (win, min(sinks, max_len)))
        size = ctypes.c_size_t(0)
        assert host.mocap_decode_attn_workspace_size(batch, max_len, h_kv * group, h_kv, 128, win, sinks,
                                                     ctypes.byref(size)) == 0
        for lens in ([max_len] * batch, [0] * batch, [1] * (batch - 1) + [max_len],
                     [rng.randint(0, max_len) for _ in range(batch)]):
            counts = [tiles_of(n, w, s) for n in lens]
            total = sum(counts)
            per = max(min(min_tiles, max(least, total // fill + 1)), total // target + 1)
            parts = [max(1, -(-c // per)) for c in counts]
            assert sum(parts) <= items
            assert size.value > 0 or max(parts) == 1
            assert size.value == 0 or size.value >= items * h_kv * group * (128 + 1) * 4


def test_window_ranges(host):
    rng = random.Random(6)
    for _ in range(300):
        P, L = rng.choice((0, 1, 700, 100000)), rng.choice((1, 2, 63, 500, 4096))
        h_q, h_kv = rng.choice(((8, 8), (8, 2), (64, 1), (6, 3)))
        win, sinks = rng.choice((1, 64, 1000, 4096, 1 << 50)), rng.choice((0, 4, 100, 1 << 50))
        splits = rng.choice((0, 0, 1, 2, 7, 1 << 30))
        kv = store(h_kv=h_kv, block_size=1024)
        n, size = ctypes.c_int32(0), ctypes.c_size_t(0)
        assert host.mocap_window_attn_workspace_size(P, L, h_q, h_kv, 128, win, sinks, splits, ctypes.byref(n),
                                                     ctypes.byref(size)) == 0
        assert window(host, kv=kv, n_table=200, P=P, L=L, h_q=h_q, h_kv=h_kv, window=win, sinks=sinks, splits=splits,
                      ws_bytes=size.value) == 0
        out = (ctypes.c_int * 5)()
        host.record_window(out)
        row_blocks, n_ranges, total, w, s = out
        assert n_ranges == n.value and total == row_blocks * h_kv * n_ranges
        assert row_blocks == -(-L * (h_q // h_kv) // 256)
        assert 0 < w < 1 << 31 and 0 <= s < 1 << 31
        assert splits != 1 or n_ranges == 1
        assert size.value >= (0 if n_ranges == 1 else n_ranges * L * h_q * 129 * 4)


def test_key_weight_blocks(host):
    for P, L, h_kv in ((0, 1, 8), (0, 2048, 8), (30720, 2048, 8), (1 << 20, 1, 1), (100, 3, 1), (5000, 64, 2), (5000, 32, 2), (5000, 33, 2)):
        kv = store(h_kv=h_kv, block_size=1 << 16)
        assert weights(host, kv=kv, P=P, L=L, h_q=4 * h_kv, h_kv=h_kv, stride=1 << 22, n_table=1 << 10) == 0
        out = (ctypes.c_int * 3)()
        host.record_weights(out)
        few, key_blocks, parts = out
        assert few == (4 * L <= 128)
        if few:
            assert parts == 1 and 1 <= key_blocks <= -(-(P + L) // 64)
            continue
        assert key_blocks * 512 >= P + L > (key_blocks - 1) * 512
        size = ctypes.c_size_t(0)
        assert host.mocap_key_weights_workspace_size(P, L, 4 * h_kv, h_kv, 128, ctypes.byref(size)) == 0
        assert size.value == (0 if parts == 1 else parts * h_kv * (P + L) * 4)
        assert parts == 1 or parts * 4 <= -(-L * 4 // 32) + 3


def test_key_weight_parts(host):
    """The workgroups of a KV head are the parts of all key blocks, counted from
    the tiles of 32 rows that see a block's first key or a later one."""
    rng = random.Random(7)
    cut = 0
    for _ in range(400):
        P, L = rng.choice((0, 0, 1, 100, 511, 512, 1500, 40000)), rng.choice((33, 500, 513, 2048, 4096, 10000))
        h_kv, group = rng.choice((1, 2, 8)), rng.choice((1, 3, 4, 64))
        rows = L * group
        if rows <= 128:
            continue
        kv = store(h_kv=h_kv, block_size=1 << 16)
        assert weights(host, kv=kv, P=P, L=L, h_q=group * h_kv, h_kv=h_kv, stride=1 << 20, n_table=64) == 0
        out = (ctypes.c_int * 3)()
        host.record_weights_cut(out)
        row_parts, part_tiles, head_wgs = out
        tiles = -(-rows // 32)
        parts = []
        for block in range(-(-(P + L) // 512)):
            first = max(0, block * 512 - P) * group // 32
            assert first < tiles
            parts.append(-(-(tiles - first) // part_tiles))
        assert row_parts == max(parts) and head_wgs == sum(parts)
        seen = min(len(parts), P // 512 + 1)
        assert set(parts[:seen]) == {row_parts}
        cut += len(set(parts)) > 1
    assert cut > 20


@pytest.mark.parametrize("src", ["decode_attn.hip", "window_attn.hip", "key_weights.hip", "kv_evict.hip"])
def test_kernels_keep_their_values_in_registers(src, tmp_path):
    for name, r in resource_report(src, str(tmp_path)).items():
        assert r.get("VGPRs Spill", 0) == 0 and r.get("ScratchSize [bytes/lane]", 0) == 0, f"{name}: {r}"


def test_blocks_and_heads_beyond_32_bits(host):
    """What a kernel addresses with 32-bit offsets is refused beyond them."""
    def kv(**kwargs):
        return store(num_blocks=2, **kwargs)
    for d in (64, 128):
        for block_size, status in (((1 << 30) // d - 64, 0), ((1 << 30) // d, UNSUPPORTED)):
            big = kv(block_size=block_size, h_kv=1, head_dim=d)
            assert window(host, kv=big, h_q=4, h_kv=1, d=d) == status
            assert decode(host, kv=big, h_q=4, h_kv=1, d=d) == status
            assert weights(host, kv=big, h_q=4, h_kv=1, d=d) == 0
            assert decode_weights(host, kv=big, h_q=4, h_kv=1, d=d) == 0
    for d, heads in ((64, 65535 * 8), (128, 65535 * 4)):
        assert append(host, kv=kv(h_kv=heads, head_dim=d)) == 0
        assert append(host, kv=kv(h_kv=heads + 1, head_dim=d)) == UNSUPPORTED
    for group in (1, 3, 4, 64, 200):
        h_kv = ((1 << 31) - 1) // ((128 // group + 2) * group * 256)
        most = dict(kv=kv(h_kv=min(h_kv, 65535)), h_q=min(h_kv, 65535) * group, h_kv=min(h_kv, 65535))
        assert weights(host, L=200, stride=1200, **most) == 0
        more = dict(kv=kv(h_kv=h_kv + 1), h_q=(h_kv + 1) * group, h_kv=h_kv + 1)
        assert weights(host, L=200, stride=1200, **more) == UNSUPPORTED
    size = ctypes.c_size_t(0)
    most = (1 << 30) - 64
    assert host.mocap_kv_evict_workspace_size(most, 1, most, ctypes.byref(size)) == 0
    assert host.mocap_kv_evict_workspace_size(most + 1, 1, 1, ctypes.byref(size)) == UNSUPPORTED


def test_weights_that_overlap(host):
    """prev is weights or apart from it; kept_weights is apart from weights."""
    n = 4 * (7 * 1200 + 1100)  # bytes of 8 rows of 1100, 1200 apart
    for prev, status in ((FAKE, 0), (FAKE + 4, INVALID), (FAKE + n - 4, INVALID), (FAKE + n, 0), (FAKE - n, 0),
                         (FAKE - n + 4, INVALID)):
        assert weights(host, stride=1200, prev=prev) == status
    n = 4 * (31 * 5000 + 4096)
    for prev, status in ((FAKE + n, 0), (FAKE + n - 4, INVALID), (FAKE, 0)):
        assert decode_weights(host, prev=prev, w_stride=5000) == status
    n = 4 * (7 * 5000 + 4096)
    for kw, status in ((FAKE, INVALID), (FAKE + n, 0), (FAKE + n - 4, INVALID), (FAKE - 4 * 8 * 1000, 0),
                       (FAKE - 4 * 8 * 1000 + 4, INVALID)):
        assert evict(host, stride=5000, kw=kw) == status


def test_debug_build_checks_the_tables(mocap_lib, tmp_path):
    """The entries that a call uses, and those alone."""
    lib = recording_build(mocap_lib, tmp_path, "-DMOCAP_DEBUG_TABLES")
    kept = []

    def ints(*values):
        kept.append((ctypes.c_int32 * len(values))(*values))
        return ctypes.addressof(kept[-1])
    kv = store(num_blocks=4)
    args = dict(kv=kv, stride=3, batch=2)
    for table, lens, status in (((0, 1, 2, 3, 1, 0), (700, 700), 0), ((0, 1, 4, 3, 1, 0), (513, 1), INVALID),
                                ((0, 1, 4, 3, 1, 0), (512, 1), 0), ((0, 1, 4, -1, 1, 0), (512, 0), 0),
                                ((0, 1, 4, -1, 1, 0), (512, 1), INVALID), ((0, 0, 0, 0, 0, 0), (768, 768), 0)):
        where = dict(tables=ints(*table), lens=ints(*lens))
        assert decode(lib, max_len=768, **where, **args) == status
        assert decode_weights(lib, max_len=768, **where, **args) == status
    bad = dict(tables=ints(0, 9, 2, 0, 1, 2), lens=ints(700, 700))
    assert decode(lib, max_len=768, window=100, sinks=4, **bad, **args) == 0
    assert decode(lib, max_len=768, window=200, sinks=4, **bad, **args) == INVALID
    assert decode(lib, max_len=768, window=100, sinks=257, **bad, **args) == INVALID
    assert append(lib, **bad, **args) == 0  # position 699 is in the third block
    assert append(lib, tables=bad["tables"], lens=ints(300, 0), **args) == INVALID
    for table, status in (((0, 1, 2), 0), ((0, 9, 2), INVALID), ((0, 1, 1), INVALID)):
        assert window(lib, kv=kv, table=ints(*table), n_table=3, P=500, L=200) == status
        assert weights(lib, kv=kv, table=ints(*table), n_table=3, P=500, L=200) == status
        assert evict(lib, src=kv, src_table=ints(*table), n_src=3, n=700, keep=300, dst_table=ints(0, 1)) == status
    assert window(lib, kv=kv, table=ints(0, 9, 2), n_table=3, P=650, L=50, window=100) == 0
    assert evict(lib, src=kv, src_table=ints(0, 1, 2), n_src=3, n=700, keep=300, dst=kv, dst_table=ints(0, 4)) == INVALID


def test_debug_build_skips_appends_beyond_the_tables(mocap_lib, tmp_path):
    """Nothing is written for a sequence that the tables do not hold, so no entry of its is looked at."""
    lib = recording_build(mocap_lib, tmp_path, "-DMOCAP_DEBUG_TABLES")
    table, args = (ctypes.c_int32 * 6)(0, 1, -1, 0, 1, 2), dict(kv=store(num_blocks=4), stride=3, batch=2)
    for lens, status in (((769, 700), 0), ((1 << 30, 1), 0), ((768, 700), INVALID), ((512, 769), 0)):
        lens = (ctypes.c_int32 * 2)(*lens)
        assert append(lib, tables=ctypes.addressof(table), lens=ctypes.addressof(lens), **args) == status


def window_tiles(P, L, group, win, sinks):
    """Tiles that some row of a workgroup of 256 rows sees, for the workgroup with the most."""
    most = 0
    for row in range(0, L * group, 256):
        first, last = P + row // group, P + min(row + 255, L * group - 1) // group
        low = max(0, first - win + 1)
        most = max(most, len({j // 64 for j in range(last + 1) if j >= low or j < sinks}))
    return most


def test_window_range_requests(host):
    """A request is met up to the number of tiles, and exceeds it by two at most."""
    rng = random.Random(8)
    for _ in range(300):
        P, L = rng.choice((0, 1, 63, 64, 700, 2001)), rng.choice((1, 2, 31, 100, 300))
        group, win = rng.choice((1, 3, 4, 64)), rng.choice((1, 2, 64, 65, 100, 1100, 5000))
        sinks = rng.choice((0, 1, 64, 70, 300, 9999))
        tiles = window_tiles(P, L, group, win, sinks)
        for splits in (1, 2, 3, tiles - 1, tiles, tiles + 1, tiles + 2, tiles + 3, 1 << 30):
            if splits < 1:
                continue
            n, size = ctypes.c_int32(0), ctypes.c_size_t(0)
            assert host.mocap_window_attn_workspace_size(P, L, 2 * group, 2, 128, win, sinks, splits, ctypes.byref(n),
                                                         ctypes.byref(size)) == 0
            assert min(splits, tiles) <= n.value <= min(splits, tiles + 2)
