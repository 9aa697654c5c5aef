"""The C ABI of mocap_cache.h on the host: exported symbols, refusals before anything
is enqueued (the pointers are fake), what is handed to the kernels, and their registers.
No GPU."""
import ctypes
import math
import os
import re
import subprocess

import pytest

from paper_2606_22968_amd import binding, build
from test_kernel_resources import resource_report

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE, MIS, INVALID, UNSUPPORTED, WORKSPACE = 0x10000, 0x10002, 1, 2, 3
FAR = 1 << 36                                    # another fake address, beyond every array at FAKE
BIG = 1 << 40


def recording_build(mocap_lib, folder, *flags):
    if not os.path.exists(build.HIPCC):
        pytest.skip("hipcc not available")
    out = str(folder / "libcache_record.so")
    sources = [os.path.join(build.CSRC, "cache_api.cpp"), os.path.join(ROOT, "tests", "cache_record.cpp")]
    cmd = [build.HIPCC, *build.FLAGS, *flags, "-x", "hip", *sources, "-shared", "-Wl,-Bsymbolic", "-o", out]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    lib = ctypes.CDLL(out)
    for name in mocap_lib.CACHE_EXPORTED:
        f, real = getattr(lib, name), getattr(mocap_lib.load_library(), name)
        f.restype, f.argtypes = real.restype, real.argtypes
    return lib


@pytest.fixture(scope="module")
def host(mocap_lib, tmp_path_factory):
    return recording_build(mocap_lib, tmp_path_factory.mktemp("cache"))


def store(num_blocks=64, block_size=256, h_kv=8, head_dim=128, k=FAKE, v=FAKE):
    return binding.mocap_kv_store(k, v, num_blocks, block_size, h_kv, head_dim)


def store4(num_blocks=64, block_size=256, h_kv=8, head_dim=128, k=FAKE, v=FAKE, ks=FAKE, vs=FAKE):
    return binding.mocap_kv4_store(k, v, ks, vs, num_blocks, block_size, h_kv, head_dim)


def ref(kv, four):
    return None if kv == "null" else ctypes.byref((store4 if four else store)() if kv is None else kv)


def rope_ref(rope):
    return None if rope is None else ctypes.byref(binding.mocap_rope(*rope))


def append(lib, four, kv=None, table=FAKE, n_table=16, start=1000, n=100, rope=(FAKE, 128, 0), first=1000, q=FAKE,
           q_stride=6144, h_q=32, k=FAKE, k_stride=6144, v=FAKE, v_stride=6144, q_out=FAR):
    call = lib.mocap_kv4_append if four else lib.mocap_rope_append
    return call(ref(kv, four), table, n_table, start, n, rope_ref(rope), first, q, q_stride, h_q, k, k_stride, v, v_stride,
                q_out, None)


def batch_append(lib, four, kv=None, tables=FAKE, stride=16, lens=FAKE, batch=4, rope=(FAKE, 128, 0), positions=None,
                 q=FAKE, q_stride=6144, h_q=32, k=FAKE, k_stride=6144, v=FAKE, v_stride=6144, q_out=FAR):
    call = lib.mocap_kv4_decode_append if four else lib.mocap_decode_rope_append
    return call(ref(kv, four), tables, stride, lens, batch, rope_ref(rope), positions, q, q_stride, h_q, k, k_stride, v,
                v_stride, q_out, None)


def load(lib, kv=None, tables=FAKE, stride=16, lens=FAKE, batch=4, n=10, k=FAKE, v=FAKE):
    return lib.mocap_kv4_load(ref(kv, True), tables, stride, lens, batch, n, k, v, None)


def decode(lib, kv=None, tables=FAKE, stride=16, lens=FAKE, batch=4, max_len=4096, q=FAKE, h_q=32, h_kv=8, d=128,
           scale=0.1, window=0, sinks=0, o=FAKE, lse=FAKE, ws=FAKE, ws_bytes=BIG):
    return lib.mocap_kv4_decode_attn(ref(kv, True), tables, stride, lens, batch, max_len, q, h_q, h_kv, d, scale, window,
                                     sinks, o, lse, ws, ws_bytes, None)


def chunk(lib, kv=None, table=FAKE, n_table=16, q=FAKE, P=1000, L=100, h_q=32, h_kv=8, d=128, scale=0.1, window=0,
          sinks=0, o=FAKE, lse=FAKE, ws=FAKE, ws_bytes=BIG, splits=0):
    return lib.mocap_kv4_chunk_attn(ref(kv, True), table, n_table, q, P, L, h_q, h_kv, d, scale, window, sinks, o, lse, ws,
                                    ws_bytes, splits, None)


CALLS = dict(rope=lambda lib, **k: append(lib, False, **k), kv4=lambda lib, **k: append(lib, True, **k),
             rope_batch=lambda lib, **k: batch_append(lib, False, **k),
             kv4_batch=lambda lib, **k: batch_append(lib, True, **k), load=load, decode=decode, chunk=chunk)
FOUR = ("kv4", "kv4_batch", "load", "decode", "chunk")


def declared():
    text = open(os.path.join(ROOT, "include", "mocap_cache.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(mocap_[a-z_0-9]+)\s*\(", text)))


def test_every_declared_symbol_is_exported(mocap_lib):
    assert declared() == sorted(mocap_lib.CACHE_EXPORTED)
    for path in (build.LIB, build.DEBUG_LIB):
        assert os.path.exists(path)
        for name in declared():
            assert hasattr(ctypes.CDLL(path), name), name


@pytest.mark.parametrize("name", sorted(CALLS))
def test_good_calls_launch(host, name):
    before = host.record_launches()
    assert CALLS[name](host) == 0
    assert host.record_launches() > before


POOLS = ["null", dict(k=0), dict(v=0), dict(k=MIS), dict(v=FAKE + 8), dict(num_blocks=0), dict(block_size=0)]
POOLS4 = POOLS + [dict(ks=0), dict(vs=0), dict(ks=MIS), dict(vs=FAKE + 8)]
BATCH = [dict(tables=0), dict(tables=MIS), dict(lens=0), dict(lens=MIS), dict(batch=-1), dict(stride=-1)]
TABLE = [dict(table=0), dict(table=MIS), dict(n_table=4), dict(n_table=-1)]
ROWS = [dict(rope=(0, 128, 0)), dict(rope=(MIS, 128, 0)), dict(rope=(FAKE, 0, 0)), dict(rope=(FAKE, -16, 0)),
        dict(rope=(FAKE, 144, 0)), dict(q=0), dict(q=MIS), dict(q_out=0), dict(q_out=FAR + 8), dict(h_q=-8), dict(h_q=30),
        dict(q_stride=4088), dict(q_stride=6148), dict(k=0), dict(k=FAKE + 8), dict(k_stride=1016), dict(k_stride=6145),
        dict(v=0), dict(v=MIS), dict(v_stride=-6144), dict(v_stride=6146),
        dict(q_out=FAKE), dict(q_out=FAKE, q=FAR), dict(q_out=FAKE, q=FAR, k=2 * FAR), dict(q_out=FAR + 16, q=FAR)]
HEADS = [dict(h_q=0), dict(h_q=30), dict(h_kv=4), dict(h_kv=0), dict(d=64), dict(scale=0.0), dict(scale=-1.0),
         dict(scale=math.nan), dict(scale=math.inf), dict(q=0), dict(q=MIS), dict(o=0), dict(o=FAKE + 8), dict(lse=0),
         dict(lse=MIS), dict(window=-1), dict(sinks=-1)]
APPEND = TABLE + ROWS + [dict(start=-1), dict(n=-1), dict(first=-1), dict(first=(1 << 31) - 127), dict(first=1 << 62),
                         dict(start=(1 << 31) - 128, n_table=1 << 30)]
REFUSED = dict(
    rope=APPEND, kv4=APPEND, rope_batch=BATCH + ROWS + [dict(positions=MIS)], kv4_batch=BATCH + ROWS + [dict(positions=MIS)],
    load=BATCH + [dict(n=-1), dict(n=(1 << 31) - 1), dict(k=0), dict(v=0), dict(k=MIS), dict(v=FAKE + 8)],
    decode=BATCH + HEADS + [dict(max_len=-1), dict(max_len=4097), dict(max_len=1 << 31, stride=1 << 30)],
    chunk=TABLE + HEADS + [dict(P=-1), dict(L=-1), dict(P=(1 << 31) - 128, n_table=1 << 30), dict(splits=-1)])


@pytest.mark.parametrize("name,kwargs", [(n, k) for n in sorted(REFUSED) for k in REFUSED[n]] +
                         [(n, dict(pools=k)) for n in sorted(REFUSED) for k in (POOLS4 if n in FOUR else POOLS)])
def test_malformed_calls_are_refused(host, name, kwargs):
    pools = kwargs.get("pools")
    if pools is not None:
        kwargs = dict(kv=pools if pools == "null" else (store4 if name in FOUR else store)(**pools))
    before = host.record_launches()
    assert CALLS[name](host, **kwargs) == INVALID
    assert host.record_launches() == before


@pytest.mark.parametrize("name", sorted(CALLS))
def test_stores_the_kernels_do_not_have(host, name):
    make = store4 if name in FOUR else store
    for kv in (make(head_dim=96), make(block_size=100), make(block_size=32)):
        assert CALLS[name](host, kv=kv) == UNSUPPORTED


@pytest.mark.parametrize("name", ["rope", "kv4", "rope_batch", "kv4_batch"])
def test_rows_and_rotations(host, name):
    call = CALLS[name]
    for rot in (8, 24, 100):
        assert call(host, rope=(FAKE, rot, 0)) == UNSUPPORTED
    out = (ctypes.c_longlong * 11)()
    for rope in (None, (FAKE, 16, 1), (FAKE, 128, 0), (FAKE + 4, 64, 7)):
        assert call(host, rope=rope) == 0
        host.record_append(out)
        assert out[0] == (0 if rope is None else rope[1]) and out[1] == int(rope is not None and rope[2] != 0)
        assert out[10] == int(name in FOUR)
    # In place, without queries, with the least strides.
    dense = dict(q=FAR, q_out=FAR, q_stride=4096, k_stride=1024, v_stride=1024)
    assert call(host, **dense) == 0
    host.record_append(out)
    assert list(out)[2:7] == [32, 8, 4096, 1024, 1024]
    assert call(host, q=0, q_out=0, h_q=0, q_stride=0) == 0
    # The last row of Q ends where q_out begins; and one value later.
    rows = 100 if name in ("rope", "kv4") else 4
    end = FAKE + 2 * ((rows - 1) * 6144 + 4096)
    assert call(host, q_out=end, k=FAR, v=FAR) == 0
    assert call(host, q_out=end - 16, k=FAR, v=FAR) == INVALID


def test_positions_apart_from_slots(host):
    out = (ctypes.c_longlong * 11)()
    assert append(host, True, start=70, first=(1 << 31) - 228) == 0
    host.record_append(out)
    assert list(out)[7:10] == [70, (1 << 31) - 228, 100]


def test_workspaces(host):
    for ws, size in ((0, BIG), (FAKE + 8, BIG), (FAKE, 100)):
        assert decode(host, max_len=4096, ws=ws, ws_bytes=size) == WORKSPACE
        assert chunk(host, splits=3, ws=ws, ws_bytes=size) == WORKSPACE
    assert chunk(host, splits=1, ws=0, ws_bytes=0) == 0
    assert decode(host, max_len=64, ws=0, ws_bytes=0) == 0
    size, n = ctypes.c_size_t(0), ctypes.c_int32(0)
    assert host.mocap_kv4_decode_attn_workspace_size(4, 4096, 32, 8, 128, 0, 0, ctypes.byref(size)) == 0
    assert decode(host, ws_bytes=size.value) == 0 and decode(host, ws_bytes=size.value - 1) == WORKSPACE
    for window in (0, 500):
        assert host.mocap_kv4_chunk_attn_workspace_size(1000, 100, 32, 8, 128, window, 4, 3, ctypes.byref(n),
                                                        ctypes.byref(size)) == 0
        assert n.value == 3
        args = dict(splits=3, window=window, sinks=4)
        assert chunk(host, ws_bytes=size.value, **args) == 0 and chunk(host, ws_bytes=size.value - 1, **args) == WORKSPACE


def test_sizes_refuse(host):
    size = ctypes.c_size_t(0)
    out = ctypes.byref(size)
    for args in ((-1, 100, 32, 8, 128, 0, 0), (1, -1, 32, 8, 128, 0, 0), (1, 100, 30, 8, 128, 0, 0),
                 (1, 100, 32, 8, 128, -1, 0), (1, 100, 32, 8, 128, 0, -1), (1, 1 << 31, 32, 8, 128, 0, 0)):
        assert host.mocap_kv4_decode_attn_workspace_size(*args, out) == INVALID
    assert host.mocap_kv4_decode_attn_workspace_size(1, 100, 32, 8, 128, 0, 0, None) == INVALID
    assert host.mocap_kv4_decode_attn_workspace_size(1, 100, 32, 8, 96, 0, 0, out) == UNSUPPORTED
    for args in ((-1, 1, 8, 8, 64, 0, 0, 0), (0, -1, 8, 8, 64, 0, 0, 0), (0, 1, 8, 3, 64, 0, 0, 0),
                 (0, 1, 8, 8, 64, -1, 0, 0), (0, 1, 8, 8, 64, 0, -1, 0), (0, 1, 8, 8, 64, 0, 0, -1)):
        assert host.mocap_kv4_chunk_attn_workspace_size(*args, None, out) == INVALID
    assert host.mocap_kv4_chunk_attn_workspace_size(0, 1, 8, 8, 64, 0, 0, 0, None, None) == INVALID
    assert host.mocap_kv4_chunk_attn_workspace_size(0, 1, 8, 8, 65, 0, 0, 0, None, out) == UNSUPPORTED


def test_sizes_too_large_for_a_grid(host):
    huge = (1 << 31) - 1
    for name in ("rope_batch", "kv4_batch", "load", "decode"):
        assert CALLS[name](host, batch=huge, **({} if name in ("load", "decode") else dict(q_out=1 << 60))) == UNSUPPORTED
    make = dict(rope=store, kv4=store4)
    for name in make:
        kv = make[name](block_size=64 << 20)
        assert CALLS[name](host, kv=kv, start=0, first=0, n=(1 << 31) - 200, n_table=64, q_out=1 << 60) == UNSUPPORTED
        wide = dict(kv=make[name](h_kv=70000), h_q=0, k_stride=1 << 24, v_stride=1 << 24)
        assert CALLS[name](host, **wide) == UNSUPPORTED
    assert load(host, kv=store4(h_kv=70000)) == UNSUPPORTED
    assert chunk(host, kv=store4(block_size=64 << 20), P=0, L=(1 << 31) - 200, n_table=64) == UNSUPPORTED


def test_empty_calls_launch_nothing(host):
    before = host.record_launches()
    for name in ("rope", "kv4"):
        assert CALLS[name](host, n=0, q=0, k=0, v=0, q_out=0) == 0
    for name in ("rope_batch", "kv4_batch"):
        assert CALLS[name](host, batch=0, tables=0, lens=0, q=0, k=0, v=0, q_out=0) == 0
    assert load(host, batch=0, tables=0, lens=0, k=0, v=0) == 0 and load(host, n=0, k=0, v=0) == 0
    assert decode(host, batch=0, tables=0, lens=0, q=0, o=0, lse=0) == 0
    assert chunk(host, L=0, q=0, o=0, lse=0) == 0
    assert host.record_launches() == before


def plan_of(host, **kwargs):
    out = (ctypes.c_int * 7)()
    assert chunk(host, **kwargs) == 0
    host.record_chunk(out)
    return dict(zip(("row_blocks", "n_ranges", "total_wgs", "window", "sinks", "mirrored", "few"), out))


def test_chunk_plans(host):
    """Windows that hide nothing are none; rows are mirrored where one workgroup per compute unit holds them; few rows,
    or many with few keys, go in blocks of 16, or 32 where those would take turns."""
    kv = store4(block_size=1024)
    for P, L, window, splits, mirrored, few in (
            (0, 2048, 0, 1, True, False), (30720, 2048, 0, 1, True, False), (0, 2049, 0, 1, False, False),
            (0, 8192, 0, 1, False, False), (0, 2048, 2047, 1, False, False), (0, 2048, 2048, 1, True, False),
            (20000, 500, 0, 4, True, False), (20000, 500, 0, 5, False, False), (20000, 500, 5000, 3, False, False),
            (100, 10, 0, 1, None, 16), (20000, 1, 0, 0, None, 16), (20000, 4, 0, 0, None, 16), (20000, 5, 5000, 0, None, 16),
            (20000, 16, 0, 40, None, 32), (0, 300, 0, 0, None, 16), (0, 600, 0, 0, None, 32)):
        p = plan_of(host, kv=kv, n_table=64, P=P, L=L, window=window, sinks=4, splits=splits)
        assert bool(p["few"]) == bool(few) and p["row_blocks"] == -(-L * 4 // (few or 256)), p
        assert p["total_wgs"] == p["row_blocks"] * 8 * p["n_ranges"]
        assert splits == 0 or p["n_ranges"] == splits
        assert few or bool(p["mirrored"]) == mirrored
        if window == 0:
            assert p["window"] >= P + L and p["sinks"] == 0
        else:
            assert (p["window"], p["sinks"]) == (window, 4)


def test_chunk_workspaces_hold_what_is_planned(host):
    """A call takes the workspace that the size function names, and no less, for either way and any count of ranges."""
    size, n = ctypes.c_size_t(), ctypes.c_int32()
    for h_q, h_kv, d in ((32, 8, 128), (16, 2, 64), (64, 1, 64), (128, 16, 128)):
        kv = store4(block_size=1024, h_kv=h_kv, head_dim=d)
        for P in (0, 700, 5000, 40000):
            for L in (1, 3, 17, 130, 700):
                for window, splits in ((0, 0), (300, 0), (0, 2), (0, 7), (1000, 100)):
                    assert host.mocap_kv4_chunk_attn_workspace_size(P, L, h_q, h_kv, d, window, 1, splits, ctypes.byref(n),
                                                                    ctypes.byref(size)) == 0
                    args = dict(kv=kv, n_table=64, P=P, L=L, h_q=h_q, h_kv=h_kv, d=d, window=window, sinks=1, splits=splits)
                    p = plan_of(host, ws_bytes=size.value, **args)
                    assert p["n_ranges"] == n.value <= max(1, -(-(P + L) // 64))
                    assert (size.value == 0) == (n.value == 1)
                    assert size.value >= (0 if n.value == 1 else n.value * L * h_q * (d + 1) * 4)
                    if size.value:
                        assert chunk(host, ws_bytes=size.value - 1, **args) == WORKSPACE


def test_the_gpu_tests_run_every_way(host):
    from test_kv4_attn_gpu import IN_32, MANY

    def block(h_q, h_kv, d, P, L, window, sinks, splits=0):
        kv = store4(block_size=64, num_blocks=4096, h_kv=h_kv, head_dim=d)
        p = plan_of(host, kv=kv, n_table=4096, P=P, L=L, h_q=h_q, h_kv=h_kv, d=d, window=window, sinks=sinks, splits=splits)
        return 256 if not p["few"] else 16 if L * h_q // h_kv <= 16 * p["row_blocks"] else 32

    for d in (64, 128):
        edges = [(200, 250, w, s, 0) for w in (1, 2, 33, 64, 65, 129, 192) for s in (0, 1, 64, 65)]
        nan = [(100, 300, w, 3 if w else 0, s) for w in (0, 100) for s in (1, 3)] + [(0, 300, 0, 0, 1), (0, 300, 0, 0, 2)]
        for case in MANY + (edges if d == 64 else []) + nan:
            assert block(128, 16, d, *case) == 256, (d, case)
        for window, sinks in ((0, 0), (100, 3)):
            assert block(128, 16, d, 250, 150, window, sinks) == 32
        for case in ((500, 1, 0, 0), (511, 2, 65, 64), (700, 137, 100, 4), (0, 300, 0, 0), (250, 150, 100, 3)):
            assert block(8, 2, d, *case) == 16, (d, case)
    for case in IN_32:
        assert block(*case) == 32, case


def test_blocks_of_heads(host):
    """Groups of more than 16 heads: blocks of 16, of 32 in batches that may be large; workspaces are as planned."""
    size = ctypes.c_size_t()
    for h_q, h_kv, batch, max_len, window, blocks in (
            (16, 1, 1, 100, 0, 1), (17, 1, 1, 100, 0, 2), (64, 1, 18, 700, 0, 4), (20, 1, 18, 700, 0, 2),
            (32, 8, 64, 1 << 20, 0, 1), (32, 1, 32, 8192, 0, 2), (32, 1, 33, 8192, 0, 1), (64, 1, 33, 8192, 0, 2),
            (64, 1, 33, 8192, 1000, 4), (40, 1, 4000, 700, 1, 2), (20, 1, 3012, 700, 1, 1), (40, 2, 3012, 700, 700, 1)):
        kv = store4(h_kv=h_kv)
        args = dict(kv=kv, stride=-(-max_len // 256), batch=batch, max_len=max_len, h_q=h_q, h_kv=h_kv, window=window, sinks=1)
        assert host.mocap_kv4_decode_attn_workspace_size(batch, max_len, h_q, h_kv, 128, window, 1, ctypes.byref(size)) == 0
        assert decode(host, ws_bytes=size.value, **args) == 0
        assert host.record_row_blocks() == blocks, (h_q, h_kv, batch, max_len, window)
        if size.value:
            assert decode(host, ws_bytes=size.value - 1, **args) == WORKSPACE


def test_debug_build_checks_tables(mocap_lib, tmp_path):
    """The checking build refuses what a call's tables may not name, and looks at no other entry."""
    lib = recording_build(mocap_lib, tmp_path, "-DMOCAP_DEBUG_TABLES")
    ints = lambda *x: (ctypes.c_int32 * len(x))(*x)
    at = ctypes.addressof
    good, bad, twice = ints(3, 1, 2, 0), ints(3, 64, 2, -1), ints(3, 1, 3, 0)
    for call in (lambda **k: append(lib, False, **k), lambda **k: append(lib, True, **k)):
        args = dict(start=300, n=200, first=0, n_table=4)             # entry 1 alone
        assert call(table=at(good), **args) == 0 and call(table=at(bad), **args) == INVALID
        assert call(table=at(ints(99, 1, 99, 99)), **args) == 0
        assert call(table=at(twice), start=0, n=600, first=0, n_table=4) == INVALID
    tables = ints(3, 99, 1, 2)
    for call in (lambda **k: batch_append(lib, False, **k), lambda **k: batch_append(lib, True, **k)):
        args = dict(tables=at(tables), stride=2, batch=2)
        assert call(lens=at(ints(256, 300)), **args) == 0
        assert call(lens=at(ints(257, 300)), **args) == INVALID
        assert call(lens=at(ints(0, 513)), **args) == 0               # none, and beyond the tables
    args = dict(tables=at(tables), stride=2, batch=2)
    assert load(lib, lens=at(ints(256, 512)), n=512, **args) == 0
    assert load(lib, lens=at(ints(257, 512)), n=1, **args) == INVALID
    assert decode(lib, lens=at(ints(256, 512)), max_len=512, **args) == 0
    assert decode(lib, lens=at(ints(300, 512)), max_len=512, **args) == INVALID
    assert chunk(lib, table=at(good), n_table=4, P=900, L=100) == 0
    assert chunk(lib, table=at(bad), n_table=4, P=900, L=100) == INVALID
    assert chunk(lib, table=at(ints(99, 99, 1, 2)), n_table=4, P=900, L=100, window=200) == 0


@pytest.mark.parametrize("src", ["rope_append.hip", "kv4_decode.hip", "kv4_chunk.hip"])
def test_kernels_keep_their_values_in_registers(src, tmp_path):
    for name, r in resource_report(src, str(tmp_path)).items():
        assert r.get("VGPRs Spill", 0) == 0 and r.get("ScratchSize [bytes/lane]", 0) == 0, f"{name}: {r}"


def test_rope_and_store_objects():
    """What the binding's objects refuse without a GPU."""
    import torch
    with pytest.raises(ValueError):
        binding.Rope(torch.ones(8))
    with pytest.raises(TypeError):
        binding.Rope([1.0])
    s = binding.Kv4Store(3, 192, 2, 128, device="cpu", fill=7)
    assert s.k_pool.shape == (3, 2, 192, 64) and s.v_pool.shape == (3, 2, 3, 64, 64)
    assert s.k_scale.shape == s.v_scale.shape == (3, 2, 3, 4, 64) and int(s.v_scale.min()) == 7


def test_the_extreme_values_run_every_way(host):
    from test_kv4_extremes_gpu import WAYS

    for way, (h_q, h_kv, P, L, splits, windows) in WAYS.items():
        for d in (64, 128):
            for window in windows:
                kv = store4(block_size=64, num_blocks=4096, h_kv=h_kv, head_dim=d)
                p = plan_of(host, kv=kv, n_table=4096, P=P, L=L, h_q=h_q, h_kv=h_kv, d=d, window=window, splits=splits)
                rows = 256 if not p["few"] else 16 if L * h_q // h_kv <= 16 * p["row_blocks"] else 32
                assert rows == way, (way, d, window, p)
