"""The binding's shortcuts in C++ (csrc/marshal.cpp) while other Python threads run.  No GPU: a build of them over CPU
tensors, and calls in the library's place that wait until another thread lets them go."""
import ctypes
import importlib.machinery
import importlib.util
import os
import subprocess
import threading
import time
import weakref

import pytest
import torch

from paper_2606_22968_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CALLS = ("mocap_rope_append", "mocap_kv4_append", "mocap_decode_rope_append", "mocap_kv4_decode_append", "mocap_kv4_load",
         "mocap_kv4_decode_attn", "mocap_kv4_chunk_attn")


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    """(module, its other symbols)"""
    import sysconfig

    from torch.utils import cpp_extension
    path = str(tmp_path_factory.mktemp("marshal") / "_marshal.so")
    includes = [*cpp_extension.include_paths(), sysconfig.get_path("include")]
    cmd = ["g++", "-O1", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", "-w",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", '-DMOCAP_TORCH="host"',
           *(f"-isystem{i}" for i in includes), f"-I{build.INCLUDE}", os.path.join(ROOT, "tests", "marshal_host.cpp"), "-o", path,
           f"-L{os.path.join(os.path.dirname(torch.__file__), 'lib')}", "-lc10", "-ltorch_cpu", "-ltorch_python"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    loader = importlib.machinery.ExtensionFileLoader("_marshal", path)
    module = importlib.util.module_from_spec(importlib.util.spec_from_loader("_marshal", loader))
    loader.exec_module(module)
    lib = ctypes.CDLL(path)
    lib.waiting_call.restype, lib.waiting_call.argtypes = ctypes.c_void_p, [ctypes.c_char_p]
    for name in CALLS:
        module.bind(name, lib.waiting_call(name.encode()))
    return module, lib


class Store:
    """What the shortcuts read of a KvStore or a Kv4Store."""

    def __init__(self, four):
        self.num_blocks, self.block_size, self.h_kv, self.head_dim = 3, 64, 2, 64
        shapes = dict(k_pool=(3, 2, 64, 32), v_pool=(3, 2, 1, 32, 64), k_scale=(3, 2, 1, 2, 64), v_scale=(3, 2, 1, 2, 64))
        if not four:
            shapes = dict(k_pool=(3, 2, 64, 64), v_pool=(3, 2, 64, 64))
        self.pools = tuple(shapes)
        for name, shape in shapes.items():
            setattr(self, name, torch.zeros(shape, dtype=torch.uint8 if four else torch.bfloat16))


class Rope:
    inv_freq, interleaved = None, False


def arguments(name):
    """A store, a rotation and the arguments behind the store, without stream and device."""
    store, rope = Store("kv4" in name), Rope()
    rope.inv_freq = torch.ones(32)
    rows = torch.zeros((2, 8, 64), dtype=torch.bfloat16)
    q, k, v, out = rows[:, :4], rows[:, 4:6], rows[:, 6:], torch.zeros((2, 4, 64), dtype=torch.bfloat16)
    table, lens = torch.zeros(3, dtype=torch.int32), torch.ones(2, dtype=torch.int32)
    tables = torch.zeros((2, 3), dtype=torch.int32)
    if name.endswith("decode_append") or "decode_rope" in name:
        return store, rope, (tables, lens, k, v, rope, lens, q, out)
    if name.endswith("append"):
        return store, rope, (table, 3, k, v, rope, None, q, out)
    if name.endswith("load"):
        return store, rope, (tables, lens, *(torch.zeros((2, 5, 2, 64), dtype=torch.bfloat16) for _ in range(2)))
    if "decode" in name:
        return store, rope, (tables, lens, out, 192, 0.1, torch.zeros_like(out), torch.zeros((2, 4)), None, 0, 0)
    return store, rope, (table, out, 50, 0.1, torch.zeros_like(out), torch.zeros((4, 2)), None, 0, 0, 1)


@pytest.mark.parametrize("name", CALLS)
def test_other_threads_run_during_a_call(host, name):
    """Another thread goes on while a call waits, and may even replace the tensors that the call's objects name: the call
    holds those that it was made with."""
    module, lib = host
    lib.waiting_reset()
    store, rope, args = arguments(name)
    uses_rope = any(a is rope for a in args)
    alive = []

    def other():
        while not lib.waiting_entered():
            time.sleep(0.001)
        for owner, names in ((store, store.pools), (rope, ("inv_freq",) if uses_rope else ())):
            for x in names:
                held = weakref.ref(getattr(owner, x))
                setattr(owner, x, None)
                alive.append((x, held, held() is not None))
        lib.waiting_release()

    thread = threading.Thread(target=other)
    thread.start()
    status = getattr(module, name)(store, *args, None, -1)
    thread.join()
    assert status == 0, "no other thread ran during the call"
    assert alive and all(held for _, _, held in alive)
    assert all(ref() is None for _, ref, _ in alive)
