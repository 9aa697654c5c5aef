"""Build libmocap_attn.so for gfx950 (in-tree, next to this file).

Every HIP source is compiled with hipcc for gfx950 only, with packed-fp32
instructions disabled in device code, then linked into one shared library.
"""
import os
import subprocess
import sys
import sysconfig
import warnings
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD_DIR = os.path.join(ROOT, "_build")
LIB = os.path.join(PKG, "libmocap_attn.so")
SOURCES = ["api.cpp", "plan.cpp", "chunk_attn.hip", "chunk_attn_short.hip", "kv_append.hip", "lse_merge.hip",
           "serve_api.cpp", "decode_attn.hip", "window_attn.hip", "key_weights.hip", "kv_evict.hip",
           "cache_api.cpp", "rope_append.hip", "kv4_decode.hip", "kv4_chunk.hip"]
ARCH = "gfx950"

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # MFMA results in VGPRs: the score accumulators feed the softmax VALU work
    # directly, with no copies out of accumulation registers.
    "-mllvm", "-amdgpu-mfma-vgpr-form=true",
    "-Wno-unused-command-line-argument",
    f"-I{INCLUDE}", f"-I{CSRC}",
]


def _compile(src: str, verbose: bool, build_dir: str, extra_flags) -> str:
    obj = os.path.join(build_dir, os.path.splitext(src)[0] + ".o")
    cmd = [HIPCC, *FLAGS, *extra_flags, "-x", "hip", "-c", os.path.join(CSRC, src), "-o", obj]
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError(f"hipcc failed on {src}")
    return obj


def build(verbose: bool = False, extra_flags=(), lib_path: str = LIB, build_dir: str = BUILD_DIR) -> str:
    """Compile every source and link ``lib_path``.  ``extra_flags`` (e.g. -D
    tuning macros) and an alternative output location serve experiments."""
    os.makedirs(build_dir, exist_ok=True)
    with ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        objs = list(ex.map(lambda s: _compile(s, verbose, build_dir, tuple(extra_flags)), SOURCES))
    tmp = lib_path + ".tmp"
    cmd = [HIPCC, f"--offload-arch={ARCH}", "-shared", "-fPIC", *objs, "-o", tmp]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    _check_stubs(tmp)
    os.replace(tmp, lib_path)
    if lib_path == LIB:
        try:
            build_marshal(verbose)
        except Exception as e:  # no g++, or without the headers of Python or torch
            if os.path.exists(MARSHAL):
                os.remove(MARSHAL)
            warnings.warn(f"the binding's shortcuts were not built, its calls take some us longer without them: {e}")
    return lib_path


# Named for the Python that it is built for; it holds the torch that it is built for.
MARSHAL = os.path.join(PKG, "_marshal" + sysconfig.get_config_var("EXT_SUFFIX"))


def build_marshal(verbose: bool = False) -> str:
    """The binding's shortcuts (csrc/marshal.cpp): a Python extension over torch's headers, host code only."""
    import torch
    from torch.utils import cpp_extension
    includes = [*cpp_extension.include_paths(), sysconfig.get_path("include")]
    lib_dir = os.path.join(os.path.dirname(torch.__file__), "lib")
    tmp = MARSHAL + ".tmp"
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", "-w",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", f'-DMOCAP_TORCH="{torch.__version__}"',
           *(f"-isystem{i}" for i in includes), f"-I{INCLUDE}", os.path.join(CSRC, "marshal.cpp"), "-o", tmp,
           f"-L{lib_dir}", "-lc10", "-ltorch_cpu", "-ltorch_python"]
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError(f"{cmd[0]} failed on marshal.cpp")
    os.replace(tmp, MARSHAL)
    return MARSHAL


def stale() -> list:
    """Which of the library and the shortcuts are missing or older than what they are built from."""
    headers = [os.path.join(INCLUDE, f) for f in os.listdir(INCLUDE)]
    marshal = os.path.join(CSRC, "marshal.cpp")
    sources = [os.path.join(CSRC, f) for f in os.listdir(CSRC)]
    made_from = {LIB: headers + [s for s in sources if s != marshal], MARSHAL: headers + [marshal]}
    return [made for made, parts in made_from.items()
            if not os.path.exists(made) or any(os.path.getmtime(s) > os.path.getmtime(made) for s in parts)]


def _check_stubs(lib: str) -> None:
    """Fail if a kernel's host launch stub was not emitted.

    If a kernel body does not compile for the host pass, clang can drop the
    template's stub without an error, leaving an undefined symbol that only
    shows up when the library is loaded."""
    out = subprocess.run(["nm", "-C", lib], check=True, capture_output=True, text=True).stdout
    missing = [ln.strip() for ln in out.splitlines() if " U " in ln and "__device_stub__" in ln]
    if missing:
        raise RuntimeError("kernel launch stubs missing from " + lib + ":\n" + "\n".join(missing))


DEBUG_LIB = os.path.join(PKG, "libmocap_attn_debug.so")


def build_debug(verbose: bool = False) -> str:
    """The library with host-side block-table checks before every launch
    (-DMOCAP_DEBUG_TABLES): libmocap_attn_debug.so, for debugging callers."""
    return build(verbose, extra_flags=("-DMOCAP_DEBUG_TABLES",), lib_path=DEBUG_LIB,
                 build_dir=os.path.join(BUILD_DIR, "debug"))


if __name__ == "__main__":
    if "--debug-tables" in sys.argv:
        print(build_debug(verbose="-v" in sys.argv))
    else:
        print(build(verbose="-v" in sys.argv))
