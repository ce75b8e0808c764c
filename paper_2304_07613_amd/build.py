"""Build step for libnmg.so (hipcc, gfx950) -- run by ``__graft_entry__.build()``.

Every translation unit under csrc/ is compiled to an object in parallel, then
the objects are linked into one shared library; the link is checked for
undefined kernel launch stubs.  csrc/gen_gelu_table.py writes the binary16
GELU table into the build folder first.  csrc/calls.cpp, the marshalling of the
attention operators' calls, becomes a Python module beside the library (host code,
g++ against torch's headers); the library does not need it.
"""
from __future__ import annotations

import glob
import importlib.metadata
import os
import subprocess
import sys
import sysconfig
import tempfile
import warnings
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
HEADER = os.path.join(ROOT, "include", "nmg.h")
LIB_PATH = os.path.join(HERE, "libnmg.so")
CALLS_SRC = os.path.join(CSRC, "calls.cpp")


def calls_path() -> str:
    """The module _calls for this Python and this torch: it is built against both."""
    try:
        torch = importlib.metadata.version("torch")
    except importlib.metadata.PackageNotFoundError:
        torch = "none"
    return os.path.join(HERE, f"_calls.torch-{torch}{sysconfig.get_config_var('EXT_SUFFIX')}")


HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall",
    # no packed binary32 instructions anywhere in the device code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # binary32 subnormals take part in the group scores: never flush them
    "-fno-gpu-flush-denormals-to-zero", "-fno-fast-math",
]


def sources() -> list:
    return sorted(glob.glob(os.path.join(CSRC, "*.hip")))


GENERATORS = [os.path.join(CSRC, "gen_gelu_table.py")]


def inputs() -> list:
    """Every file the library is built from."""
    return sorted(sources() + glob.glob(os.path.join(CSRC, "*.hpp")) +
                  [HEADER, CALLS_SRC] + GENERATORS)


def _clean(text: str) -> str:
    return "\n".join(l for l in text.splitlines()
                     if "packed-fp32-ops" not in l and "not a recognized feature" not in l)


def build_calls() -> str:
    """Compile csrc/calls.cpp into the Python module _calls."""
    import torch
    from torch.utils import cpp_extension

    inc = [os.path.dirname(HEADER), os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "include"),
           sysconfig.get_paths()["include"], *cpp_extension.include_paths()]
    path = calls_path()
    tmp = path + ".tmp"
    lib = cpp_extension.library_paths()[0]
    res = subprocess.run(
        [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall",
         "-D__HIP_PLATFORM_AMD__",   # what HIP's headers (nmg.h's stream type) ask of a host compiler
         f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
         *[arg for d in inc for arg in ("-isystem", d)], "-o", tmp, CALLS_SRC, "-L", lib,
         "-ltorch_python", "-ltorch_cpu", "-lc10"], capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"calls.cpp failed:\n{res.stdout}{res.stderr}")
    os.replace(tmp, path)
    return path


def build(verbose: bool = False, jobs: int | None = None) -> str:
    """Compile csrc/*.hip into libnmg.so, and the module _calls, next to this
    file (always rebuilds).  A module that does not compile is a warning, and gone:
    the library is there without it, and the binding's attention operators say so
    when they are called."""
    with ThreadPoolExecutor(max_workers=1) as pool:
        calls = pool.submit(build_calls)
        library = build_library(verbose, jobs)
    try:
        calls.result()
    except Exception as e:
        if os.path.exists(calls_path()):    # of other sources
            os.remove(calls_path())
        warnings.warn(f"the attention operators' Python module is not built: {e}", RuntimeWarning)
    return library


def build_library(verbose: bool = False, jobs: int | None = None) -> str:
    """Compile csrc/*.hip into libnmg.so."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    jobs = jobs or min(16, os.cpu_count() or 4)
    inc = ["-I", os.path.join(ROOT, "include")]
    with tempfile.TemporaryDirectory(prefix="nmg_build_") as tmpdir:
        # generated sources (the binary16 GELU table) go to the build folder
        gen = subprocess.run([sys.executable, GENERATORS[0], os.path.join(tmpdir, "gelu_f16_table.inc")],
                             capture_output=True, text=True)
        if gen.returncode != 0:
            raise RuntimeError(f"gen_gelu_table.py failed:\n{gen.stdout}{gen.stderr}")
        inc += ["-I", tmpdir]
        def compile_one(src):
            obj = os.path.join(tmpdir, os.path.basename(src) + ".o")
            res = subprocess.run([hipcc, *HIPCC_FLAGS, *inc, "-c", "-o", obj, src],
                                 capture_output=True, text=True)
            return src, obj, res
        with ThreadPoolExecutor(max_workers=jobs) as pool:
            results = list(pool.map(compile_one, sources()))
        errors = [(s, r) for s, _, r in results if r.returncode != 0]
        if errors:
            s, r = errors[0]
            raise RuntimeError(f"hipcc failed on {os.path.basename(s)}:\n{_clean(r.stdout + r.stderr)}")
        if verbose:
            for s, _, r in results:
                out = _clean(r.stdout + r.stderr).strip()
                if out:
                    print(f"{os.path.basename(s)}:\n{out}")
        tmp = LIB_PATH + ".tmp"
        res = subprocess.run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp,
                              *[o for _, o, _ in results]], capture_output=True, text=True)
        if res.returncode != 0:
            raise RuntimeError(f"link failed:\n{_clean(res.stdout + res.stderr)}")
    # every kernel's host launch stub must be defined in the library
    nm = subprocess.run(["nm", "-D", "--undefined-only", tmp], capture_output=True, text=True)
    missing = [l.split()[-1] for l in nm.stdout.splitlines() if "__device_stub__" in l]
    if nm.returncode != 0 or missing:
        raise RuntimeError(f"libnmg.so has undefined kernel stubs: {missing[:3]} (nm rc {nm.returncode})")
    os.replace(tmp, LIB_PATH)
    return LIB_PATH


def is_stale() -> bool:
    """Whether the library, or the module for this Python and torch, is missing or
    older than what it is built from."""
    if not (os.path.exists(LIB_PATH) and os.path.exists(calls_path())):
        return True
    t = min(os.path.getmtime(LIB_PATH), os.path.getmtime(calls_path()))
    return any(os.path.getmtime(p) > t for p in inputs())


if __name__ == "__main__":
    print(build(verbose=True))
