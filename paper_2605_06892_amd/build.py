"""Build libhsa_step.so, the HIP library behind include/hsa_step.h, for gfx950.

Every translation unit under csrc/ is compiled to an object in parallel with
hipcc, then linked into a shared library next to this file. Only the C ABI
symbols are exported (hidden visibility, -Bsymbolic binding), and one of the binding's
(csrc/packed_tile.h). _seq_binding.so, the Python binding of the calls over several
sequences, is host code against torch's headers and that library.

    python -m paper_2605_06892_amd.build
"""

from __future__ import annotations

import glob
import os
import shutil
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
OBJ = os.path.join(ROOT, "_build", "obj")
LIB = os.path.join(PKG, "libhsa_step.so")
BINDING = os.path.join(PKG, "_seq_binding.so")
ARCH = "gfx950"
ROCM = "/opt/rocm"

COMMON = [
    f"--offload-arch={ARCH}",
    "-O3",
    "-std=c++17",
    "-fPIC",
    "-fvisibility=hidden",
    # no packed fp32 VALU instructions in device code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I", os.path.join(ROOT, "include"),
]


def hipcc() -> str:
    exe = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(exe):
        raise RuntimeError("hipcc not found; the HSA step library needs ROCm")
    return exe


def _compile(src: str) -> str:
    obj = os.path.join(OBJ, os.path.basename(src) + ".o")
    cmd = [hipcc(), *COMMON, "-c", src, "-o", obj]
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{r.stdout}")
    return obj


def _run(cmd: list, what: str) -> None:
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"{what} failed:\n{r.stdout}")


def _compile_binding() -> str:
    import torch
    from torch.utils import cpp_extension

    obj = os.path.join(OBJ, "seq_binding.cpp.o")
    includes = [*cpp_extension.include_paths(), sysconfig.get_path("include"), os.path.join(ROCM, "include")]
    _run(["g++", "-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden", "-D__HIP_PLATFORM_AMD__",
          f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}", *[f"-I{i}" for i in includes],
          "-c", os.path.join(CSRC, "seq_binding.cpp"), "-o", obj], "g++ for seq_binding.cpp")
    return obj


def _link_binding(obj: str) -> None:
    from torch.utils import cpp_extension

    tmp = BINDING + ".tmp"
    _run(["g++", "-shared", "-o", tmp, obj, f"-L{PKG}", "-l:libhsa_step.so", "-Wl,-rpath,$ORIGIN",
          *[f"-L{p}" for p in cpp_extension.library_paths()], "-ltorch_python", "-ltorch_cpu", "-lc10"],
         "linking _seq_binding.so")
    os.replace(tmp, BINDING)


def build(jobs: int | None = None) -> str:
    """Compile and link the library and its binding; returns the library's path. Always
    rebuilds. What only the binding needs (g++, torch's headers) does not keep the library from
    being built: without it the library is in place when this raises, and a former binding is not."""
    os.makedirs(OBJ, exist_ok=True)
    srcs = sorted(glob.glob(os.path.join(CSRC, "*.hip")))
    if not srcs:
        raise RuntimeError("no HIP sources found")
    jobs = jobs or min(len(srcs), max(1, min(16, os.cpu_count() or 1)))
    with ThreadPoolExecutor(jobs) as ex:
        binding = ex.submit(_compile_binding)
        objs = list(ex.map(_compile, srcs))
    tmp = LIB + ".tmp"
    cmd = [hipcc(), f"--offload-arch={ARCH}", "-shared", "-fPIC", "-Wl,-Bsymbolic", "-o", tmp, *objs]
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}")
    os.replace(tmp, LIB)
    try:
        _link_binding(binding.result())
    except Exception as e:
        if os.path.exists(BINDING):
            os.remove(BINDING)
        raise RuntimeError(f"{LIB} is built, its binding of the calls over several sequences is not: {e}") from e
    return LIB


if __name__ == "__main__":
    path = build()
    print(path)
    sys.exit(0)
