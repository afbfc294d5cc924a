"""Compile csrc/*.hip for gfx950 into paper_2504_18154_amd/libecoserve.so, and csrc/bind.cpp (the binding's marshalling, against the
installed torch) into paper_2504_18154_amd/_bind.so (in-tree).

    python -m paper_2504_18154_amd.build [--force]

hipcc cross-compiles without a GPU.  Objects go to paper_2504_18154_amd/_build/.
"""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libecoserve.so")
BIND = os.path.join(HERE, "_bind.so")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")

SOURCES = ["api.hip", "kv_append.hip", "attn_plain.hip", "attn_any_mfma.hip", "attn_decode_mfma.hip", "decode_noalloc.hip", "attn_prefill_mfma.hip", "attn_prefill_short.hip", "kv_rope.hip", "kv_summary.hip", "block_select.hip", "attn_sparse.hip", "probes.hip", "padg.hip"]
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall", "-Wno-unused-command-line-argument",
         # packed fp32 VALU forms are kept out of generated code on this target
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]


def _hipcc() -> str:
    for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if c and (os.path.isabs(c) and os.path.exists(c) or not os.path.isabs(c)):
            return c
    return "hipcc"


def _deps_mtime() -> float:
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(INCLUDE, "ecoserve.h")]
    return max(os.path.getmtime(p) for p in deps)


def _bind_fits() -> str:
    """What csrc/bind.cpp is compiled against, as it stands in _bind.so (its module's documentation)."""
    import torch
    return f"for {sys.implementation.cache_tag}, torch {torch.__version__}, C++11 ABI {int(torch._C._GLIBCXX_USE_CXX11_ABI)}."


def is_current() -> bool:
    """Both libraries are newer than their sources, and _bind.so is for the installed torch and this interpreter."""
    if not all(os.path.exists(p) and os.path.getmtime(p) >= _deps_mtime() for p in (LIB, BIND)):
        return False
    with open(BIND, "rb") as f:
        return _bind_fits().encode() in f.read()


def _build_bind() -> None:
    import torch
    root = os.path.dirname(torch.__file__)
    rocm = os.path.dirname(os.path.dirname(os.path.realpath(_hipcc()))) if os.path.isabs(_hipcc()) else "/opt/rocm"
    includes = [os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"), os.path.join(rocm, "include"),
                sysconfig.get_paths()["include"]]
    abi = f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}"
    libs = os.path.join(root, "lib")
    cmd = [os.environ.get("CXX") or "g++", "-std=c++17", "-O2", "-fPIC", "-shared", "-Wall", "-D__HIP_PLATFORM_AMD__=1", "-DUSE_ROCM=1", abi,
           f'-DECO_BIND_FITS="{_bind_fits()}"',
           *(a for i in includes for a in ("-isystem", i)), os.path.join(CSRC, "bind.cpp"), "-o", BIND, "-L", libs, "-ltorch_python", "-ltorch_cpu", "-lc10",
           "-lc10_hip", f"-Wl,-rpath,{libs}"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"{cmd[0]} failed on bind.cpp:\n{r.stderr}")


def build(force: bool = False, verbose: bool = True) -> str:
    if not force and is_current():
        return LIB
    os.makedirs(OBJ, exist_ok=True)
    hipcc = _hipcc()

    def compile_one(src: str) -> str:
        obj = os.path.join(OBJ, src.replace(".hip", ".o"))
        cmd = [hipcc, *FLAGS, "-I", INCLUDE, "-c", os.path.join(CSRC, src), "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        # the host pass does not know the target feature above and says so; drop that line
        err = "\n".join(l for l in r.stderr.splitlines() if "is not a recognized feature for this target" not in l)
        if r.returncode != 0:
            raise RuntimeError(f"hipcc failed on {src}:\n{err}")
        if verbose and err.strip():
            print(err, file=sys.stderr)
        return obj

    with ThreadPoolExecutor(max_workers=min(8, len(SOURCES) + 1)) as ex:
        bind = ex.submit(_build_bind)
        objs = list(ex.map(compile_one, SOURCES))
        bind.result()
    cmd = [hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objs]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stderr}")
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv))
