"""What the compiler says of the kernels for formed scores in the objects that the library is linked from: heads of 64 and 128 in groups of up to eight keep a step's loop in registers, and no instance
spills more than the figures that its times were measured with."""
import os
import re
import subprocess

import pytest

from paper_2504_18154_amd import build


def _vector_spills(source, kernel):
    """{template arguments of an instance: vector registers spilled}"""
    build.build()
    obj = os.path.join(build.OBJ, source.replace(".hip", ".o"))
    tools = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(build._hipcc()))), "llvm", "bin")
    if not os.path.exists(obj) or not os.path.exists(os.path.join(tools, "clang-offload-bundler")):
        pytest.skip("no object, or no tools")
    run = lambda *a: subprocess.run([os.path.join(tools, a[0]), *a[1:]], check=True, capture_output=True, text=True).stdout
    fat, dev = (os.path.join(build.OBJ, f"notes.{os.getpid()}.{x}") for x in ("fat", "dev"))
    try:
        run("llvm-objcopy", f"--dump-section=.hip_fatbin={fat}", obj, fat + ".o")
        run("clang-offload-bundler", "--unbundle", "--type=o", f"--input={fat}", "--targets=hipv4-amdgcn-amd-amdhsa--gfx950", f"--output={dev}")
        notes = run("llvm-readelf", "--notes", dev)
    finally:
        for f in (fat, fat + ".o", dev):
            if os.path.exists(f):
                os.remove(f)
    found = re.findall(rf"\.name:\s+_Z\w*{kernel}I((?:L[ib]\d+E)+)E.*?\.vgpr_spill_count:\s+(\d+)", notes, re.S)
    return {tuple(int(x) for x in re.findall(r"L[ib](\d+)E", args)): int(n) for args, n in found}


def test_decode():
    of = _vector_spills("attn_scored_decode.hip", "decode_scored_kernel")   # (format, chunks, form, wavefronts, full, wide)
    assert len(of) >= 117
    for (fmt, chunks, form, waves, full, wide), n in of.items():
        if fmt == 0 or chunks == 2 or (chunks == 4 and wide and waves == 4):
            most = 0
        elif chunks == 4 and full:
            most = 0 if form < 2 else 2
        elif chunks == 4:
            most = 30
        else:
            most = 24
        assert n <= most, (fmt, chunks, form, waves, full, wide, n)


def test_prefill():
    of = _vector_spills("attn_scored_prefill.hip", "prefill_scored_kernel")   # (format, chunks, form, full, wavefronts)
    assert len(of) >= 96
    for (fmt, chunks, form, full, waves), n in of.items():
        assert n <= (0 if chunks < 8 or form < 2 and full else 15), (fmt, chunks, form, full, waves, n)
