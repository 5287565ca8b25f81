"""Wide buffer stores of the built library keep their whole offset in a vector register.

With part of it in a scalar register the compiler takes a store's data for read at once and leaves no instruction between
it and the next write of those registers; on gfx950 the store may then write some of the new values.  Looked at in the
assembly, since nothing in the source says what the compiler does with an offset.
"""
import os
import re
import shutil
import subprocess

import pytest

from paper_2410_10989_amd import _build

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"


def wide_stores(assembly):
    """Scalar offsets of the buffer stores of 8 bytes or more per lane."""
    return re.findall(r"buffer_store_dwordx[234] v\[[0-9:]+\], (?:v\d+|off), s\[[0-9:]+\], (\S+)", assembly)


def test_the_pattern():
    text = ("\tbuffer_store_dwordx4 v[40:43], v66, s[0:3], s9 offen       // 00\n\tbuffer_store_dwordx4 v[4:7], v6, s[0:3], 0 offen offset:16\n"
            "\tbuffer_store_dwordx2 v[4:5], off, s[0:3], s4\n\tbuffer_store_short v4, v6, s[0:3], s4 offen\n")
    assert wide_stores(text) == ["s9", "0", "s4"]


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no disassembler")
def test_no_wide_store_has_a_scalar_offset(tmp_path):
    if _build.is_stale():
        _build.build()
    lib = shutil.copy(_build.LIB_PATH, tmp_path)   # (its device code is put beside it)
    subprocess.run([OBJDUMP, "--offloading", lib], check=True, stdout=subprocess.DEVNULL)
    objects = sorted(p for p in os.listdir(tmp_path) if p.endswith("gfx950"))
    assert len(objects) == len(_build.sources())
    seen = []
    for name in objects:
        res = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", "--no-leading-addr", name], cwd=tmp_path, check=True,
                             stdout=subprocess.PIPE, text=True)
        seen += wide_stores(res.stdout)
    assert len(seen) > 100, "the products' stores are not where they were"
    scalar = [s for s in seen if s != "0"]
    assert not scalar, f"{len(scalar)} of {len(seen)} wide stores with a scalar offset"
