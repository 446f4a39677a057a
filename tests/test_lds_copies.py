"""The machine code of the built library around its copies from memory to LDS -- CPU only.

Such a copy takes its LDS address from m0, and the instruction set asks for one
wait state between a scalar write of m0 and the copy.  The copies are inline
assembly, where the compiler adds none."""
import glob
import os
import re
import shutil
import subprocess

import pytest

spk = pytest.importorskip("paper_1903_02440_amd")

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no disassembler")
def test_no_copy_directly_after_a_write_of_m0(tmp_path):
    lib = shutil.copy(os.path.join(os.path.dirname(spk.__file__), "libspyke.so"), tmp_path)
    subprocess.run([OBJDUMP, "--offloading", lib], check=True, capture_output=True, cwd=tmp_path)
    copies, bad = 0, []
    for obj in sorted(glob.glob(os.path.join(tmp_path, "*gfx950"))):
        text = subprocess.run([OBJDUMP, "-d", obj], check=True, capture_output=True, text=True).stdout
        kernel, before = "", ""
        for line in text.splitlines():
            name = re.match(r"[0-9a-f]+ <(.*)>:", line)
            if name:
                kernel, before = name.group(1), ""
            elif line.startswith("\t"):
                if "load_lds" in line:
                    copies += 1
                    if re.match(r"\ts_\w+ m0\b", before):
                        bad.append((kernel, before.split("//")[0].strip()))
                before = line
    assert copies > 0
    assert not bad, f"{len(bad)} of {copies}, the first in {bad[0]}"
