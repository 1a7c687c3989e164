"""What the compiler made of the conversions of queries in the 4-bit cache's attention."""
import os
import re
import shutil
import subprocess

import pytest

OBJDUMP = os.environ.get("LLVM_OBJDUMP", "/opt/rocm/llvm/bin/llvm-objdump")


@pytest.mark.skipif(shutil.which(OBJDUMP) is None, reason="llvm-objdump not found")
def test_conversions_of_queries_write_over_nothing_they_read(tmp_path):
    """v_cvt_scalef32_2xpk16_fp6_f32 and v_cvt_scalef32_pk32_f32_fp6 write several registers while they still read: no register of the result may be one of theirs."""
    from paper_2605_25655_amd import build
    lib = shutil.copy(build.LIB, str(tmp_path / "lib.so"))
    subprocess.run([OBJDUMP, "--offloading", lib], cwd=tmp_path, check=True, stdout=subprocess.DEVNULL)
    seen = 0
    for code in sorted(str(p) for p in tmp_path.iterdir() if p.name.endswith("gfx950")):
        for line in subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", code], capture_output=True, text=True, check=True).stdout.split("\n"):
            if not re.search(r"v_cvt_scalef32_(2xpk16|pk32)_", line):
                continue
            seen += 1
            to, *of = [set(range(int(a), int(b or a) + 1)) for a, b in re.findall(r"\bv\[?(\d+)(?::(\d+))?", line.split("scalef32", 1)[1].split(" ", 1)[1])]
            assert len(to) in (6, 32) and len(of) in (2, 3) and not to & set().union(*of), line.strip()
    assert seen >= 7 * 8, seen              # seven of a tile of rows, eight tiles in the six kernels
