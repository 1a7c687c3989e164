"""How attention over the 4-bit cache is cut: into no more workgroups than fit on the compute units at a time, by the registers that the kernels have as built."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
LLVM = os.environ.get("LLVM_BIN", "/opt/rocm/llvm/bin")
CUS = 256


@pytest.fixture(scope="module")
def fits(tmp_path_factory):
    """{(kernel, D, several tokens): workgroups that fit on a compute unit}, from the registers of a lane (512 to share on each of four SIMDs)."""
    from paper_2605_25655_amd import build
    d = tmp_path_factory.mktemp("lib")
    lib = shutil.copy(build.LIB, str(d / "lib.so"))
    subprocess.run([os.path.join(LLVM, "llvm-objdump"), "--offloading", lib], cwd=d, check=True, stdout=subprocess.DEVNULL)
    found = {}
    for code in sorted(str(p) for p in d.iterdir() if p.name.endswith("gfx950")):
        notes = subprocess.run([os.path.join(LLVM, "llvm-readelf"), "--notes", code], capture_output=True, text=True, check=True).stdout
        for part in notes.split(".agpr_count")[1:]:
            m = re.search(r"kv4_attn_(decode|prompt)ILi(\d+)E(?:Lb(\d)|Li\d+)E", part)
            if m:
                registers = -(-int(re.search(r"\.vgpr_count:\s*(\d+)", part).group(1)) // 8) * 8
                found[m.group(1), int(m.group(2)), m.group(3) == "1"] = 512 // registers // (1 if m.group(1) == "decode" else 2)
    assert len(found) == 6, found
    return found


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("plan") / "driver")
    res = subprocess.run([HIPCC, "-O1", "-std=c++17", "--offload-arch=gfx950", "-Wno-unused-command-line-argument", "-o", exe,
                          os.path.join(ROOT, "paper_2605_25655_amd", "csrc", "kv4_api.hip"), "-x", "hip", os.path.join(ROOT, "tests", "plan", "kv4_plan_driver.cpp")],
                         capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-4000:]

    def ask(shapes):
        out = subprocess.run([exe], input="\n".join(" ".join(map(str, s)) for s in shapes), capture_output=True, text=True, check=True).stdout
        return [tuple(map(int, line.split())) for line in out.splitlines()]
    return ask


@pytest.mark.skipif(shutil.which(HIPCC) is None, reason="hipcc not found")
@pytest.mark.parametrize("Hq,Hkv,D", [(8, 8, 64), (32, 32, 128), (64, 8, 128), (34, 2, 64), (40, 40, 128)])
def test_no_more_chunks_than_fit(plan, fits, Hq, Hkv, D):
    shapes = [(B, Hq, Hkv, D, new, pages) for B in (1, 2, 3, 4, 6, 16, 33) for new in (1, 2, 4, 8, 33, 65, 129, 700, 3000) for pages in (1, 16, 17, 40, 300, 2047)]
    plans, cut = plan(shapes), set()
    assert len(plans) == len(shapes)
    for (B, _, _, _, new, pages), (few, tiles, nsplit, least) in zip(shapes, plans):
        if nsplit == 1:
            continue
        items = B * Hkv * (tiles if few else -(-tiles // 16))
        room = fits["decode" if few else "prompt", D, few and new > 1]
        assert items * nsplit <= room * CUS and nsplit <= -(-pages // least), (B, new, pages, nsplit)
        cut.add((few, new > 1))
    assert cut == {(1, False), (1, True), (0, True)}, cut
