"""The 4-bit cache's attention on the CPU: that the bounds of the GPU tests notice a summand less, and what the compiler made of the queries' conversions."""
import os
import re
import shutil
import subprocess

import numpy as np
import pytest

from tests import kv4_bounds as bounds
from tests.test_kv4_gpu import attention_case

OBJDUMP = os.environ.get("LLVM_OBJDUMP", "/opt/rocm/llvm/bin/llvm-objdump")


def _summands(x, n):
    """x [..., D] as n e2m3 summands, 2^-4 apart, of scales by blocks of 32."""
    rest = x.reshape(*x.shape[:-1], -1, 32)
    big = np.abs(rest).max(-1, keepdims=True)
    e = np.floor(np.log2(big)) - 2
    e = np.where(big > 7.5 * 2.0 ** e, e + 1, e)
    total = np.zeros_like(rest)
    for s in range(n):
        u = rest / 2.0 ** (e - 4 * s)
        step = 2.0 ** np.maximum(np.floor(np.log2(np.maximum(np.abs(u), 1e-30))) - 3, -3)
        part = np.clip(np.round(u / step) * step, -7.5, 7.5) * 2.0 ** (e - 4 * s)
        total, rest = total + part, rest - part
    return total.reshape(x.shape)


@pytest.mark.parametrize("D", [64, 128])
def test_bounds_notice_a_summand_less(D):
    """The definition with queries of four summands stays inside the tolerance, with three it does not; with weights of two fp16 summands it does, with one not."""
    for lens, new in (([2] * 40, [1] * 40), ([12] * 3, [12] * 3)):
        c = bounds.far_queries(D, 4, 2, D, lens, new)
        y, tol = bounds.attention(c, 0.125)
        for n in (4, 3):
            off = dict(c, q=_summands(c["q"].astype(np.float64), n))
            ratio = (np.abs(bounds.attention(off, 0.125)[0] - y) / tol).max()
            assert (ratio <= 1) == (n == 4), (n, ratio)
    c, scale = bounds.whole_queries(attention_case(D + 1, 4, 2, D, [2, 3, 4, 5, 7, 9, 12, 16] * 3, [1] * 24))
    assert np.array_equal(_summands(c["q"].astype(np.float64), 4), c["q"].astype(np.float64))
    y, tol = bounds.attention(c, scale, query=0.0)

    def fp16(p):
        return (512 * p).astype(np.float16).astype(np.float64) / 512

    for weights, fine in ((lambda p: fp16(p) + fp16(p - fp16(p)), True), (fp16, False)):
        ratio = (np.abs(bounds.attention(c, scale, query=0.0, weights=weights)[0] - y) / tol).max()
        assert (ratio <= 1) == fine, ratio


def test_queries_left_is_within_the_bound():
    """Four summands over all of a block's borders: what is left against 2^-16 / 3.75 of the largest, and that 2^-18 would be too little."""
    rng = np.random.default_rng(5)
    x = rng.uniform(-1, 1, (4000, 64)) * np.repeat(np.linspace(3.75, 7.5, 4000), 64).reshape(4000, 64)
    x[:, ::32] = np.linspace(3.7501, 7.5, 4000)[:, None]
    x = x.astype(np.float32).astype(np.float64)
    left = np.abs(_summands(x, 4) - x).reshape(-1, 32).max(-1) / np.abs(x).reshape(-1, 32).max(-1)
    assert 2.0 ** -18 < left.max() <= bounds.QUERY


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
