"""The 4-bit cache on the CPU: refusals and workspace sizes of the C ABI (no launch), the host code under sanitizers, and the plain
implementation that the GPU tests compare with."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

from tests import kv4_reference as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
NULL, SHAPE, ALIGN, WORKSPACE = 1, 2, 3, 4


@pytest.fixture(scope="module")
def lib():
    from paper_2605_25655_amd import binding
    if not os.path.exists(binding.library_path()):
        from paper_2605_25655_amd import build
        build.build(verbose=False)
    return binding.load_library()


def _places():
    buf = ctypes.create_string_buffer(1 << 13)
    p = (ctypes.addressof(buf) + 255) // 256 * 256
    return buf, p


def refused(call, good, changes):
    """call(*good) with one argument changed at a time returns the status that goes with it."""
    for (i, value), status in changes:
        args = list(good)
        args[i] = value
        assert call(*args) == status, (i, value, status)


def test_append_refusals(lib):
    buf, p = _places()
    #       0    1    2  3  4     5  6  7  8  9  10 11 12 13   14  15
    good = [p, 1024, p, p, 1e-6, p, p, p, p, p, 3, 4, 2, 128, 10, None]
    refused(lib.thi_qk_norm_rope_kv4, good, [
        ((0, None), NULL), ((7, None), NULL), ((8, None), NULL), ((9, None), NULL), ((5, None), NULL),      # theta without positions
        ((10, 0), SHAPE), ((10, -1), SHAPE), ((11, 3), SHAPE), ((11, 0), SHAPE), ((12, 0), SHAPE), ((12, -2), SHAPE), ((13, 96), SHAPE), ((13, 256), SHAPE),
        ((1, 1016), SHAPE), ((1, 1028), SHAPE), ((14, 0), SHAPE), ((14, (1 << 25)), SHAPE),
        ((0, p + 8), ALIGN), ((2, p + 2), ALIGN), ((3, p + 4), ALIGN), ((5, p + 2), ALIGN), ((6, p + 1), ALIGN), ((7, p + 2), ALIGN), ((8, p + 8), ALIGN), ((9, p + 8), ALIGN)])


def test_read_refusals(lib):
    buf, p = _places()
    good = [p, p, p, p, 3, 2, 64, 10, None]
    refused(lib.thi_kv4_read, good, [((0, None), NULL), ((1, None), NULL), ((4, 0), SHAPE), ((5, 0), SHAPE), ((6, 32), SHAPE), ((7, 0), SHAPE),
                                     ((1, p + 2), ALIGN), ((2, p + 8), ALIGN), ((3, p + 2), ALIGN)])
    assert lib.thi_kv4_read(p, p, None, None, 3, 2, 64, 10, None) == NULL


def test_attention_refusals(lib):
    buf, p = _places()
    big = 1 << 40
    #       0  1  2  3  4  5    6  7  8  9  10 11   12 13 14 15 16  17
    good = [p, p, p, p, p, 0.1, p, 2, 5, 8, 2, 128, 4, 9, 3, p, big, None]
    refused(lib.thi_kv4_attention, good, [
        ((0, None), NULL), ((1, None), NULL), ((2, None), NULL), ((3, None), NULL), ((6, None), NULL), ((15, None), NULL),
        ((7, 0), SHAPE), ((7, 65536), SHAPE), ((8, 0), SHAPE), ((9, 7), SHAPE), ((10, 3), SHAPE), ((11, 80), SHAPE), ((12, 0), SHAPE), ((12, 6), SHAPE), ((13, 0), SHAPE),
        ((14, 0), SHAPE), ((14, 1 << 25), SHAPE), ((4, None), SHAPE),                        # one token per request: T = B, max_q = 1
        ((0, p + 8), ALIGN), ((1, p + 4), ALIGN), ((2, p + 2), ALIGN), ((3, p + 1), ALIGN), ((4, p + 2), ALIGN), ((6, p + 2), ALIGN), ((15, p + 16), ALIGN),
        ((16, 0), WORKSPACE)])


def test_page_operator_refusals(lib):
    buf, p = _places()
    big = 1 << 40
    o = p + 1024                      # other buffers for what is written
    #       refs table lens parents headroom refs table lens info pages  bytes L stride R N  P   MP ws bytes stream
    good = [p, p, p, p, p, o, o, o, p, p, 4352, 2, 4352 * 50, 4, 6, 50, 8, p, big, None]
    refused(lib.thi_kv4_fork, good, [
        ((0, None), NULL), ((1, None), NULL), ((2, None), NULL), ((3, None), NULL), ((5, None), NULL), ((6, None), NULL), ((7, None), NULL), ((9, None), NULL), ((17, None), NULL),
        ((5, p), SHAPE), ((6, p), SHAPE), ((7, p), SHAPE), ((10, 0), SHAPE), ((10, 4360), SHAPE), ((11, 0), SHAPE), ((12, 4352 * 49), SHAPE), ((12, 4352 * 50 + 8), SHAPE), ((13, 0), SHAPE),
        ((14, -1), SHAPE), ((15, 0), SHAPE), ((16, 0), SHAPE), ((16, 1 << 25), SHAPE),
        ((0, p + 2), ALIGN), ((3, p + 1), ALIGN), ((4, p + 2), ALIGN), ((8, p + 2), ALIGN), ((9, p + 8), ALIGN), ((17, p + 64), ALIGN), ((18, 255), WORKSPACE)])
    #       refs table refs table info pages bytes L stride R P MP ws bytes stream
    good = [p, p, o, o, p, p, 4352, 2, 4352 * 50, 4, 50, 8, p, big, None]
    refused(lib.thi_kv4_compact, good, [
        ((0, None), NULL), ((1, None), NULL), ((2, None), NULL), ((3, None), NULL), ((5, None), NULL), ((12, None), NULL), ((2, p), SHAPE), ((3, p), SHAPE),
        ((6, 8), SHAPE), ((7, 0), SHAPE), ((8, 16), SHAPE), ((9, 0), SHAPE), ((10, 0), SHAPE), ((11, 0), SHAPE), ((1, p + 2), ALIGN), ((5, p + 4), ALIGN), ((12, p + 8), ALIGN), ((13, 16), WORKSPACE)])


def test_sizes(lib):
    assert lib.thi_kv4_page_bytes(8, 128) == 8 * 68 * 128 and lib.thi_kv4_page_bytes(3, 64) == 3 * 68 * 64
    assert lib.thi_kv4_page_bytes(8, 96) == 0 and lib.thi_kv4_page_bytes(0, 64) == 0
    f = lib.thi_kv4_attention_workspace_bytes
    assert f(2, 2, 8, 2, 128, 1, 100) > 0 and f(2, 2, 8, 2, 128, 1, 100) % 256 == 0
    assert f(2, 2, 8, 3, 128, 1, 100) == 0 and f(2, 2, 8, 2, 100, 1, 100) == 0 and f(2, 2, 8, 2, 128, 3, 100) == 0 and f(0, 2, 8, 2, 128, 1, 100) == 0
    f = lib.thi_kv4_pages_workspace_bytes
    assert f(4, 4, 8, 1000) >= 4 * 1000 and f(4, 4, 8, 0) == 0 and f(0, 4, 8, 10) == 0 and f(4, 4, 8, 1 << 25) == 0


def test_reference_codes():
    """The plain implementation itself: round trip of grid values, ties to the even code, the scale's borders, what is not finite."""
    x = np.zeros(32)
    x[:8] = ref.GRID
    x[8:16] = -ref.GRID
    x[16:23] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]
    codes, byte, vals = ref.quantise(x)
    assert byte[0] == 127 and (vals[:16] == x[:16]).all() and vals[16:23].tolist() == [0, 1, 1, 2, 2, 4, 4]
    assert codes[9] == 9 and codes[8] == 8
    for big, e in ((7.0, 0), (7.0000001, 1), (3.5, -1), (3.50001, 0), (0.0, -23), (2.0 ** -24, -23), (57344.0, 13), (65504.0, 13)):
        assert ref.block_exponent(big) == e, big
    assert np.isnan(ref.quantise(np.r_[np.inf, np.zeros(31)])[2]).all()
    rng = np.random.default_rng(1)
    pages = rng.integers(0, 256, (3, 2, 68 * 64), dtype=np.uint8)
    before = pages.copy()
    k, v = rng.standard_normal((2, 64)), rng.standard_normal((2, 64))
    ref.store(pages, 64 + 37, k, v)
    k2, v2 = ref.load(pages, 64 + 37)
    assert (k2 == ref.quantise(k)[2]).all() and (v2 == ref.quantise(v)[2]).all()
    assert (pages[0] == before[0]).all() and (pages[2] == before[2]).all()
    assert (pages[1] != before[1]).sum(-1).max() <= 64 + 4            # 32 bytes of codes and 2 scales each of key and value


def test_reference_layout_covers_a_page():
    """Every byte of a head's block belongs to exactly one position and pair of columns, or position and block."""
    for D in (64, 128):
        seen = np.zeros(68 * D, int)
        for pos in range(64):
            key, ks, value, vs = ref.places(pos, D)
            for at in (key[0::2], value[0::2], ks[0::32], vs[0::32]):
                seen[at] += 1
        assert (seen == 1).all()


@pytest.mark.skipif(shutil.which(HIPCC) is None, reason="hipcc not found")
def test_host_side_under_sanitizers(tmp_path):
    """kv4_api.hip's checks and launch arithmetic over odd and extreme arguments, built with address and undefined-behaviour sanitizers; the
    launchers are stand-ins that check what the kernels assume."""
    driver = tmp_path / "driver.cpp"
    driver.write_text(r'''
#include "%(root)s/include/thi.h"
#include "%(root)s/paper_2605_25655_amd/csrc/kv4.h"
#include <cstdio>
#include <cstdlib>
namespace thi {
static long launches = 0;
#define NEED(x) do { ++launches; if (!(x)) { std::printf("stand-in %%s\n", #x); std::exit(1); } } while (0)
hipError_t launch_kv4_append(const Kv4AppendArgs& a, int, hipStream_t) { NEED(a.ld >= (a.Hq + 2L * a.Hkv) * a.D && a.T >= 1); return hipSuccess; }
hipError_t launch_kv4_read(const Kv4ReadArgs& a, hipStream_t) { NEED(a.T >= 1 && (a.k_out || a.v_out)); return hipSuccess; }
hipError_t launch_kv4_fork(const PagesArgs& a, int, hipStream_t) { NEED(a.ws && a.refs_in != a.refs_out); return hipSuccess; }
hipError_t launch_kv4_compact(const PagesArgs& a, int, hipStream_t) { NEED(a.ws && a.refs_in != a.refs_out); return hipSuccess; }
size_t pages_workspace_words(int r, int n, int p) { return 64 + (size_t)r + n + 3 * (size_t)p; }
%(extra)s
}
int main()
{
    static char buf[8192];
    char* const p = (char*)(((size_t)buf + 255) / 256 * 256);
    const int* const w = (const int*)p;
    int* const o = (int*)(p + 1024);
    const int extents[] = {-2147483647 - 1, -1, 0, 1, 2, 5, 64, 65535, 65536, 33554431, 33554432, 2147483647};
    const size_t bytes[] = {0, 16, 4352, (size_t)1 << 40, (size_t)-1, (size_t)-16};
    long calls = 0;
    for (int x : extents)
        for (int y : extents) {
            for (int D : {64, 128, 96, 0}) {
                thi_kv4_page_bytes(x, D);
                thi_qk_norm_rope_kv4(p, y, p, p, 1e-6f, w, (const float*)p, w, p, p, x, 4, 2, D, 7, nullptr);
                thi_qk_norm_rope_kv4(p, 2147483640, p, p, 1e-6f, w, (const float*)p, w, p, p, 3, x, y, D, 7, nullptr);
                thi_kv4_read(p, w, p, p, x, y, D, 7, nullptr);
                thi_kv4_read(p, w, p, p, 5, 2, D, x, nullptr);
                for (int z : extents) {
                    thi_kv4_attention_workspace_bytes(x, y, 8, 2, D, z, 9);
                    thi_kv4_attention(p, p, w, w, w, 0.1f, p, x, y, 8, 2, D, z, 7, 9, p, (size_t)1 << 50, nullptr);
                    thi_kv4_attention(p, p, w, w, w, 0.1f, p, 3, 9, x, y, D, 4, 7, z, p, (size_t)1 << 50, nullptr);
                    calls += 3;
                }
            }
            for (int z : extents) {
                thi_kv4_pages_workspace_bytes(x, y, z, 50);
                for (size_t b : bytes) {
                    thi_kv4_fork(w, w, w, w, w, o, o, o, o, p, b, 2, (size_t)1 << 41, x, y, 50, z, p, (size_t)1 << 50, nullptr);
                    thi_kv4_fork(w, w, w, w, w, o, o, o, o, p, 4352, x, b, 4, 6, y, z, p, (size_t)1 << 50, nullptr);
                    thi_kv4_compact(w, w, o, o, o, p, b, x, (size_t)1 << 41, y, z, 8, p, (size_t)1 << 50, nullptr);
                    calls += 3;
                }
            }
        }
    std::printf("ok %%ld calls, %%ld launches\n", calls, thi::launches);
    return thi::launches > 100 ? 0 : 1;
}
''' % dict(root=ROOT, extra=ATTENTION_STAND_INS))
    exe = str(tmp_path / "kv4_san")
    csrc = os.path.join(ROOT, "paper_2605_25655_amd", "csrc")
    res = subprocess.run([HIPCC, "-O1", "-g", "-std=c++17", "--offload-arch=gfx950", "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
                          "-Xarch_host", "-fno-omit-frame-pointer", "-Wno-unused-command-line-argument", "-o", exe, os.path.join(csrc, "kv4_api.hip"),
                          "-x", "hip", str(driver)], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-6000:]
    env = dict(os.environ, ASAN_OPTIONS="verify_asan_link_order=0:detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    res = subprocess.run([exe], env=env, capture_output=True, text=True)
    assert res.returncode == 0 and res.stdout.startswith("ok "), res.stdout[-1000:] + res.stderr[-4000:]
    assert "runtime error" not in res.stderr and "AddressSanitizer" not in res.stderr, res.stderr[-4000:]


ATTENTION_STAND_INS = "hipError_t launch_kv4_attention(const Kv4AttnArgs& a, hipStream_t) { NEED(a.B >= 1 && a.T >= 1 && a.max_q >= 1 && a.max_q <= a.T); return hipSuccess; }"
