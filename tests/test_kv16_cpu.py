"""The fp16 cache on the CPU: refusals and workspace sizes of the C ABI (no launch), the host code under sanitizers, and the plain
implementation that the GPU tests compare with."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

from tests import kv16_reference as ref

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
    refused(lib.thi_qk_norm_rope_kv16, good, [
        ((0, None), NULL), ((7, None), NULL), ((8, None), NULL), ((9, None), NULL), ((5, None), NULL),      # theta without positions
        ((10, 0), SHAPE), ((10, -1), SHAPE), ((10, (1 << 28) + 1), SHAPE), ((11, 3), SHAPE), ((11, 0), SHAPE), ((12, 0), SHAPE), ((12, -2), SHAPE), ((13, 96), SHAPE), ((13, 256), SHAPE),
        ((1, 1016), SHAPE), ((1, 1028), SHAPE), ((14, 0), SHAPE), ((14, (1 << 25)), SHAPE),
        ((0, p + 8), ALIGN), ((2, p + 2), ALIGN), ((3, p + 4), ALIGN), ((5, p + 2), ALIGN), ((6, p + 1), ALIGN), ((7, p + 2), ALIGN), ((8, p + 8), ALIGN), ((9, p + 8), ALIGN)])


def test_attention_refusals(lib):
    buf, p = _places()
    big = 1 << 40
    #       0  1  2  3  4  5    6  7  8  9  10 11 12 13 14 15   16 17 18 19 20   21
    good = [p, p, p, p, p, 0.1, 5, 1, p, p, p, 2, 5, 8, 2, 128, 4, 9, 3, p, big, None]
    refused(lib.thi_kv16_attention, [*good[:18], (1 << 22) + 1, *good[19:]], [((10, p), SHAPE)])      # (of two cache heads, with weights)
    refused(lib.thi_kv16_attention, good, [
        ((0, None), NULL), ((1, None), NULL), ((2, None), NULL), ((3, None), NULL), ((8, None), NULL), ((10, None), NULL), ((19, None), NULL),
        ((6, -1), SHAPE), ((7, -1), SHAPE),
        ((11, 0), SHAPE), ((11, 65536), SHAPE), ((12, 0), SHAPE), ((13, 7), SHAPE), ((14, 3), SHAPE), ((15, 80), SHAPE), ((16, 0), SHAPE), ((16, 6), SHAPE), ((17, 0), SHAPE),
        ((17, 1 << 25), SHAPE), ((18, 0), SHAPE), ((18, (1 << 24) + 1), SHAPE), ((4, None), SHAPE),      # one token per request: T = B, max_q = 1
        ((0, p + 8), ALIGN), ((1, p + 4), ALIGN), ((2, p + 2), ALIGN), ((3, p + 1), ALIGN), ((4, p + 2), ALIGN), ((8, p + 2), ALIGN), ((9, p + 2), ALIGN), ((10, p + 1), ALIGN),
        ((19, p + 16), ALIGN), ((20, 0), WORKSPACE), ((20, 511), WORKSPACE)])


def test_evict_refusals(lib):
    buf, p = _places()
    big, o = 1 << 40, p + 1024
    stride = 2 * 256 * 64 * 50
    #       refs table lens w  budget sinks recent head refs table lens w info pages stride  L  R  Hkv D  P  MP  ws bytes stream
    good = [p, p, p, p, 100, 4, 96, 0, o, o, o, o, p, p, stride, 2, 4, 2, 64, 50, 8, p, big, None]
    refused(lib.thi_kv16_evict, [*good[:4], (1 << 28) + 1, *good[5:17], 1, *good[18:20], 1 << 23, *good[21:]], [((12, p), SHAPE)])
    refused(lib.thi_kv16_evict, good, [
        *(((i, None), NULL) for i in (0, 1, 2, 3, 8, 9, 10, 11, 13, 21)),
        ((4, 0), SHAPE), ((4, 99), SHAPE), ((5, -1), SHAPE), ((6, -1), SHAPE), ((6, 97), SHAPE), ((6, 2147483647), SHAPE), ((7, -1), SHAPE),
        ((8, p), SHAPE), ((9, p), SHAPE), ((10, p), SHAPE), ((11, p), SHAPE), ((14, stride - 16), SHAPE), ((14, stride + 8), SHAPE), ((15, 0), SHAPE), ((15, 16384), SHAPE), ((16, 0), SHAPE),
        ((17, 0), SHAPE), ((18, 80), SHAPE), ((19, 0), SHAPE), ((19, 1 << 25), SHAPE), ((20, 0), SHAPE), ((20, (1 << 24) + 1), SHAPE),
        *(((i, p + 2049), ALIGN) for i in (0, 1, 2, 3, 8, 9, 10, 11, 12)), ((13, p + 8), ALIGN), ((21, p + 128), ALIGN), ((22, 1000), WORKSPACE)])


def test_sizes(lib):
    assert lib.thi_kv16_page_bytes(8, 128) == 8 * 256 * 128 and lib.thi_kv16_page_bytes(3, 64) == 3 * 256 * 64
    assert lib.thi_kv16_page_bytes(8, 96) == 0 and lib.thi_kv16_page_bytes(0, 64) == 0
    f = lib.thi_kv16_attention_workspace_bytes
    assert f(2, 2, 8, 2, 128, 1, 100, 0) > 0 and f(2, 2, 8, 2, 128, 1, 100, 0) % 256 == 0 and f(2, 2, 8, 2, 128, 1, 100, 1) > f(2, 2, 8, 2, 128, 1, 100, 0)
    assert f(2, 2, 8, 8, 128, 1, 1 << 20, 1) > 0 and f(2, 2, 8, 8, 128, 1, (1 << 20) + 1, 1) == 0 and f(2, 2, 8, 8, 128, 1, (1 << 20) + 1, 0) > 0
    assert f(1, 60000, 17920, 1, 128, 59918, 1, 0) > 0 and f(1, 60000, 17920, 1, 128, 59919, 1, 0) == 0      # 2^23 tiles of 128 rows, and one more
    assert f(2, 2, 8, 3, 128, 1, 100, 0) == 0 and f(2, 2, 8, 2, 100, 1, 100, 0) == 0 and f(2, 2, 8, 2, 128, 3, 100, 0) == 0 and f(0, 2, 8, 2, 128, 1, 100, 0) == 0
    f = lib.thi_kv16_evict_workspace_bytes
    assert f(1, 128, 8, 1 << 24, 10) == 0 and f(1, 127, 8, 1 << 24, 10) > 0
    assert f(2, 4, 8, 10, 1000) >= 4 * 2 * 4 * 8 * 10 * 64 and f(2, 4, 8, 10, 0) == 0 and f(0, 4, 8, 10, 10) == 0 and f(256, 256, 8, 1, 1) == 0


def test_reference_layout_covers_a_page():
    for D in (64, 128):
        seen = np.zeros(128 * D, int)
        for pos in range(64):
            for at in ref.places(pos, D):
                seen[at] += 1
        assert (seen == 1).all()


def test_reference_tolerances_notice_a_position():
    """The attention test's tolerance is smaller than what one position more, less or elsewhere changes (planted in the reference, here)."""
    rng = np.random.default_rng(0)
    c = dict(q=rng.standard_normal((3, 4, 64)).astype(np.float16) * 2, pages=rng.standard_normal((9, 2, 128 * 64)).astype(np.float16), table=np.arange(9, dtype=np.int32)[None],
             lens=np.array([500]), offsets=np.array([0, 3]))
    y, tol, w, wtol = ref.attention(c, 0.125, window=100, sinks=4)
    for window, sinks in ((99, 4), (101, 4), (100, 3), (100, 5)):
        z, _, u, _ = ref.attention(c, 0.125, window=window, sinks=sinks)
        # every row's sum changes by about a two-hundredth, the results by more than their rounding in most columns
        assert (np.abs(z - y) > 2 * tol).mean() > 0.3 and (np.abs(u - w) > 2 * wtol)[:, :, :500].mean() > 0.15


@pytest.mark.skipif(shutil.which(HIPCC) is None, reason="hipcc not found")
def test_host_side_under_sanitizers(tmp_path):
    """kv16_api.hip's checks and launch arithmetic over odd and extreme arguments, built with address and undefined-behaviour sanitizers; the
    launchers are stand-ins that check what the kernels assume: what a call takes of its workspace is there, and for every smaller call, too."""
    driver = tmp_path / "driver.cpp"
    driver.write_text(r'''
#include "%(root)s/include/thi.h"
#include "%(root)s/paper_2605_25655_amd/csrc/kv16.h"
#include <cstdio>
#include <cstdlib>
namespace thi {
static long launches = 0, both = 0;
static size_t given = (size_t)1 << 50;
static char* space;
#define NEED(x) do { ++launches; if (!(x)) { std::printf("stand-in %%s\n", #x); std::exit(1); } } while (0)
hipError_t launch_kv16_append(const Kv16AppendArgs& a, int, hipStream_t) { NEED(a.ld >= (a.Hq + 2L * a.Hkv) * a.D && a.T >= 1); return hipSuccess; }
static void look(const Kv16AttnArgs& a, long q)
{
    NEED(a.B >= 1 && a.T >= 1 && a.max_q >= 1 && a.max_q <= a.T && a.nsplit >= 1 && a.nsplit <= KV16_MAX_SPLIT && a.window >= 0 && a.sinks >= 0);
    const size_t rows = (size_t)a.B * a.Hkv * a.tiles * KV16_TILE_ROWS;
    NEED(a.tiles * (long)KV16_TILE_ROWS >= a.max_q * (long)a.group && a.part_q == q);
    NEED(a.nsplit == 1 || (char*)a.part + (size_t)a.B * q * a.Hq * a.nsplit * kv16_part(a.D) * 4 <= space + given);
    NEED((char*)a.part <= space + given);
    NEED(a.parts <= 1 || (char*)a.part + (size_t)a.parts * a.B * a.Hkv * a.max_pages * 256 <= space + given);
    NEED(!a.queries || a.whose == Kv16AttnArgs::THOSE_OF_FEW_ROWS || (a.parts >= 1 && a.part_tiles >= 1 && (long)a.parts * a.part_tiles * 16 >= (long)a.max_q * a.group));
    NEED(!a.weights_out || ((char*)a.stats == space && space + rows * 8 <= (char*)a.part));
    NEED(!a.queries || ((char*)a.queries >= space + rows * 8 && (char*)a.queries + rows * a.D * 2 <= (char*)a.part));
    NEED(!a.scores || ((char*)a.scores >= space + rows * 8 && (char*)a.scores + (size_t)a.B * a.max_q * a.Hq * a.max_pages * 256 <= (char*)a.part));
}
hipError_t launch_kv16_attention(const Kv16AttnArgs* few, const Kv16AttnArgs* many, hipStream_t)
{
    NEED(few || many);
    const Kv16AttnArgs& a = few ? *few : *many;
    const long q_few = KV16_FEW_ROWS / a.group;
    if (few) look(*few, many ? q_few : a.max_q);
    if (many) look(*many, a.max_q);
    NEED((many == nullptr) == ((long)a.max_q * a.group <= KV16_FEW_ROWS));
    NEED(few && many ? few->whose == Kv16AttnArgs::THOSE_OF_FEW_ROWS && many->whose == Kv16AttnArgs::THOSE_OF_MORE && !few->scores && few->queries == many->queries && few->tiles == many->tiles
                     : a.whose == Kv16AttnArgs::EVERYONES);
    NEED(!a.weights_out || (few && !many ? a.scores && !a.queries : a.queries && !a.scores));
    if (few && many) ++both;
    return hipSuccess;
}
size_t kv16_evict_words(int layers, int rows, int Hkv, int max_pages, int num_pages) { return 2 * (size_t)rows + num_pages + (size_t)layers * rows * Hkv * max_pages * 64; }
hipError_t launch_kv16_evict(const Kv16EvictArgs& a, hipStream_t) { NEED(a.ws && a.sinks + a.recent <= a.budget && a.layers * a.rows <= 65535); return hipSuccess; }
}
int main()
{
    static char buf[8192];
    char* const p = (char*)(((size_t)buf + 255) / 256 * 256);
    thi::space = p;
    const int* const w = (const int*)p;
    int* const o = (int*)(p + 1024);
    float* const f = (float*)(p + 2048);
    const int extents[] = {-2147483647 - 1, -1, 0, 1, 2, 5, 64, 65535, 65536, 16777216, 33554431, 33554432, 2147483647};
    long calls = 0;
    for (int x : extents)
        for (int y : extents) {
            for (int D : {64, 128, 96, 0}) {
                thi_kv16_page_bytes(x, D);
                thi_qk_norm_rope_kv16(p, y, p, p, 1e-6f, w, (const float*)p, w, p, p, x, 4, 2, D, 7, nullptr);
                thi_qk_norm_rope_kv16(p, 2147483640, p, p, 1e-6f, w, (const float*)p, w, p, p, 3, x, y, D, 7, nullptr);
                for (int z : extents) {
                    thi_kv16_attention_workspace_bytes(x, y, 8, 2, D, z, 9, 1);
                    thi_kv16_attention(p, p, w, w, w, 0.1f, 0, 0, p, f, f, x, y, 8, 2, D, z, 7, 9, p, (size_t)1 << 50, nullptr);
                    thi_kv16_attention(p, p, w, w, w, 0.1f, 1, 2, p, f, f, 3, 9, x, y, D, 4, 7, z, p, (size_t)1 << 50, nullptr);
                    thi_kv16_attention(p, p, w, w, w, 0.1f, x, y, p, nullptr, nullptr, 3, 9, 8, 2, D, 4, z, 9, p, (size_t)1 << 50, nullptr);
                    calls += 3;
                }
            }
            for (int z : extents)
                for (int v : extents) {
                    thi_kv16_evict_workspace_bytes(x, y, z, v, 50);
                    thi_kv16_evict(w, w, w, f, x, y, z, v, o, o, o, f + 1, o, p, (size_t)1 << 40, 2, 4, 2, 64, 50, 8, p, (size_t)1 << 50, nullptr);
                    thi_kv16_evict(w, w, w, f, 100, 4, 4, 0, o, o, o, f + 1, o, p, (size_t)1 << 40, x, y, z, 64, v, 8, p, (size_t)1 << 60, nullptr);
                    thi_kv16_evict(w, w, w, f, 100, 4, 4, 0, o, o, o, f + 1, o, p, (size_t)1 << 40, 1, x, 2, 64, y, z, p, (size_t)1 << 60, nullptr);
                    calls += 3;
                }
        }
    // a workspace for the largest call serves every smaller one
    const int heads[][3] = {{1, 1, 64}, {8, 8, 64}, {32, 32, 128}, {40, 8, 128}, {64, 8, 128}, {64, 1, 128}, {130, 2, 64}};
    for (auto& h : heads)
        for (int B : {1, 2, 5, 17, 300})
            for (int q : {1, 2, 7, 64, 500})
                for (int mp : {1, 3, 16, 17, 100, 3000})
                    for (int weights : {0, 1}) {
                        thi::given = thi_kv16_attention_workspace_bytes(B, B * q, h[0], h[1], h[2], q, mp, weights);
                        for (int b : {1, 2, 5, 17, 300})
                            for (int r : {1, 2, 7, 64, 500})
                                for (int m : {1, 3, 16, 17, 100, 3000})
                                    for (int t : {b * r, (b - 1) * r + 1})
                                    if (b <= B && r <= q && m <= mp && t >= r) {
                                        const int rc = thi_kv16_attention(p, p, w, w, w, 0.1f, 0, 0, p, nullptr, weights ? f : nullptr, b, t, h[0], h[1], h[2], r, 7, m, p, thi::given, nullptr);
                                        if (rc != 0) { std::printf("%%d for %%d %%d %%d in %%d %%d %%d\n", rc, b, r, m, B, q, mp); return 1; }
                                    }
                    }
    std::printf("ok %%ld calls, %%ld launches\n", calls, thi::launches);
    return thi::launches > 100 && thi::both > 100 ? 0 : 1;
}
''' % dict(root=ROOT))
    exe = str(tmp_path / "kv16_san")
    csrc = os.path.join(ROOT, "paper_2605_25655_amd", "csrc")
    res = subprocess.run([HIPCC, "-O1", "-g", "-std=c++17", "--offload-arch=gfx950", "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
                          "-Xarch_host", "-fno-omit-frame-pointer", "-Wno-unused-command-line-argument", "-o", exe, os.path.join(csrc, "kv16_api.hip"),
                          "-x", "hip", str(driver)], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-6000:]
    env = dict(os.environ, ASAN_OPTIONS="verify_asan_link_order=0:detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    res = subprocess.run([exe], env=env, capture_output=True, text=True)
    assert res.returncode == 0 and res.stdout.startswith("ok "), res.stdout[-1000:] + res.stderr[-4000:]
    assert "runtime error" not in res.stderr and "AddressSanitizer" not in res.stderr, res.stderr[-4000:]


@pytest.mark.skipif(shutil.which(HIPCC) is None, reason="hipcc not found")
def test_rows_that_stay_are_copied_once_at_the_limits(tmp_path):
    """Which weights the eviction's threads copy where a row stays as it is, at the largest budgets, tables and lengths that are not refused: every step-th from the thread's own place
    on, all of them in the row, and no more; built with the undefined-behaviour sanitizer."""
    driver = tmp_path / "driver.cpp"
    driver.write_text(r'''
#include "%(root)s/paper_2605_25655_amd/csrc/kv16.h"
#include <cstdio>
#include <cstdlib>
using namespace thi;
int main()
{
    long walks = 0;
    for (int budget : {1, 64, 65, 100000, 1 << 26, (1 << 27) - 1, 1 << 27, (1 << 28) - 1, 1 << 28, 2147483647})
        for (int max_pages : {1, 2, 1000, 1 << 20, 1 << 22, (1 << 22) + 1, 1 << 24}) {
            if (budget > 1 << 28 && max_pages > 1 << 22) continue;      // refused
            const unsigned groups = kv16_move_groups(budget, max_pages);
            const long step = (long)groups * KE_MOVE, reach = (long)max_pages * KV16_PAGE;
            if (groups < 1 || (long)groups * KV16_PAGE < (budget < reach ? budget : reach) || step >= 1L << 32) { std::printf("groups %%u of %%d %%d\n", groups, budget, max_pages); return 1; }
            for (long n : {0L, 1L, 5L, 100L, 4000L, reach - 1, reach}) {
                if (n < 0 || n > reach) continue;
                for (unsigned group : {0u, 1u, groups / 2, groups - 1})
                    for (unsigned thread : {0u, 5u, KE_MOVE - 1u}) {
                        if (group >= groups) continue;
                        long next = (long)group * KE_MOVE + thread, last = -1;
                        kv16_each_copied(group, groups, thread, (int)n, [&](long p) {
                            if (p != next || p < 0 || p >= n) { std::printf("%%ld, not %%ld, of %%ld; budget %%d, %%d pages\n", p, next, n, budget, max_pages); std::exit(1); }
                            last = p;
                            next += step;
                        });
                        if (next < n || (last >= 0 && last + step < n)) { std::printf("ends at %%ld of %%ld\n", last, n); return 1; }
                        ++walks;
                    }
            }
        }
    std::printf("ok %%ld walks\n", walks);
    return 0;
}
''' % dict(root=ROOT))
    exe = str(tmp_path / "kv16_walks")
    res = subprocess.run([HIPCC, "-O1", "-g", "-std=c++17", "--offload-arch=gfx950", "-Xarch_host", "-fsanitize=undefined", "-Wno-unused-command-line-argument", "-o", exe, "-x", "hip", str(driver)],
                         capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-6000:]
    res = subprocess.run([exe], env=dict(os.environ, UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1"), capture_output=True, text=True, timeout=300)
    assert res.returncode == 0 and res.stdout.startswith("ok "), res.stdout[-1000:] + res.stderr[-4000:]
