"""The 4-bit cache's store and read-back at their edges: infinities under the norm, special values in every way a value takes into a page, the one rounding of a query, and calls of
many tokens, which store and give what calls of few do."""
import numpy as np
import pytest

from tests.gpu_common import say
from tests.test_kv4_gpu import PAGE, append_case, check_append, dev, host, thi  # noqa: F401

pytestmark = pytest.mark.gpu


def _special(T, Hkv, D, seed):
    """Rows of zeros, fp16's smallest and largest numbers, the borders of scales and codes, infinities and NaN, each many times among ordinary rows."""
    c = append_case(seed, T, 2, Hkv, D, -(-T // PAGE) + 3)
    x = c["qkv"].reshape(T, 2 + 2 * Hkv, D)
    for t in range(0, T, 2):
        what = t // 2 % 9
        if what == 0:
            x[t] = 0
        elif what == 1:
            x[t] = np.float16(2.0 ** -24)
        elif what == 2:
            x[t], x[t, :, ::3] = np.float16(65504), np.float16(-40000)
        elif what == 3:
            x[t] = np.tile(np.float16([7, 0.25, -0.75, 1.25, 1.75, -2.5, 3.5, 5]), (len(x[t]), D // 8))
        elif what == 4:
            x[t] = np.tile(np.float16([7.004, 0.5, -1.5, 2.5, 3.5, -5, 7, 6]), (len(x[t]), D // 8))
        elif what == 5:
            x[t, :, 5] = np.inf
        elif what == 6:
            x[t, :, D - 26] = -np.inf
        elif what == 7:
            x[t, :, D - 1] = np.nan
        else:
            x[t] = np.tile(np.float16([6e-8, -1.2e-7, 4e-7, 3.6e-7, 8.4e-7, 0, -0.0, 1e-6]), (len(x[t]), D // 8))
    return c


def _slots(kind, T):
    if kind == "aligned":
        return 8 + np.arange(T)
    if kind == "unaligned":
        return 5 + np.arange(T)
    s = 64 + np.arange(T)                                             # with padding rows in between
    s[[T // 3, T // 3 + 1, T // 2]] = -1
    return s


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kind,T", [("aligned", 18), ("aligned", 150), ("unaligned", 150), ("padded", 150)])
@pytest.mark.parametrize("norm,rope", [(True, True), (True, False), (False, False)])
def test_special_values(thi, kind, T, D, norm, rope):  # noqa: F811
    c = _special(T, 2, D, T + D)
    c["slots"] = _slots(kind, T).astype(np.int32)
    if not norm:
        c["q_gamma"] = c["k_gamma"] = None
    if not rope:
        c["theta"] = c["positions"] = None
    with np.errstate(invalid="ignore"):
        check_append(thi, c, 2, 2, D)


def _many_slots(kind, T, rng):
    if kind == "scattered":
        return rng.permutation(T + 2 * PAGE)[:T]
    if kind == "prompts":                                             # runs of odd lengths that begin anywhere, one of them backwards, in pages of random order
        page, slots = list(rng.permutation(T // PAGE + 40)), []
        while len(slots) < T:
            n, at = int(rng.integers(1, 200)), int(rng.integers(0, PAGE))
            pages = [page.pop() for _ in range((at + n + PAGE - 1) // PAGE)]
            run = [int(pages[(at + i) // PAGE]) * PAGE + (at + i) % PAGE for i in range(n)]
            slots += run if n % 7 else run[::-1]
            if len(page) < 5:
                page = list(rng.permutation(T // PAGE + 40) + (T // PAGE + 40) * (1 + max(slots) // PAGE // (T // PAGE + 40)))
        return np.array(slots[:T])
    return _slots(kind, T)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kind", ["aligned", "unaligned", "padded", "scattered", "prompts"])
@pytest.mark.parametrize("norm", [True, False])
def test_many_tokens_store_what_few_do(thi, kind, D, norm):  # noqa: F811
    """One call of rows of more than 8 MB against calls of 61 tokens, bit for bit: four rows that exchange bytes inside a wave, LDS where they are no whole runs, special
    values among them."""
    import torch
    Hq, Hkv, T = 10, 5, 1701 if D == 128 else 3303
    rng = np.random.default_rng(D + len(kind))
    c = _special(149, 9, D, 3)                                        # 20 heads a row
    qkv = dev(np.tile(c["qkv"], (-(-T // 149), 1))[:T])
    assert qkv.numel() * 2 > 8.2e6
    slots = _many_slots(kind, T, rng)
    P = int(slots.max()) // PAGE + 2
    assert len(set(slots[slots >= 0].tolist())) == (slots >= 0).sum()
    slots, positions, theta = dev(slots.astype(np.int32)), dev(rng.integers(0, 100000, T).astype(np.int32)), dev(c["theta"])
    g = dev(c["q_gamma"]) if norm else None
    say(f"[case] many tokens {kind} D={D} T={T} norm={norm}")
    start = torch.randint(0, 256, (P, Hkv, 68 * D), dtype=torch.uint8, device="cuda")
    got = []
    for piece in (T, 61):
        pages, q = start.clone(), torch.full((T, Hq, D), 7.0, dtype=torch.float16, device="cuda")
        for a in range(0, T, piece):
            e = min(a + piece, T)
            thi.thi_qk_norm_rope_kv4(qkv[a:e], g, g, 1e-6, positions[a:e].clone(), theta, slots[a:e].clone(), q[a:e], pages)
        got.append((pages, q))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1].view(torch.int16), got[1][1].view(torch.int16))
    assert not torch.equal(got[0][0], start)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kind", ["aligned", "unaligned", "padded", "scattered", "prompts"])
def test_many_tokens_read_what_few_do(thi, kind, D):  # noqa: F811
    """One call of keys of more than 4 MB (four tokens a thread) against calls of 61 tokens, bit for bit."""
    import torch
    Hkv, T = 24, 811 if D == 128 else 1499
    rng = np.random.default_rng(D + len(kind))
    slots = _many_slots(kind, T, rng)
    P = int(slots.max()) // PAGE + 1
    slots[T // 2 + 40] = P * PAGE                                     # no page
    pages = torch.randint(0, 256, (P, Hkv, 68 * D), dtype=torch.uint8, device="cuda")
    assert T * Hkv * D * 2 > 4.1e6
    say(f"[case] read {kind} D={D} T={T}")
    slots, got = dev(slots.astype(np.int32)), []
    for piece in (T, 61):
        k, v = (torch.full((T, Hkv, D), 7.0, dtype=torch.float16, device="cuda") for _ in range(2))
        for a in range(0, T, piece):
            e = min(a + piece, T)
            thi.thi_kv4_read(pages, slots[a:e].clone(), k[a:e], v[a:e])
        got.append((k, v))
    for x, y in zip(*got):
        assert torch.equal(x.view(torch.int16), y.view(torch.int16))


@pytest.mark.parametrize("T", [1, 150])
@pytest.mark.parametrize("size,step", [(1.0, 2.0 ** -10), (2.0 ** -16, 2.0 ** -8)])
def test_queries_are_rounded_once(thi, T, size, step):  # noqa: F811
    """Rotated queries a little beside the middle between two fp16 numbers (also of those with fewer bits), on the side on which a rounding to 32 bits first (to the
    middle, then to the even one) would end on the wrong one."""
    import torch
    D = 64
    k = np.arange(D // 2)
    middle = 1 + (2 * k + 1) * step / 2
    beside = np.where(k % 2 == 0, 2.0 ** -25, -2.0 ** -25)
    theta = (np.arcsin((middle + beside) / np.sqrt(2)) - np.pi / 4).astype(np.float32)
    exact = np.cos(theta.astype(np.float64)) + np.sin(theta.astype(np.float64))
    assert (np.abs(exact - middle) < 2.0 ** -24).all() and (np.abs(exact - middle) > 2.0 ** -30).all() and (np.sign(exact - middle) == np.sign(beside)).all()
    want = (size * exact).astype(np.float16)
    assert (want != (size * exact).astype(np.float32).astype(np.float16)).all()
    qkv = np.tile(np.float16([size, -size]), (T, 3 * D // 2))
    q_out = torch.empty(T, 1, D, dtype=torch.float16, device="cuda")
    pages = torch.zeros(4, 1, 68 * D, dtype=torch.uint8, device="cuda")
    say(f"[case] one rounding T={T} size={size}")
    thi.thi_qk_norm_rope_kv4(dev(qkv), None, None, 1e-6, torch.ones(T, dtype=torch.int32, device="cuda"), dev(theta), torch.arange(T, dtype=torch.int32, device="cuda"), q_out, pages)
    got = host(q_out)
    assert (got[:, 0, 0::2] == want).all()
