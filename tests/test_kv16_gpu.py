"""The fp16 cache's operators on the GPU, through the binding, against the plain implementation in tests/kv16_reference.py (64 bits).

Tables, counts, moved keys, values and weights have to be equal; what is computed is held to tolerances that count its roundings (derived there)."""
import numpy as np
import pytest

from tests import kv16_reference as ref
from tests.gpu_common import say, to_dev

pytestmark = pytest.mark.gpu
PAGE = ref.PAGE


@pytest.fixture(scope="module")
def thi():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    import paper_2605_25655_amd as thi
    thi.load_library()
    return thi


def dev(a):
    import torch
    if a is None:
        return None
    a = np.ascontiguousarray(a)
    return torch.from_numpy(a).cuda() if a.dtype != np.float16 else to_dev(a)


def host(t):
    import torch
    torch.cuda.synchronize()
    return t.cpu().numpy()


# ---- norm, rotation, store ----------------------------------------------------------------------------------------


def append_case(seed, T, Hq, Hkv, D, P, far=5000):
    rng = np.random.default_rng(seed)
    qkv = (rng.standard_normal((T, (Hq + 2 * Hkv) * D)) * np.exp(rng.standard_normal((Hq + 2 * Hkv) * D))).astype(np.float16)
    return dict(qkv=qkv, q_gamma=(1 + 0.3 * rng.standard_normal(D)).astype(np.float16), k_gamma=(1 + 0.3 * rng.standard_normal(D)).astype(np.float16),
                theta=(10000.0 ** (-2 * np.arange(D // 2) / D)).astype(np.float32), positions=rng.integers(0, far, T).astype(np.int32),
                slots=rng.permutation(P * PAGE)[:T].astype(np.int32), pages=rng.standard_normal((P, Hkv, 128 * D)).astype(np.float16))


def check_append(thi, c, Hq, Hkv, D, pad=0, eps=1e-6):
    import torch
    T = len(c["slots"])
    say(f"[case] append T={T} Hq={Hq} Hkv={Hkv} D={D} pad={pad} norm={c['q_gamma'] is not None},{c['k_gamma'] is not None} rope={c['theta'] is not None}")
    qkv = np.concatenate([c["qkv"], np.full((T, pad), np.nan, np.float16)], 1) if pad else c["qkv"]
    pages = dev(c["pages"])
    q_out = torch.full((T + 1, Hq, D), float("nan"), dtype=torch.float16, device="cuda")
    thi.thi_qk_norm_rope_kv16(dev(qkv), dev(c["q_gamma"]), dev(c["k_gamma"]), eps, dev(c["positions"]), dev(c["theta"]), dev(c["slots"]), q_out[:T], pages)
    q, k, v, tq, tk = ref.append(c["qkv"], c["q_gamma"], c["k_gamma"], eps, c["positions"], c["theta"], Hq, Hkv, D)
    got = host(q_out.double())
    assert np.isnan(got[T]).all()                                   # behind the last row nothing is written

    def near(x, y, tol, what):
        fine = np.isfinite(y) & (np.abs(y) + tol < 65504)
        assert (np.abs(x - y)[fine] <= tol[fine]).all(), (what, (np.abs(x - y)[fine] / tol[fine]).max())
        assert not np.isfinite(x[~np.isfinite(y)]).any(), what

    near(got[:T], q, tq, "queries")
    after, want = host(pages.double()).reshape(c["pages"].shape), c["pages"].copy()
    for t in range(T):
        s = int(c["slots"][t])
        if not 0 <= s < len(c["pages"]) * PAGE:
            continue
        kk, vv = ref.load(after.astype(np.float64), s)
        near(kk, k[t], tk[t], f"key of token {t}")
        assert np.array_equal(vv, v[t], equal_nan=True), f"value of token {t}"
        ref.store(want, s, kk.astype(np.float16), vv.astype(np.float16))
    assert np.array_equal(after.astype(np.float16).view(np.uint16), want.view(np.uint16)), "what was not written has changed"


@pytest.mark.parametrize("T,Hq,Hkv,D", [(1, 1, 1, 64), (1, 5, 5, 128), (3, 8, 2, 128), (7, 6, 3, 64), (17, 32, 32, 128), (33, 64, 8, 64)])
def test_append(thi, T, Hq, Hkv, D):
    check_append(thi, append_case(T + Hq, T, Hq, Hkv, D, max(2, T // 8)), Hq, Hkv, D, pad=8 * (T % 3))


@pytest.mark.parametrize("missing", ["q_gamma", "k_gamma", "theta", "all"])
def test_append_without_norm_or_rotation(thi, missing):
    for T in (5, 400):
        c = append_case(3, T, 16, 16, 128, 8)
        for name in ("q_gamma", "k_gamma", "theta") if missing == "all" else (missing,):
            c[name] = None
        if c["theta"] is None:
            c["positions"] = None
        check_append(thi, c, 16, 16, 128)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("first", [0, 1, 2, 3, 61])
def test_append_runs_of_slots(thi, D, first):
    """Many tokens (the variant that stores four positions at once), in one run that begins anywhere in a page, then with the run broken, reversed and interleaved."""
    Hq, Hkv, T = 20, 20, 600 if D == 128 else 1100
    c = append_case(first, T, Hq, Hkv, D, T // PAGE + 3)
    c["slots"] = (first + np.arange(T)).astype(np.int32)
    check_append(thi, c, Hq, Hkv, D)
    if first < 2:
        order = np.arange(T)
        order[100:200] = order[100:200][::-1]
        order[301:401:2], order[302:402:2] = order[302:402:2].copy(), order[301:401:2].copy()
        c["slots"] = (first + order).astype(np.int32)
        check_append(thi, c, Hq, Hkv, D)
        c["slots"][[0, 5, 6, 77, T - 1]] = [-1, len(c["pages"]) * PAGE, 2 ** 31 - 1, -2 ** 31, -7]
        check_append(thi, c, Hq, Hkv, D)


def test_append_scattered_slots(thi):
    check_append(thi, append_case(9, 500, 24, 24, 128, 9), 24, 24, 128, pad=16)


def test_append_slots_outside_the_pool(thi):
    c = append_case(5, 6, 4, 2, 64, 2)
    c["slots"][[0, 2, 5]] = [-1, 2 * PAGE, 2 ** 31 - 1]
    check_append(thi, c, 4, 2, 64)


@pytest.mark.parametrize("far", [131072, 2 ** 24, 2 ** 31 - 1])
def test_append_far_positions(thi, far):
    c = append_case(6, 9, 4, 2, 128, 2)
    c["positions"] = (far - 1 - np.arange(9)).astype(np.int32)
    check_append(thi, c, 4, 2, 128)
    c["positions"] = -c["positions"]
    check_append(thi, c, 4, 2, 128)


def test_append_special_values(thi):
    """Infinities and NaN stay in their own row and head; zeros with eps; subnormal and largest values as they are."""
    c = append_case(7, 8, 4, 2, 64, 2)
    x = c["qkv"].reshape(8, -1, 64)
    x[0, 0, 3], x[1, 4, 5], x[2, 6, 7], x[3, 5, 0] = np.inf, np.nan, np.inf, -np.inf
    x[4], x[5, :, :], x[6] = 0, 2.0 ** -24, 65504
    check_append(thi, c, 4, 2, 64)


# ---- attention ----------------------------------------------------------------------------------------------------


def attention_case(seed, Hq, Hkv, D, lens, new, extra=2):
    """Pages in random order, NaN in every position behind a request's last one and in the pages that nobody has."""
    rng = np.random.default_rng(seed)
    B, MP = len(lens), max(1, max(-(-n // PAGE) for n in lens)) + 1
    need = [-(-n // PAGE) for n in lens]
    P = sum(need) + extra
    order, table, at = rng.permutation(P), np.full((B, MP), -1, np.int32), 0
    pages = np.full((P, Hkv, 128 * D), np.nan, np.float16)
    for b, n in enumerate(lens):
        table[b, : need[b]] = order[at: at + need[b]]
        at += need[b]
        for p in range(n):
            ref.store(pages, int(table[b, p // PAGE]) * PAGE + p % PAGE, rng.standard_normal((Hkv, D)) * np.exp(0.5 * rng.standard_normal((Hkv, D))), rng.standard_normal((Hkv, D)))
    T = sum(new)
    return dict(q=(2 * rng.standard_normal((T, Hq, D))).astype(np.float16), pages=pages, table=table, lens=np.array(lens, np.int32),
                offsets=np.concatenate([[0], np.cumsum(new)]).astype(np.int32), max_q=max(new))


def run_attention(thi, c, scale, window=0, sinks=0, decode=False, weights=False, weights_in=None, max_q=None, ws_extra=0):
    import torch
    T, Hq, D = c["q"].shape
    B, MP = c["table"].shape
    Hkv, max_q = c["pages"].shape[1], max_q or c["max_q"]
    out = torch.full((T + 1, Hq, D), float("nan"), dtype=torch.float16, device="cuda")
    w = torch.full((B, Hkv, MP * PAGE), float("nan"), device="cuda") if weights else None
    ws = thi.Workspace(thi.thi_kv16_attention_workspace_bytes(B, T, Hq, Hkv, D, max_q, MP, weights), init=False)
    say(f"[case] attention T={T} Hq={Hq} Hkv={Hkv} D={D} lens={c['lens'].tolist()[:8]} max_q={max_q} window={window},{sinks} weights={weights}")
    thi.thi_kv16_attention(dev(c["q"]), dev(c["pages"]), dev(c["table"]), dev(c["lens"]), None if decode else dev(c["offsets"]), scale, window, sinks, out[:T], max_q, ws,
                           dev(weights_in), w)
    assert np.isnan(host(out[T].float())).all()
    return host(out[:T].double()), host(w.double()) if weights else None


def one_or_two(c):
    # (past 16 rows, weights are cut by (1 - d) with 0 <= d <= 2^-10: as one of 2^-11 around a mean of 2^-11, and what all have in common the sum cancels)
    group = c["q"].shape[1] // c["pages"].shape[1]
    return ref.TWO_SUMMANDS if c["max_q"] * group <= 16 else ref.ONE_SUMMAND


def check_attention(thi, c, window=0, sinks=0, decode=False, weights=False, weights_in=None, scale=None):
    scale = c["q"].shape[2] ** -0.5 if scale is None else scale
    got, w = run_attention(thi, c, scale, window, sinks, decode, weights or weights_in is not None, weights_in)
    y, tol, u, utol = ref.attention(c, scale, window, sinks, one_or_two(c), weights_in)
    assert (np.abs(got - y) <= tol).all(), (np.abs(got - y) / tol).max()
    if w is not None:
        assert np.array_equal(np.isnan(w), np.isnan(u))             # exactly the positions of a request are written
        fine = ~np.isnan(u)
        assert (np.abs(w - u)[fine] <= utol[fine]).all(), (np.abs(w - u)[fine] / utol[fine]).max()
    return got


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (4, 4), (8, 4), (6, 2), (8, 1), (16, 1), (20, 1), (34, 2)])
def test_decode_heads(thi, D, Hq, Hkv):
    """One token per request, every kind of group (one head, odd, more than a matrix tile holds); empty and one-position requests."""
    c = attention_case(Hq * 10 + D, Hq, Hkv, D, [130, 0, 1, 64], [1, 1, 1, 1])
    check_attention(thi, c, decode=True, weights=True)


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 255, 257, 511, 513, 1025])
def test_decode_lengths(thi, n):
    check_attention(thi, attention_case(n, 4, 1, 128, [n], [1]), decode=True)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (2, 4), (31, 0), (32, 0), (33, 4), (63, 64), (64, 1), (65, 70), (100, 128), (129, 0), (300, 4), (2 ** 31 - 1, 4), (40, 2 ** 31 - 1)])
def test_decode_windows(thi, window, sinks):
    """Windows that end inside and at the borders of pages, sinks below, at and past a page, both longer than the request."""
    c = attention_case(window % 97, 4, 2, 64, [400, 129, 3, 0, 64], [1] * 5)
    check_attention(thi, c, window, sinks, decode=True, weights=True)


@pytest.mark.parametrize("Hq,Hkv,D,n,new", [(64, 8, 128, 7020, 94), (16, 1, 64, 9000, 260), (64, 8, 128, 1300, 3), (8, 8, 64, 3000, 150)])
def test_many_rows_in_many_chunks(thi, Hq, Hkv, D, n, new):
    """New tokens of one long request, which is cut, against the same tokens as requests of their own, one each.  Off by a rounding each, and by one of the weights (2^-11 of them, times a value's
    distance to the mean, which is at most twice the largest)."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(n)
    P = -(-n // PAGE)
    pages = torch.randn(P, Hkv, 128 * D, generator=g, device="cuda").half()
    q = (torch.randn(new, Hq, D, generator=g, device="cuda") * 3).half()
    table = torch.randperm(P, generator=g, device="cuda").int()[None].contiguous()
    one, each = torch.empty_like(q), torch.empty_like(q)
    w = torch.zeros(1, Hkv, P * PAGE, device="cuda")
    ws = thi.Workspace(max(thi.thi_kv16_attention_workspace_bytes(1, new, Hq, Hkv, D, new, P, True), thi.thi_kv16_attention_workspace_bytes(new, new, Hq, Hkv, D, 1, P, False)), init=False)
    thi.thi_kv16_attention(q, pages, table, dev(np.array([n], np.int32)), dev(np.array([0, new], np.int32)), D ** -0.5, 0, 0, one, new, ws, None, w)
    thi.thi_kv16_attention(q, pages, table.repeat(new, 1), dev(np.arange(n - new + 1, n + 1, dtype=np.int32)), None, D ** -0.5, 0, 0, each, 1, ws)
    a, b, v = host(one.double()), host(each.double()), float(pages[..., 64 * D:].abs().max())
    assert (np.abs(a - b) <= 2.0 ** -10 * np.maximum(np.abs(a), np.abs(b)) + 2.0 ** -10 * v + 2.0 ** -20).all(), np.abs(a - b).max()
    rows = new * Hq // Hkv                                          # every row's weights are one in all, but for sums of n and of all rows in 32 bits
    assert np.abs(host(w.double()).sum(-1) - rows).max() <= rows * (n + rows + 128) * 2.0 ** -24


@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (20, 3), (64, 64), (90, 70), (250, 1)])
@pytest.mark.parametrize("Hq,Hkv,D", [(4, 4, 128), (8, 1, 128), (5, 1, 64)])
def test_few_new_tokens(thi, window, sinks, Hq, Hkv, D):
    """Speculative tokens: several rows per request, some with as many positions as rows, some with fewer (rows that see nothing)."""
    for new in (2, 5, 17):
        c = attention_case(new * 7 + Hq, Hq, Hkv, D, [250, new, max(0, new - 2), 66], [new, new, new, 1])
        check_attention(thi, c, window, sinks, weights=True)


@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 1), (64, 0), (65, 4), (130, 70)])
@pytest.mark.parametrize("Hq,Hkv,D", [(2, 2, 128), (8, 2, 128), (3, 1, 64), (1, 1, 64)])
def test_prompts(thi, window, sinks, Hq, Hkv, D):
    """Whole prompts and chunks on a cache that is there, of odd lengths, next to a single token and a request without rows."""
    c = attention_case(Hq + D, Hq, Hkv, D, [300, 90, 64, 400, 200], [300, 1, 64, 129, 0])
    check_attention(thi, c, window, sinks, weights=True)


@pytest.mark.parametrize("Hq,Hkv,D,window,sinks", [(4, 1, 64, 0, 0), (8, 2, 128, 0, 0), (4, 4, 64, 4500, 70), (16, 1, 64, 0, 0), (17, 1, 64, 0, 0)])
def test_single_tokens_next_to_chunks_far_behind(thi, Hq, Hkv, D, window, sinks):
    """Long tables: requests of few rows of a call with larger ones are dealt as if they were alone, and their result is as near as then (17 rows are not few)."""
    c = attention_case(Hq + D, Hq, Hkv, D, [150, 4700, 0, 1, 4650, 70], [40, 1, 1, 1, 16 // min(16, Hq // Hkv), 0])
    c["table"][4, 3] = -1
    got = check_attention(thi, c, window, sinks, weights=True)
    if Hq // Hkv <= 16:
        y, tol, _, _ = ref.attention(c, D ** -0.5, window, sinks, ref.TWO_SUMMANDS)
        assert (np.abs(got - y) <= tol)[40:].all()
    without = run_attention(thi, c, D ** -0.5, window, sinks)[0]
    assert np.array_equal(without[40:], got[40:])


def test_prompt_of_one_long_request(thi):
    check_attention(thi, attention_case(17, 2, 1, 128, [700], [700]), weights=True)


def test_long_requests_next_to_short_ones(thi):
    """Requests that are cut into chunks next to ones that are not; a request's result does not depend on the others."""
    for window, sinks in ((0, 0), (900, 4)):
        c = attention_case(3, 4, 2, 64, [2200, 3, 700, 0, 1500, 64], [1] * 6)
        check_attention(thi, c, window, sinks, decode=True, weights=True)
        order = [4, 3, 0, 5, 2, 1]
        d = dict(c, q=c["q"][order], table=c["table"][order], lens=c["lens"][order])
        one, other = (run_attention(thi, x, 0.125, window, sinks, decode=True, weights=True) for x in (c, d))
        assert np.array_equal(other[0], one[0][order]) and np.array_equal(other[1], one[1][order], equal_nan=True)


def test_weights_add_to_what_was_there(thi):
    """Accumulated weights: of the positions in front of the new tokens only; in place too; and over steps they are what one call over all tokens gives."""
    import torch
    rng = np.random.default_rng(5)
    for new in (1, 3, 40):
        c = attention_case(new, 6, 2, 64, [200, 100, new], [new] * 3)
        before = rng.standard_normal((3, 2, c["table"].shape[1] * PAGE)).astype(np.float32)
        check_attention(thi, c, weights_in=before)
        check_attention(thi, c, 50, 4, weights_in=before)
        want = run_attention(thi, c, 0.1, weights=True, weights_in=before)[1]
        w = dev(before)
        ws = thi.Workspace(thi.thi_kv16_attention_workspace_bytes(3, 3 * new, 6, 2, 64, new, c["table"].shape[1], True), init=False)
        thi.thi_kv16_attention(dev(c["q"]), dev(c["pages"]), dev(c["table"]), dev(c["lens"]), dev(c["offsets"]), 0.1, 0, 0, torch.empty(3 * new, 6, 64, dtype=torch.float16, device="cuda"),
                               new, ws, w, w)
        got = host(w.double())
        written = ~np.isnan(want)
        assert np.array_equal(got[written], want[written]) and np.array_equal(got[~written].astype(np.float32), before[~written])


@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("B,n", [(64, 16700), (100, 20000)])
def test_long_requests_that_are_not_cut(thi, B, n, weights):
    """As many requests as fill the compute units, one of them long: a workgroup of four waves (of eight, with 100) walks more pages than its waves' lists hold at once, some of them missing."""
    c = attention_case(B, 8, 8, 64, [n] + [(11 * b) % 90 for b in range(1, B)], [1] * B)
    c["table"][0, [3, 127, 128, 200, 257]] = [-1, 2 ** 31 - 1, -1, -7, -1]
    check_attention(thi, c, decode=True, weights=weights)
    check_attention(thi, c, 15000, 70, decode=True, weights=weights)


@pytest.mark.parametrize("window,sinks", [(0, 0), (7000, 70)])
@pytest.mark.parametrize("Hq,Hkv,D", [(8, 8, 64), (8, 8, 128), (16, 8, 64)])
def test_many_rows_of_long_requests_that_are_not_cut(thi, Hq, Hkv, D, window, sinks):
    """Chunks of as many requests as fill the compute units, one of them far behind: a workgroup walks more pages than its list holds at once, some of them missing behind the 64th."""
    c = attention_case(Hq + D, Hq, Hkv, D, [8930] + [20 + 7 * b % 50 for b in range(1, 34)], [20] * 34)
    c["table"][0, [0, 63, 66, 130]] = [-1, -1, 2 ** 31 - 1, -1]
    check_attention(thi, c, window, sinks, weights=True)


@pytest.mark.parametrize("Hq,Hkv,D,n,new", [(64, 8, 128, 12100, 1), (64, 8, 128, 12100, 2), (8, 2, 128, 19000, 3), (8, 2, 64, 19000, 1)])
def test_requests_in_more_chunks_than_are_joined_at_once(thi, Hq, Hkv, D, n, new):
    """One long request of few rows, cut into 48 or 64 chunks, some pages and a whole chunk's missing."""
    c = attention_case(new + D, Hq, Hkv, D, [n], [new])
    c["table"][0, 100:112] = -1
    c["table"][0, 180] = -1
    check_attention(thi, c, weights=True)
    check_attention(thi, c, n - 500, 70)


@pytest.mark.parametrize("D,weights", [(64, False), (64, True), (128, True)])
def test_more_requests_than_run_at_once(thi, D, weights):
    """Cache heads of all requests that are more than three times the compute units, with a long table: workgroups of eight waves."""
    lens = [1300 if D == 64 else 700] + [(7 * b) % 150 for b in range(96)]
    check_attention(thi, attention_case(D, 8, 8, D, lens, [1] * 97), decode=True, weights=weights)
    check_attention(thi, attention_case(D + 1, 16, 8, D, lens, [1] * 97), 100, 3, decode=True, weights=weights)


@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 70)])
@pytest.mark.parametrize("D", [64, 128])
def test_weights_of_many_pages(thi, D, window, sinks):
    """Weights of more rows than a tile where pages times cache heads are more than twice the compute units, and entries that are no page."""
    c = attention_case(60 + D, 8, 8, D, [500, 64, 1, 0, 130, 20, 300, 65, 33], [150, 20, 1, 0, 17, 20, 40, 3, 33])
    c["table"][0, [1, 6]] = [-1, 2 ** 31 - 1]
    check_attention(thi, c, window, sinks, weights=True)
    d = attention_case(61 + D, 24, 8, D, [500, 64, 1, 0, 130, 20, 300, 65, 33], [50, 20, 1, 0, 17, 20, 40, 3, 33])
    check_attention(thi, d, window, sinks, weights=True)


@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 3), (130, 70)])
@pytest.mark.parametrize("Hq,Hkv,D", [(16, 2, 64), (16, 1, 128)])
def test_weights_of_rows_in_parts(thi, Hq, Hkv, D, window, sinks):
    """Weights of more rows of a cache head than one part has, next to requests of fewer, with weights from before."""
    c = attention_case(70 + D, Hq, Hkv, D, [330, 90, 64], [330 if Hkv == 2 else 200, 17, 64])
    before = np.random.default_rng(6).standard_normal((3, Hkv, c["table"].shape[1] * PAGE)).astype(np.float32)
    check_attention(thi, c, window, sinks, weights_in=before)


@pytest.mark.parametrize("new", [1, 4, 90])
def test_missing_pages(thi, new):
    """Entries that are no page (-1, past the pool, negative) are positions that are not there: at the front, in the middle, at the end, all of them."""
    c = attention_case(21, 4, 2, 128, [400, 400, 130, 400], [new] * 4)
    c["table"][0, [0, 3]] = [-1, 2 ** 31 - 1]
    c["table"][1, [1, 2, 6]] = [-5, len(c["pages"]), -2 ** 31]
    c["table"][2, :] = -1
    check_attention(thi, c, weights=True)
    check_attention(thi, c, 150, 70, weights=True)


def test_lengths_outside_the_table(thi):
    """A length past the table's reach is the table's reach; a negative one is none."""
    c = attention_case(22, 2, 2, 64, [192, 192, 100], [1, 1, 1])
    c["table"] = c["table"][:, :3].copy()
    c["lens"][:] = [2 ** 31 - 1, 193, -7]
    check_attention(thi, c, decode=True, weights=True)


def test_offsets_and_rows_past_max_q(thi):
    """Rows of a request past max_q are not written, and the others see what they see without them."""
    c = attention_case(27, 4, 2, 64, [150, 90], [7, 3])
    got, w = run_attention(thi, c, 0.125, weights=True, max_q=4)
    assert np.isnan(got[4:7]).all()
    d = dict(c, q=c["q"][[0, 1, 2, 3, 7, 8, 9]], lens=np.array([147, 90], np.int32), offsets=np.array([0, 4, 7], np.int32), max_q=4)
    want, u = run_attention(thi, d, 0.125, weights=True)
    assert np.array_equal(got[[0, 1, 2, 3, 7, 8, 9]], want) and np.array_equal(w, u, equal_nan=True)


@pytest.mark.parametrize("new,window", [(1, 0), (1, 30), (3, 0), (3, 30), (70, 0), (70, 30)])
def test_what_is_not_finite_reaches_the_rows_that_see_it(thi, new, window):
    """A NaN or an infinity among the values: in its own column of the rows that see it, and nowhere else; among the keys: the rows that see it are NaN.  The request is
    long enough to be cut, and one request's page must not show in another's result."""
    lens = [150, 150, 600]
    for where, what in (("v", np.nan), ("v", np.inf), ("v", -np.inf), ("k", np.nan)):
        c = attention_case(25, 4, 2, 128, lens, [new] * 3)
        clean, tol, u, utol = ref.attention(c, 0.1, window, 4, one_or_two(c))
        marks = [(0, 149 - new // 2), (0, 100), (2, 2), (2, 596)]
        for b, p in marks:
            slot = int(c["table"][b, p // PAGE]) * PAGE + p % PAGE
            at = ref.places(p % PAGE, 128)[where == "v"][7]
            c["pages"][slot // PAGE, 1, at] = what
        got, w = run_attention(thi, c, 0.1, window, 4, weights=True)
        for b in range(3):
            for i in range(new):
                here = lens[b] - new + i
                seen = any(x == b and p <= here and (not window or p > here - window or p < 4) for x, p in marks)
                t = b * new + i
                for h in range(4):
                    bad = np.zeros(128, bool)
                    if seen and h // 2 == 1:
                        bad[7 if where == "v" else slice(None)] = True
                    assert (np.abs(got[t, h] - clean[t, h])[~bad] <= tol[t, h][~bad]).all(), (where, what, b, i, h)
                    if bad.any():
                        assert np.isnan(got[t, h][bad]).all() if np.isnan(what) else (got[t, h][bad] == what).all(), (where, what, b, i, h)
        if where == "v":                                          # (weights do not know values)
            fine = ~np.isnan(u)
            assert (np.abs(w - u)[fine] <= utol[fine]).all()


@pytest.mark.parametrize("window", [0, 30, 100])
@pytest.mark.parametrize("new", [1, 3, 8, 70])
@pytest.mark.parametrize("what", ["key", "query", "infinite"])
def test_weights_of_rows_that_are_not_numbers(thi, what, new, window):
    """Accumulated weights next to a row whose softmax is not a number (a NaN in a key that it sees, or in its query; a score of infinity, next to one of minus infinity): NaN at the
    positions that such a row sees, and at no other -- later tokens', in front of the window, without a page, behind a longer request's cut."""
    lens, sinks = [150, 150, 1500], 4
    c = attention_case(28, 4, 2, 128, lens, [new] * 3)
    c["table"][1, 1] = -1
    if what == "infinite":
        c["q"][..., 7] = np.abs(c["q"][..., 7]) + 1
    before = np.random.default_rng(8).standard_normal((3, 2, c["table"].shape[1] * PAGE)).astype(np.float32)
    _, _, u, utol = ref.attention(c, 0.1, window, sinks, one_or_two(c), before)
    clean, tol, _, _ = ref.attention(c, 0.1, window, sinks, one_or_two(c))
    marks, queries = [], []
    if what == "key":
        marks = [(0, 149 - new // 2, np.nan), (1, 149, np.nan), (2, 1496, np.nan), (2, 2, np.nan) if new == 8 else (2, 1400, np.nan)]
    elif what == "query":
        queries = [(0, new // 2), (1, 0), (2, new - 1)]
    else:                                                         # (a position of the sinks is seen by every row, and one of them is enough)
        marks = [(b, p, x) for b in (0, 2) for p, x in ((1, np.inf), (2, -np.inf))]
    for b, p, x in marks:
        slot = int(c["table"][b, p // PAGE]) * PAGE + p % PAGE
        c["pages"][slot // PAGE, 1, ref.places(p % PAGE, 128)[0][7]] = x
    for b, i in queries:
        c["q"][b * new + i, 3, 5] = np.nan
    got, w = run_attention(thi, c, 0.1, window, sinks, weights=True, weights_in=before)
    none = np.zeros(w.shape, bool)
    for b in range(3):
        for i in range(new):
            here = lens[b] - new + i
            at = np.array([p for p in range(here + 1) if c["table"][b, p // PAGE] >= 0 and (not window or p > here - window or p < sinks)])
            for h in range(4):
                bad = (b, i) in queries and h == 3 or h // 2 == 1 and any(x == b and p in at for x, p, _ in marks)
                t = b * new + i
                if bad:
                    none[b, 1, at] = True
                    assert np.isnan(got[t, h]).all(), (b, i, h)
                else:
                    assert (np.abs(got[t, h] - clean[t, h]) <= tol[t, h]).all(), (b, i, h)
    assert none.any()
    there = ~np.isnan(u)
    assert np.array_equal(np.isnan(w), none | ~there), [np.argwhere(np.isnan(w)[b, 1] != (none | ~there)[b, 1]).ravel().tolist()[:9] for b in range(3)]
    fine = there & ~none
    assert (np.abs(w - u)[fine] <= utol[fine]).all(), (np.abs(w - u)[fine] / utol[fine]).max()


@pytest.mark.parametrize("window", [0, 100])
@pytest.mark.parametrize("new", [1, 4, 40])
def test_rows_whose_scores_are_all_minus_infinity(thi, new, window):
    """Such a row's results are zero, also where values are not finite, and it adds no weight; a row next to it whose scores are finite is what it is."""
    lens = [90, 2600]
    c = attention_case(30, 2, 1, 64, lens, [new, new])
    c["q"][:, 0, 7], c["q"][:, 1, 7] = -1, 0.5
    before = np.random.default_rng(12).standard_normal((2, 1, c["table"].shape[1] * PAGE)).astype(np.float32)
    for p in range(lens[1]):
        c["pages"][int(c["table"][1, p // PAGE]), 0, ref.places(p % PAGE, 64)[0][7]] = 0
    y, tol, u, utol = ref.attention(c, 0.125, window, 4, one_or_two(c), before)
    for p in range(lens[0]):                                      # the first request: minus infinity for one head, infinity for the other
        c["pages"][int(c["table"][0, p // PAGE]), 0, ref.places(p % PAGE, 64)[0][7]] = np.inf
    for p in range(2, lens[0], 9):
        c["pages"][int(c["table"][0, p // PAGE]), 0, ref.places(p % PAGE, 64)[1][3]] = np.nan if p % 2 else -np.inf
    got, w = run_attention(thi, c, 0.125, window, 4, weights=True, weights_in=before)
    assert (got[:new, 0] == 0).all() and np.isnan(got[:new, 1]).all()
    assert (np.abs(got - y)[new:] <= tol[new:]).all() and (np.abs(w - u)[1][~np.isnan(u[1])] <= utol[1][~np.isnan(u[1])]).all()
    c["q"][:, 1, 7] = -2                                          # now both heads
    got, w = run_attention(thi, c, 0.125, window, 4, weights=True, weights_in=before)
    assert (got[:new] == 0).all()
    front = lens[0] - new
    assert np.array_equal(w[0, 0, :front], before[0, 0, :front]) and (w[0, 0, front: lens[0]] == 0).all()


@pytest.mark.parametrize("n", [600, 1500, 5000])
@pytest.mark.parametrize("new", [1, 4, 30])
def test_infinite_score_next_to_growing_ones(thi, new, n):
    """A score of infinity early on in one query head's rows, whose softmax is not a number from there on, and in the other's, for whom it is minus infinity, scores that grow along the
    positions, so that maxima move on and on behind it: the first's outputs and all weights are NaN, the second's outputs what they are without that position."""
    c = attention_case(29, 2, 1, 64, [n], [new])
    for p in range(n):
        slot = int(c["table"][0, p // PAGE]) * PAGE + p % PAGE
        k, v = ref.load(c["pages"], slot)
        ref.store(c["pages"], slot, np.sign(c["q"][0, 1].astype(np.float64)) * p * 13 / n + 0 * k, v)
    c["q"][:, 0, 7], c["q"][:, 1, 7] = 1, -1
    place = (int(c["table"][0, 0]), 0, ref.places(5, 64)[0][7])
    c["pages"][place] = 60000                                     # (a weight of zero; and what a tolerance can count with)
    y, tol, _, _ = ref.attention(c, 0.125, 0, 0, one_or_two(c))
    c["pages"][place] = np.inf
    got, w = run_attention(thi, c, 0.125, weights=True)
    assert np.isnan(got[:, 0]).all() and np.isnan(w[0, 0, : n]).all()
    assert (np.abs(got - y)[:, 1] <= tol[:, 1]).all()


@pytest.mark.parametrize("new", [1, 30])
def test_peaked_and_large_scores(thi, new):
    """Scores far apart, growing along the positions (the maximum moves on and on), and a scale of zero and below."""
    c = attention_case(26, 2, 1, 64, [520], [new])
    for p in range(520):
        k, v = ref.load(c["pages"], int(c["table"][0, p // PAGE]) * PAGE + p % PAGE)
        ref.store(c["pages"], int(c["table"][0, p // PAGE]) * PAGE + p % PAGE, np.sign(c["q"][0, 0].astype(np.float64)) * p / 40 + 0 * k, v)
    for scale in (0.125, 1.0, -0.5, 0.0):
        check_attention(thi, c, weights=True, scale=scale)
        check_attention(thi, c, 100, 4, weights=True, scale=scale)


@pytest.mark.parametrize("new", [1, 40])
def test_pages_past_32_bits(thi, new):
    """A pool of more than 2^32 values, pages at both ends of it: reads of the attention, writes of the store."""
    import torch
    Hkv, D, P = 8, 128, 33000                                      # 131072 values a page
    pool = torch.empty(P, Hkv, 128 * D, dtype=torch.float16, device="cuda")
    c = attention_case(30, 8, Hkv, D, [150], [new])
    place = [P - 1, 0, P // 2 + 77, P - 2, 5][: len(c["pages"])]
    for i, p in enumerate(place):
        pool[p] = to_dev(c["pages"][i])
    table = np.array([[place[e] if e >= 0 else -1 for e in c["table"][0]]], np.int32)
    rng = np.random.default_rng(1)
    qkv = rng.standard_normal((1, 24 * 128)).astype(np.float16)
    slot = place[c["table"][0, 2]] * PAGE + 21                      # the last position
    q = torch.empty(1, 8, 128, dtype=torch.float16, device="cuda")
    thi.thi_qk_norm_rope_kv16(dev(qkv), None, None, 1e-6, None, None, dev(np.array([slot], np.int32)), q, pool)
    ref.store(c["pages"], int(c["table"][0, 2]) * PAGE + 21, qkv[0, 8 * 128: 16 * 128].reshape(8, 128), qkv[0, 16 * 128:].reshape(8, 128))
    out = torch.empty(new, 8, D, dtype=torch.float16, device="cuda")
    ws = thi.Workspace(thi.thi_kv16_attention_workspace_bytes(1, new, 8, Hkv, D, new, table.shape[1]), init=False)
    thi.thi_kv16_attention(dev(c["q"]), pool, dev(table), dev(c["lens"]), dev(c["offsets"]), 0.1, 0, 0, out, new, ws)
    y, tol, _, _ = ref.attention(c, 0.1, weight=one_or_two(c))
    assert (np.abs(host(out.double()) - y) <= tol).all()
    del pool
    torch.cuda.empty_cache()


@pytest.mark.parametrize("new,weights,MP", [(1, True, 1 << 23), (3, False, 1 << 24), (40, False, 1 << 24), (40, True, 1 << 20)])
def test_longest_tables(thi, new, weights, MP):
    """Tables of as many pages as are not refused, of which a few are there: what a request of these pages alone has."""
    import torch
    c = attention_case(33, 2, 1, 64, [384], [new])
    at = np.array([0, 5, 63, 64, MP // 2 + 77, MP - 1])
    table = torch.full((1, MP), -1, dtype=torch.int32, device="cuda")
    table[0, dev(at)] = dev(c["table"][0, :6])
    say(f"[case] attention new={new} MP={MP} weights={weights}")
    out = torch.full((new, 2, 64), float("nan"), dtype=torch.float16, device="cuda")
    w = torch.full((1, 1, MP * PAGE), 7.0, device="cuda") if weights else None
    ws = thi.Workspace(thi.thi_kv16_attention_workspace_bytes(1, new, 2, 1, 64, new, MP, weights), init=False)
    thi.thi_kv16_attention(dev(c["q"]), dev(c["pages"]), table, dev(np.array([MP * PAGE], np.int32)), dev(c["offsets"]), 0.125, 0, 0, out, new, ws, None, w)
    y, tol, u, utol = ref.attention(c, 0.125, weight=one_or_two(c))
    assert (np.abs(host(out.double()) - y) <= tol).all()
    if weights:
        got = w.view(MP, PAGE)
        mine = dev(at)
        assert (np.abs(host(got[mine].double()).ravel() - u[0, 0, :384]) <= utol[0, 0, :384]).all()
        got[mine] = 0
        assert bool((w == 0).all())
    del w, ws, table
    torch.cuda.empty_cache()


def test_most_requests(thi):
    """As many requests as are not refused, of up to one page each, some empty, with weights."""
    import torch
    from perf import more_operators as plain
    B = 65535
    g = torch.Generator(device="cuda").manual_seed(34)
    pages = torch.randn(B, 1, 128 * 64, device="cuda", generator=g).half()
    table = torch.randperm(B, device="cuda", generator=g).int()[:, None].contiguous()
    lens = torch.randint(0, 65, (B,), device="cuda", generator=g).int()
    q = (2 * torch.randn(B, 1, 64, device="cuda", generator=g)).half()
    out, w = torch.full_like(q, float("nan")), torch.full((B, 1, PAGE), -1.0, device="cuda")
    ws = thi.Workspace(thi.thi_kv16_attention_workspace_bytes(B, B, 1, 1, 64, 1, 1, True), init=False)
    say(f"[case] attention B={B}")
    thi.thi_kv16_attention(q, pages, table, lens, None, 0.125, 0, 0, out, 1, ws, None, w)
    held = pages[table[:, 0].long()]
    k, v = plain._keys(held, 64)[:, 0].double(), plain._values(held, 64)[:, 0].double()
    seen = torch.arange(PAGE, device="cuda") < lens[:, None]
    x = q.double()
    p = torch.where(lens[:, None] > 0, torch.softmax(((k * x).sum(-1) * 0.125).masked_fill(~seen, -float("inf")), -1), 0.0)
    y = (p[..., None] * v).sum(1)
    e = 0.125 * (k.abs() * x.abs()).sum(-1) * 72 * 2.0 ** -24 + 2.0 ** -18 + 2.0 ** -20 + ref.TWO_SUMMANDS      # (as tests/kv16_reference.py has it)
    tol = 2.0 ** -25 + 2.0 ** -11 * y.abs() + ((p * torch.expm1(e))[..., None] * (v - y[:, None]).abs()).sum(1) * torch.exp(e.amax(-1))[:, None] + 256 * 2.0 ** -24 * (p[..., None] * v.abs()).sum(1) \
        + 2.0 ** -33 * v.abs().sum(1)
    assert bool(((out[:, 0].double() - y).abs() <= tol).all())
    off = p * torch.expm1(e + e.amax(-1, keepdim=True) + 128 * 2.0 ** -24) + 1e-30
    assert bool(((w[:, 0] - p).abs() <= off)[seen].all()) and bool((w[:, 0][~seen] == -1).all())


# ---- eviction -----------------------------------------------------------------------------------------------------


def evict_case(seed, layers, Hkv, D, lens, MP, P, shared=False):
    rng = np.random.default_rng(seed)
    R = len(lens)
    need = [min(MP, -(-max(0, n) // PAGE)) for n in lens]
    order, table, at = rng.permutation(P), np.full((R, MP), -1, np.int32), 0
    refs = np.zeros(P, np.int32)
    for b in range(R):
        table[b, : need[b]] = order[at: at + need[b]]
        at += need[b]
    assert at <= P
    if shared:                                                     # rows with the same first pages
        table[1, :2] = table[0, :2]
    for e in table[table >= 0]:
        refs[e] += 1
    w = np.maximum(np.exp(2 * rng.standard_normal((layers, R, Hkv, MP * PAGE))) - 0.3, 0).astype(np.float32)
    return dict(refs=refs, table=table, lens=np.array(lens, np.int32), weights=w, pages=rng.integers(0, 65536, (layers, P, Hkv, 128 * D)).astype(np.uint16).view(np.float16))


def check_evict(thi, c, budget, sinks=0, recent=0, headroom=0, info=True):
    import torch
    L, P, Hkv, _ = c["pages"].shape
    R, MP = c["table"].shape
    say(f"[case] evict layers={L} Hkv={Hkv} rows={R} MP={MP} P={P} lens={c['lens'].tolist()[:8]} budget={budget},{sinks},{recent},{headroom}")
    pool, ins = dev(c["pages"]), [dev(c[k]) for k in ("refs", "table", "lens", "weights")]
    outs = [torch.full_like(x, 77 if x.dtype == torch.int32 else float("nan")) for x in ins]
    inf = torch.full((2,), 77, dtype=torch.int32, device="cuda") if info else None
    ws = thi.Workspace(thi.thi_kv16_evict_workspace_bytes(L, R, Hkv, MP, P), init=False)
    thi.thi_kv16_evict(*ins, budget, sinks, recent, headroom, *outs, inf, pool, ws)
    want = ref.evict(c, budget, sinks, recent, headroom)
    for name, x in zip(("refs", "table", "lens"), outs):
        assert np.array_equal(host(x), want[name]), name
    if info:
        assert np.array_equal(host(inf), want["info"]), host(inf)
    assert np.array_equal(host(outs[3]).view(np.uint32)[~np.isnan(want["weights"])], want["weights"].view(np.uint32)[~np.isnan(want["weights"])])
    assert np.isnan(host(outs[3])[np.isnan(want["weights"])]).all()
    assert np.array_equal(host(pool).view(np.uint16), want["pages"].view(np.uint16)), "pages"
    for x, name in zip(ins, ("refs", "table", "lens", "weights")):      # what is read stays
        assert np.array_equal(host(x).view(np.uint32), c[name].view(np.uint32))
    return want


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("layers,Hkv,lens,budget,sinks,recent", [
    (1, 1, [65], 64, 0, 0), (2, 2, [300, 10, 0, 200], 100, 4, 32), (1, 3, [130, 129, 128, 64], 64, 1, 63), (3, 1, [500], 65, 0, 65), (1, 2, [90, 200], 1, 0, 0),
    (1, 2, [90, 200], 1, 1, 0), (2, 5, [700, 512, 513], 511, 70, 200), (1, 1, [1500, 3000], 1100, 4, 100), (1, 1, [64, 63], 64, 0, 0)])
def test_evict(thi, D, layers, Hkv, lens, budget, sinks, recent):
    MP = max(1, -(-max(lens) // PAGE)) + 1
    check_evict(thi, evict_case(len(lens) + budget, layers, Hkv, D, lens, MP, 2 * MP * len(lens) + 3), budget, sinks, recent)


@pytest.mark.parametrize("headroom", [0, 1, 27, 28, 64, 100000])
def test_evict_headroom(thi, headroom):
    c = evict_case(3, 1, 2, 64, [300, 40, 250], 6, 40)
    check_evict(thi, c, 100, 4, 20, headroom)


def test_evict_equal_and_odd_weights(thi):
    """Equal weights by their number, zeros of both signs, infinities, negative ones, NaN below all."""
    c = evict_case(4, 1, 2, 64, [400, 300], 7, 40)
    c["weights"][0, 0, 0, :] = 1
    c["weights"][0, 0, 1, 10:200] = 3
    w = c["weights"][0, 1]
    w[0, :] = np.nan
    w[0, 50:60], w[0, 60:65], w[0, 65:80], w[0, 80:90] = -np.inf, np.inf, -1.5, 0.0
    w[1, 0::2], w[1, 1::2] = 0.0, -0.0
    for budget, sinks, recent in ((64, 0, 0), (100, 4, 32), (33, 0, 0), (15, 5, 5), (8, 0, 8)):
        check_evict(thi, c, budget, sinks, recent)


def test_evict_missing_pages(thi):
    """Positions without a page are gone: kept are those of the budget that there are, none of them at the worst."""
    c = evict_case(5, 2, 2, 64, [400, 300, 200, 260], 7, 60)
    c["table"][0, [0, 3]] = [-1, 2 ** 31 - 1]
    c["table"][1, [1, 2, 3, 4]] = [-5, 60, -2 ** 31, -1]
    c["table"][2, :] = -1
    check_evict(thi, c, 120, 4, 32)
    check_evict(thi, c, 120, 100, 20, headroom=10)


@pytest.mark.parametrize("P", [14, 15, 16, 18, 30])
def test_evict_runs_out_of_pages(thi, P):
    check_evict(thi, evict_case(6, 1, 1, 64, [300, 300, 40, 200], 5, max(P, 15)) if P > 14 else evict_case(6, 1, 1, 64, [300, 300, 200], 5, 14), 64, 4, 10)


def test_evict_shared_pages(thi):
    """Rows that share their first pages each take what they keep along; the shared ones lose a reference for each."""
    want = check_evict(thi, evict_case(7, 2, 2, 128, [300, 260, 100], 6, 40, shared=True), 80, 4, 16)
    assert want["info"][0] == 3


def test_evict_lengths_outside_the_table(thi):
    c = evict_case(8, 1, 2, 64, [192, 192, -7], 3, 30)
    c["lens"][:] = [2 ** 31 - 1, 193, -2 ** 31]
    check_evict(thi, c, 100, 0, 10, info=False)


def test_evict_large_pool_and_many_rows(thi):
    rng = np.random.default_rng(9)
    check_evict(thi, evict_case(9, 1, 1, 64, rng.integers(0, 130, 1100).tolist(), 3, 4000), 64, 2, 8)


@pytest.mark.parametrize("rows,MP,P", [(40, 120, 5300), (40, 120, 4500), (200, 30, 6100), (200, 30, 5000)])
def test_evict_into_more_pages_than_a_plan_holds(thi, rows, MP, P):
    """Headroom for whole tables, so that rows get pages from the 4096th free one on; with the smaller pools the last rows stay."""
    lens = np.random.default_rng(11).integers(50, 200, rows).tolist()
    want = check_evict(thi, evict_case(11, 1, 1, 64, lens, MP, P), 64, 2, 8, headroom=100000)
    assert want["refs"].sum() > 4096 + 200


def test_evict_long_rows(thi):
    c = evict_case(10, 1, 2, 64, [20000], 320, 700)
    check_evict(thi, c, 9000, 4, 1000)


@pytest.mark.parametrize("n", [1, 100, 1 << 28])
def test_evict_row_that_stays_at_the_largest_budget(thi, n):
    """A table of 2^28 positions and a budget as large: the row stays, and its weights are copied, all of them and nothing else."""
    import torch
    MP = 1 << 22
    say(f"[case] evict MP={MP} budget={1 << 28} n={n}")
    table = torch.full((1, MP), -1, dtype=torch.int32, device="cuda")
    table[0, 0] = 0
    w = torch.rand(1, 1, 1, MP * PAGE, device="cuda")
    ins = [dev(np.array([1], np.int32)), table, dev(np.array([n], np.int32)), w]
    outs = [torch.full_like(x, 7) for x in ins]
    info = torch.full((2,), 7, dtype=torch.int32, device="cuda")
    pool = torch.ones(1, 1, 1, 128 * 64, dtype=torch.float16, device="cuda")
    ws = thi.Workspace(thi.thi_kv16_evict_workspace_bytes(1, 1, 1, MP, 1), init=False)
    thi.thi_kv16_evict(*ins, 1 << 28, 4, 100, 0, *outs, info, pool, ws)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(ins[:3], outs[:3])) and host(info).tolist() == [0, 0] and bool((pool == 1).all())
    assert torch.equal(outs[3][..., :n], w[..., :n]) and bool((outs[3][..., n:] == 7).all())
    del w, ins, outs, ws
    torch.cuda.empty_cache()


def test_evict_pages_past_32_bits(thi):
    import torch
    D, P = 128, 33000
    pool = torch.empty(1, P, 8, 128 * D, dtype=torch.float16, device="cuda")
    old, free = [P - 1, 3, P - 5], [1, P - 2, P - 3]
    for p in old:
        pool[0, p] = torch.randn(8, 128 * D, device="cuda").half()
    refs = np.ones(P, np.int32)
    refs[free] = 0
    ins = [dev(refs), dev(np.array([old], np.int32)), dev(np.array([190], np.int32)), torch.rand(1, 1, 8, 192, device="cuda")]
    outs = [torch.empty_like(x) for x in ins]
    ws = thi.Workspace(thi.thi_kv16_evict_workspace_bytes(1, 1, 8, 3, P), init=False)
    thi.thi_kv16_evict(*ins, 150, 4, 20, 0, *outs, None, pool, ws)
    c = dict(refs=np.array([1, 1, 1, 0, 0, 0], np.int32), table=np.array([[0, 1, 2]], np.int32), lens=np.array([190], np.int32), weights=host(ins[3]),
             pages=np.concatenate([host(pool[:, old]), np.zeros((1, 3, 8, 128 * D), np.float16)], 1))
    want = ref.evict(c, 150, 4, 20, 0)
    assert host(outs[1]).tolist() == [sorted(free)]
    got = host(pool[:, sorted(free)])
    for i in range(150):
        for a, b in zip(ref.load(got[0], i), ref.load(want["pages"][0, 3:], i)):
            assert np.array_equal(a, b, equal_nan=True), i
    del pool
    torch.cuda.empty_cache()


# ---- together, on streams, in graphs ------------------------------------------------------------------------------


class Served:
    """Two requests on a bounded cache: a prompt each, then single tokens, evicted when they pass their budget; the plain implementation beside it."""

    def __init__(self, thi, seed, Hq, Hkv, D, prompts, budget, sinks, recent, window=0):
        import torch
        self.thi, self.torch, self.rng = thi, torch, np.random.default_rng(seed)
        self.Hq, self.Hkv, self.D, self.budget, self.sinks, self.recent, self.window = Hq, Hkv, D, budget, sinks, recent, window
        self.MP, self.P, B = 5, 24, len(prompts)
        self.pages = np.zeros((1, self.P, Hkv, 128 * D), np.float16)
        self.refs, self.table, self.lens = np.zeros(self.P, np.int32), np.full((B, self.MP), -1, np.int32), np.zeros(B, np.int32)
        self.weights = np.zeros((1, B, Hkv, self.MP * PAGE), np.float32)
        self.place, self.theta = np.zeros(B, int), (10000.0 ** (-2 * np.arange(D // 2) / D)).astype(np.float32)

    def step(self, new):
        """One call of each operator on what the device gave last, each checked against the plain implementation of the same inputs."""
        thi, torch, B, T = self.thi, self.torch, len(new), sum(new)
        for b, n in enumerate(new):                                # pages for the new tokens
            for j in range(-(-int(self.lens[b] + n) // PAGE)):
                if self.table[b, j] < 0:
                    self.table[b, j] = int((self.refs == 0).argmax())
                    self.refs[self.table[b, j]] += 1
        rows = [(b, int(self.lens[b]) + i, self.place[b] + i) for b, n in enumerate(new) for i in range(n)]
        slots = np.array([self.table[b, p // PAGE] * PAGE + p % PAGE for b, p, _ in rows], np.int32)
        qkv = self.rng.standard_normal((T, (self.Hq + 2 * self.Hkv) * self.D)).astype(np.float16)
        positions = np.array([x for _, _, x in rows], np.int32)
        pool = dev(self.pages)
        q = torch.empty(T, self.Hq, self.D, dtype=torch.float16, device="cuda")
        thi.thi_qk_norm_rope_kv16(dev(qkv), None, None, 1e-6, dev(positions), dev(self.theta), dev(slots), q, pool[0])
        yq, yk, yv, tq, tk = ref.append(qkv, None, None, 1e-6, positions, self.theta, self.Hq, self.Hkv, self.D)
        assert (np.abs(host(q.double()) - yq) <= tq).all()
        self.pages = host(pool).copy()
        for t, s in enumerate(slots):
            k, v = ref.load(self.pages[0], int(s))
            assert (np.abs(k - yk[t]) <= tk[t]).all() and np.array_equal(v, yv[t])
        self.lens = (self.lens + np.array(new)).astype(np.int32)
        self.place += np.array(new)
        c = dict(q=host(q).view(np.float16), pages=self.pages[0], table=self.table, lens=self.lens, offsets=np.concatenate([[0], np.cumsum(new)]).astype(np.int32), max_q=max(new))
        w = dev(self.weights)
        out = torch.empty_like(q)
        ws = thi.Workspace(max(thi.thi_kv16_attention_workspace_bytes(B, T, self.Hq, self.Hkv, self.D, max(new), self.MP, True),
                               thi.thi_kv16_evict_workspace_bytes(1, B, self.Hkv, self.MP, self.P)), init=False)
        thi.thi_kv16_attention(q, pool[0], dev(self.table), dev(self.lens), dev(c["offsets"]), 0.125, self.window, self.sinks, out, max(new), ws, w[0], w[0])
        y, tol, u, utol = ref.attention(c, 0.125, self.window, self.sinks, one_or_two(c), self.weights[0])
        assert (np.abs(host(out.double()) - y) <= tol).all()
        fine = ~np.isnan(u)
        assert (np.abs(host(w[0].double()) - u)[fine] <= utol[fine]).all()
        self.weights = host(w).copy()
        state = dict(refs=self.refs, table=self.table, lens=self.lens, weights=self.weights, pages=self.pages)
        want = ref.evict(state, self.budget, self.sinks, self.recent, 1)
        ins = [dev(state[k]) for k in ("refs", "table", "lens", "weights")]
        outs = [torch.zeros_like(x) for x in ins]
        info = torch.empty(2, dtype=torch.int32, device="cuda")
        thi.thi_kv16_evict(*ins, self.budget, self.sinks, self.recent, 1, *outs, info, pool, ws)
        self.refs, self.table, self.lens, self.weights = (host(x).copy() for x in outs)
        self.pages = host(pool).copy()
        for name, x in (("refs", self.refs), ("table", self.table), ("lens", self.lens), ("pages", self.pages.view(np.uint16))):
            assert np.array_equal(x, want[name].view(np.uint16) if name == "pages" else want[name]), name
        kept = ~np.isnan(want["weights"])
        assert np.array_equal(self.weights[kept], want["weights"][kept])
        return int(host(info)[0])


@pytest.mark.parametrize("Hq,Hkv,D,window", [(4, 2, 64, 0), (8, 1, 128, 40), (2, 2, 128, 0)])
def test_a_bounded_cache_in_use(thi, Hq, Hkv, D, window):
    """Prompts, single tokens and a few at a time, evicted whenever a request passes its budget: every operator on what the one before it left."""
    s = Served(thi, 1, Hq, Hkv, D, [90, 130], budget=100, sinks=4, recent=30, window=window)
    moved = s.step([90, 130])
    for new in ([1, 1], [1, 1], [3, 2], [12, 1], [1, 1], [40, 7], [1, 1]):
        moved += s.step(new)
    assert moved >= 8 and (s.lens <= 100).all() and (s.refs >= 0).all()


def test_on_a_stream_of_its_own_and_in_graphs(thi):
    """Every operator on a side stream, then captured and replayed three times, with other work between the replays, against the eager results; then two graphs that
    share the workspaces, one after the other."""
    import torch
    Hq, Hkv, D, B = 8, 2, 128, 3
    c = attention_case(31, Hq, Hkv, D, [700, 66, 129], [1, 1, 1], extra=20)
    c["pages"] = np.nan_to_num(c["pages"])
    pages, table, lens, q = (dev(c[k]) for k in ("pages", "table", "lens", "q"))
    a = append_case(32, B, Hq, Hkv, D, 2)
    slots = dev(np.array([c["table"][b, (n - 1) // PAGE] * PAGE + (n - 1) % PAGE for b, n in enumerate(c["lens"])], np.int32))
    qkv, g, pos, th = (dev(a[k]) for k in ("qkv", "q_gamma", "positions", "theta"))
    refs = torch.zeros(len(c["pages"]), dtype=torch.int32, device="cuda")
    refs[table[table >= 0].long()] = 1
    ws = thi.Workspace(thi.thi_kv16_attention_workspace_bytes(B, B, Hq, Hkv, D, 1, table.shape[1], True), init=False)
    we = thi.Workspace(thi.thi_kv16_evict_workspace_bytes(1, B, Hkv, table.shape[1], len(refs)), init=False)

    def outputs():
        return dict(q=torch.empty_like(q), out=torch.empty_like(q), w=torch.zeros(1, B, Hkv, table.shape[1] * PAGE, device="cuda"), refs=torch.empty_like(refs),
                    table=torch.empty_like(table), lens=torch.empty_like(lens), w2=torch.zeros(1, B, Hkv, table.shape[1] * PAGE, device="cuda"),
                    info=torch.empty(2, dtype=torch.int32, device="cuda"))

    def step(o, window):
        thi.thi_qk_norm_rope_kv16(qkv, g, g, 1e-6, pos, th, slots, o["q"], pages)
        thi.thi_kv16_attention(q, pages, table, lens, None, 0.1, window, 4, o["out"], 1, ws, None, o["w"][0])
        thi.thi_kv16_evict(refs, table, lens, o["w"], 100, 4, 20, 0, o["refs"], o["table"], o["lens"], o["w2"], o["info"], pages.unsqueeze(0), we)

    want = []
    for window in (0, 80):
        o = outputs()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(o, window)
        torch.cuda.synchronize()
        p = outputs()
        step(p, window)
        assert all(torch.equal(o[k], p[k]) for k in o)
        want.append((p, pages.clone()))
    graphs, outs = [], []
    for window in (0, 80):
        o, graph = outputs(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(o, window)
        graphs.append(graph)
        outs.append(o)
    for i in range(3):
        for k in (0, 1):
            for t in outs[k].values():
                t.fill_(0 if t.dtype == torch.float32 else 7)
            torch.ones(1000, device="cuda").sum().item()
            graphs[k].replay()
            torch.cuda.synchronize()
            for name, t in outs[k].items():
                assert torch.equal(t, want[k][0][name]), (i, k, name)
            assert torch.equal(pages.view(torch.int16), want[k][1].view(torch.int16)), (i, k)


def test_prompts_and_mixed_calls_in_graphs(thi):
    """Two captured calls with weights that share a workspace, one of prompts and one of single tokens next to a chunk far behind, replayed in turn, with eager calls of a third kind between."""
    import torch
    cases = [(attention_case(50, 8, 2, 64, [300, 70, 128], [300, 33, 0]), 100, 4), (attention_case(51, 8, 2, 64, [4700, 200], [1, 40]), 0, 0), (attention_case(52, 8, 2, 64, [500, 66], [1, 1]), 0, 0)]
    need = max(thi.thi_kv16_attention_workspace_bytes(*c["table"].shape[:1], len(c["q"]), 8, 2, 64, c["max_q"], c["table"].shape[1], True) for c, _, _ in cases)
    ws = thi.Workspace(need, init=False)
    calls = []
    for c, window, sinks in cases:
        t = {k: dev(c[k]) for k in ("q", "pages", "table", "lens", "offsets")}
        o = dict(out=torch.empty_like(t["q"]), w=torch.zeros(len(c["lens"]), 2, c["table"].shape[1] * PAGE, device="cuda"))
        calls.append((lambda t=t, o=o, c=c, window=window, sinks=sinks: thi.thi_kv16_attention(t["q"], t["pages"], t["table"], t["lens"], t["offsets"], 0.1, window, sinks, o["out"], c["max_q"],
                                                                                              ws, None, o["w"]), o))
    want, graphs = [], []
    for call, o in calls:
        call()
        want.append({k: x.clone() for k, x in o.items()})
    torch.cuda.synchronize()
    for call, _ in calls[:2]:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        graphs.append(graph)
    for i in range(3):
        for k in (0, 1):
            calls[k][1]["out"].fill_(7)
            calls[k][1]["w"].zero_()
            calls[2][0]()
            graphs[k].replay()
            torch.cuda.synchronize()
            for j in (k, 2):
                for name, x in calls[j][1].items():
                    assert torch.equal(x, want[j][name]), (i, k, j, name)


def test_calls_at_the_same_time(thi):
    """Calls of different kinds on three streams at once, each with a workspace of its own: what each gives alone, every time."""
    import torch
    kinds = [(attention_case(60, 8, 2, 64, [4000, 700, 66], [1, 1, 2]), 0, 0), (attention_case(61, 4, 4, 128, [300, 200], [300, 33]), 90, 4),
             (attention_case(62, 8, 1, 128, [5000, 4800, 90], [1, 2, 50]), 0, 0)]
    calls, want, streams = [], [], [torch.cuda.Stream() for _ in kinds]
    for c, window, sinks in kinds:
        t = {k: dev(c[k]) for k in ("q", "pages", "table", "lens", "offsets")}
        (B, MP), (T, Hq, D), Hkv = c["table"].shape, c["q"].shape, c["pages"].shape[1]
        o = dict(out=torch.zeros_like(t["q"]), w=torch.zeros(B, Hkv, MP * PAGE, device="cuda"))
        ws = thi.Workspace(thi.thi_kv16_attention_workspace_bytes(B, T, Hq, Hkv, D, c["max_q"], MP, True), init=False)
        calls.append((lambda t=t, o=o, c=c, ws=ws, window=window, sinks=sinks, D=D: thi.thi_kv16_attention(t["q"], t["pages"], t["table"], t["lens"], t["offsets"], D ** -0.5, window, sinks,
                                                                                                       o["out"], c["max_q"], ws, None, o["w"]), o))
    for call, o in calls:
        call()
        torch.cuda.synchronize()
        want.append({k: x.clone() for k, x in o.items()})
    for _ in range(5):
        for _, o in calls:
            o["out"].fill_(7)
            o["w"].zero_()
        torch.cuda.synchronize()
        for _ in range(8):
            for stream, (call, _) in zip(streams, calls):
                with torch.cuda.stream(stream):
                    call()
        torch.cuda.synchronize()
        for (_, o), w in zip(calls, want):
            assert all(torch.equal(o[k], w[k]) for k in o)


@pytest.mark.parametrize("new", [[1, 1, 2], [40, 1, 17]])
def test_rows_behind_the_last_request_are_left(thi, new):
    """A batch padded to more rows than its requests have: those rows are not written, and the others are what they are without them."""
    import torch
    c = attention_case(53, 4, 2, 128, [100, 70, 64], new)
    T = sum(new)
    want, w = run_attention(thi, c, 0.125, weights=True)
    q = dev(np.concatenate([c["q"], np.full((5, 4, 128), np.nan, np.float16)]))
    out, got = torch.full_like(q, 7.0), torch.full((3, 2, c["table"].shape[1] * PAGE), float("nan"), device="cuda")
    ws = thi.Workspace(thi.thi_kv16_attention_workspace_bytes(3, T + 5, 4, 2, 128, max(new), c["table"].shape[1], True), init=False)
    thi.thi_kv16_attention(q, dev(c["pages"]), dev(c["table"]), dev(c["lens"]), dev(c["offsets"]), 0.125, 0, 0, out, max(new), ws, None, got)
    assert np.array_equal(host(out)[:T].astype(np.float64), want) and (host(out)[T:] == 7).all() and np.array_equal(host(got).astype(np.float64), w, equal_nan=True)


def test_the_same_bits_every_time(thi):
    import torch
    c = attention_case(40, 8, 2, 64, [900, 333], [5, 70])
    one = run_attention(thi, c, 0.125, 200, 4, weights=True)
    for _ in range(3):
        torch.randn(1 << 20, device="cuda").sort()
        two = run_attention(thi, c, 0.125, 200, 4, weights=True)
        assert np.array_equal(one[0], two[0]) and np.array_equal(one[1], two[1], equal_nan=True)


def test_a_workspace_that_is_too_small_is_refused(thi):
    import torch
    c = attention_case(41, 8, 1, 64, [1000], [1])
    out = torch.full((1, 8, 64), 7.0, dtype=torch.float16, device="cuda")
    need = thi.thi_kv16_attention_workspace_bytes(1, 1, 8, 1, 64, 1, c["table"].shape[1])
    assert need > 256
    rc = thi.thi_kv16_attention(dev(c["q"]), dev(c["pages"]), dev(c["table"]), dev(c["lens"]), None, 0.1, 0, 0, out, 1, thi.Workspace(256, init=False), check=False)
    assert rc == thi.THI_ERR_WORKSPACE and (host(out) == 7).all()
