"""The 4-bit cache's operators on the GPU, through the binding, against the plain implementation in tests/kv4_reference.py (64 bits).

Codes, scales, tables, counts and copied pages have to be equal; rotated queries and attention's outputs are held to tolerances that count
their roundings (each derived where it is used)."""
import numpy as np
import pytest

from tests import kv4_reference as ref
from tests.gpu_common import say, to_dev, to_host

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
    a = np.ascontiguousarray(a)
    return torch.from_numpy(a).cuda() if a.dtype != np.float16 else to_dev(a)


def host(t):
    import torch
    torch.cuda.synchronize()
    return t.cpu().numpy()


# ---- norm, rotation, store, read-back -----------------------------------------------------------------------------


def append_case(seed, T, Hq, Hkv, D, P, far=5000):
    rng = np.random.default_rng(seed)
    qkv = (rng.standard_normal((T, (Hq + 2 * Hkv) * D)) * np.exp(rng.standard_normal((Hq + 2 * Hkv) * D))).astype(np.float16)
    theta = (10000.0 ** (-2 * np.arange(D // 2) / D)).astype(np.float32)
    slots = rng.permutation(P * PAGE)[:T].astype(np.int32)
    return dict(qkv=qkv, q_gamma=(1 + 0.3 * rng.standard_normal(D)).astype(np.float16), k_gamma=(1 + 0.3 * rng.standard_normal(D)).astype(np.float16),
                theta=theta, positions=rng.integers(0, far, T).astype(np.int32), slots=slots, pages=rng.integers(0, 256, (P, Hkv, 68 * D), dtype=np.uint8))


def check_append(thi, c, Hq, Hkv, D, pad=0, eps=1e-6):
    import torch
    T = len(c["slots"])
    say(f"[case] append T={T} Hq={Hq} Hkv={Hkv} D={D} pad={pad} norm={c['q_gamma'] is not None},{c['k_gamma'] is not None} rope={c['theta'] is not None}")
    qkv = np.concatenate([c["qkv"], np.full((T, pad), np.nan, np.float16)], 1) if pad else c["qkv"]
    full = dev(qkv)
    pages = dev(c["pages"])
    q_out = torch.full((T + 1, Hq, D), float("nan"), dtype=torch.float16, device="cuda")
    opt = {k: dev(c[k]) if c[k] is not None else None for k in ("q_gamma", "k_gamma", "positions", "theta")}
    thi.thi_qk_norm_rope_kv4(full, opt["q_gamma"], opt["k_gamma"], eps, opt["positions"], opt["theta"], dev(c["slots"]), q_out[:T], pages)
    want = c["pages"].copy()
    q = np.zeros((T, Hq, D))
    for t in range(T):
        x = c["qkv"][t].astype(np.float64).reshape(-1, D)
        pos = None if c["theta"] is None else int(c["positions"][t])
        q[t] = ref.norm_rope(x[:Hq], c["q_gamma"], eps, pos, c["theta"])
        k = ref.norm_rope(x[Hq:Hq + Hkv], c["k_gamma"], eps, pos, c["theta"])
        ref.store(want, int(c["slots"][t]), k, x[Hq + Hkv:])
    got = host(q_out.float()).astype(np.float64)
    assert np.isnan(got[T]).all()                                   # behind the last row nothing is written
    fine = np.isfinite(q)
    # one rounding to fp16, by way of fp32: half a step, 2^-11 of the value (2^-25 where fp16 has no smaller step), and 2^-24 of it
    err = np.abs(got[:T] - q)[fine]
    bound = (np.abs(q) * (2.0 ** -11 + 2.0 ** -23) + 2.0 ** -25)[fine]
    over = np.abs(q[fine]) > 65504                                  # past fp16's range
    assert (err[~over] <= bound[~over]).all(), (err[~over] / bound[~over]).max()
    assert not np.isfinite(got[:T][~fine]).any()
    gp = host(pages)
    # a block that is not a number keeps whatever codes: only its scale byte is asked for
    where = np.argwhere(gp != want)
    if len(where):
        nan_ok = True
        for p, h, _ in where:
            for pos in range(PAGE):
                a, b = ref.load(gp[p:p + 1, h:h + 1], pos), ref.load(want[p:p + 1, h:h + 1], pos)
                nan_ok = nan_ok and all(np.array_equal(x, y, equal_nan=True) for x, y in zip(a, b))
        assert nan_ok, f"{len(where)} bytes differ, first {where[0]}"
    # read-back: what is stored, exactly; zeros where nothing is
    k_out, v_out = (torch.full((T, Hkv, D), float("nan"), dtype=torch.float16, device="cuda") for _ in range(2))
    thi.thi_kv4_read(pages, dev(c["slots"]), k_out, v_out)
    only_v = torch.empty_like(v_out)
    thi.thi_kv4_read(pages, dev(c["slots"]), None, only_v)
    k_got, v_got, v_only = host(k_out.double()), host(v_out.double()), host(only_v.double())
    for t in range(T):
        k, v = ref.load(want, int(c["slots"][t]))
        assert np.array_equal(k_got[t], k, equal_nan=True) and np.array_equal(v_got[t], v, equal_nan=True), t
        assert np.array_equal(v_only[t], v, equal_nan=True), t


@pytest.mark.parametrize("T,Hq,Hkv,D", [(1, 8, 8, 64), (1, 64, 8, 128), (3, 5, 5, 128), (7, 6, 2, 64), (33, 4, 1, 128), (70, 3, 3, 64), (130, 2, 1, 128)])
def test_append(thi, T, Hq, Hkv, D):
    check_append(thi, append_case(T * 100 + Hq, T, Hq, Hkv, D, 4), Hq, Hkv, D, pad=8 * (T % 3))


@pytest.mark.parametrize("missing", [("q_gamma",), ("k_gamma",), ("q_gamma", "k_gamma"), ("theta", "positions"), ("q_gamma", "k_gamma", "theta", "positions")])
def test_append_without_norm_or_rotation(thi, missing):
    c = append_case(5, 9, 4, 2, 128, 3)
    for m in missing:
        c[m] = None
    check_append(thi, c, 4, 2, 128)


@pytest.mark.parametrize("D", [64, 128])
def test_append_runs_of_slots(thi, D):
    """A prompt's tokens: runs of neighbouring slots that begin and end anywhere in a page, in pages that do not follow each other, and in
    descending order."""
    c = append_case(11, 150, 2, 2, D, 7)
    run = np.r_[np.arange(37, 64), np.arange(64 * 5, 64 * 6), np.arange(64 * 2, 64 * 2 + 50), np.arange(64 * 4 + 9, 64 * 4, -1)]
    c["slots"] = run.astype(np.int32)
    check_append(thi, c, 2, 2, D)


def test_append_many_tokens(thi):
    """More tokens than the few-token launch shape takes: a token's heads in one workgroup."""
    T = 1100
    c = append_case(12, T, 1, 1, 64, 20)
    c["slots"] = (np.arange(T) + 17).astype(np.int32)
    check_append(thi, c, 1, 1, 64)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("first", [-1, 0, 2, 6 * PAGE])
def test_append_first_slot_and_run(thi, D, first):
    """Padding, or a slot of its own, in front of runs that begin a dword of the page, or do not; the last run ends inside one."""
    T = 205
    c = append_case(13 + first, T, 2, 1, D, 6)
    c["slots"] = np.r_[first, 4 + np.arange(100), 130 + np.arange(T - 101)].astype(np.int32)
    check_append(thi, c, 2, 1, D)
    c["slots"] = (8 + np.arange(T)).astype(np.int32)
    check_append(thi, c, 2, 1, D)


def test_append_slots_outside_the_pool(thi):
    c = append_case(6, 12, 4, 2, 128, 3)
    c["slots"][[0, 3, 4, 11]] = [-1, 3 * PAGE, 2 ** 31 - 1, -2 ** 31]
    check_append(thi, c, 4, 2, 128)


@pytest.mark.parametrize("far", [131072, 2 ** 31 - 1])
def test_append_far_positions(thi, far):
    c = append_case(7, 6, 4, 2, 128, 3)
    c["positions"] = np.array([0, 1, far - 1, far, far // 2, far // 3], np.int32)
    check_append(thi, c, 4, 2, 128)


def test_append_special_values(thi):
    """Blocks of zeros, of fp16's smallest numbers, of its largest, at the scales' borders, on the borders between codes, with infinities and NaN."""
    D, Hkv = 128, 2
    c = append_case(8, 10, 2, Hkv, D, 2)
    x = c["qkv"].reshape(10, 6, D)
    x[0, 2:] = 0
    x[1, 2:] = np.float16(2.0 ** -24)
    x[2, 2:] = np.float16(65504)
    x[2, 2:, ::3] = np.float16(-40000)
    x[3, 2:] = np.tile(np.float16([7, 0.25, -0.75, 1.25, 1.75, -2.5, 3.5, 5]), (4, D // 8))
    x[4, 2:] = np.tile(np.float16([7.004, 0.5, -1.5, 2.5, 3.5, -5, 7, 6]), (4, D // 8))
    x[5, 2:, 5], x[6, 2:, 70], x[7, 2:, 127] = np.inf, -np.inf, np.nan
    x[8, 2:] = np.tile(np.float16([6e-8, -1.2e-7, 4e-7, 3.6e-7, 8.4e-7, 0, -0.0, 1e-6]), (4, D // 8))
    c["q_gamma"] = c["k_gamma"] = None
    c["theta"] = c["positions"] = None
    check_append(thi, c, 2, Hkv, D)


# ---- attention ----------------------------------------------------------------------------------------------------


def attention_case(seed, Hq, Hkv, D, lens, new, spare=3, scale_of_q=2.0):
    """Pages with quantised Gaussian keys and values for each request's positions, everything else 0xff (NaN scales)."""
    rng = np.random.default_rng(seed)
    need = [-(-n // PAGE) for n in lens]
    P, MP = sum(need) + spare, max(max(need), 1)
    order = rng.permutation(P)
    pages = np.full((P, Hkv, 68 * D), 255, np.uint8)
    table = np.full((len(lens), MP), -1, np.int32)
    at = 0
    for b, n in enumerate(lens):
        table[b, :need[b]] = order[at:at + need[b]]
        at += need[b]
        for pos in range(n):
            ref.store(pages, int(table[b, pos // PAGE]) * PAGE + pos % PAGE, rng.standard_normal((Hkv, D)), rng.standard_normal((Hkv, D)))
    T = sum(new)
    q = (scale_of_q * rng.standard_normal((T, Hq, D))).astype(np.float16)
    offsets = np.r_[0, np.cumsum(new)].astype(np.int32)
    return dict(q=q, pages=pages, table=table, lens=np.array(lens, np.int32), offsets=offsets)


def run_attention(thi, c, scale, decode=False, max_q=None, stream=None):
    import torch
    T, Hq, D = c["q"].shape
    B, MP = c["table"].shape
    Hkv = c["pages"].shape[1]
    max_q = max_q or (1 if decode else max(1, int(np.diff(c["offsets"]).max())))
    ws = thi.Workspace(thi.thi_kv4_attention_workspace_bytes(B, T, Hq, Hkv, D, max_q, MP), init=False)
    ws.buffer.fill_(255)
    out = torch.full((T + 1, Hq, D), 777.0, dtype=torch.float16, device="cuda")
    args = (dev(c["q"]), dev(c["pages"]), dev(c["table"]), dev(c["lens"]), None if decode else dev(c["offsets"]), scale)
    thi.thi_kv4_attention(*args, out[:T], max_q, ws)
    again = torch.full_like(out, 777.0)
    thi.thi_kv4_attention(*args, again[:T], max_q, ws)
    assert torch.equal(out.view(torch.int16), again.view(torch.int16)), "two runs differ"
    got = host(out.double())
    assert (got[T] == 777).all()
    return got[:T]


def check_attention(thi, c, scale=None, decode=False, what=""):
    T, Hq, D = c["q"].shape
    scale = D ** -0.5 if scale is None else scale
    say(f"[case] attention {what} Hq={Hq} Hkv={c['pages'].shape[1]} D={D} lens={c['lens'].tolist()[:8]} rows={np.diff(c['offsets']).tolist()[:8]}")
    y, S, E = ref.attention(c["q"], c["pages"], c["table"], c["lens"], None if decode else c["offsets"], scale)
    got = run_attention(thi, c, scale, decode)
    tol = ref.attention_tolerance(y, S, E, D, c["table"].shape[1] * PAGE)
    err = np.abs(got - y)
    assert (err <= tol).all(), f"worst {(err / tol).max():.3g} of the tolerance at {np.unravel_index((err / tol).argmax(), err.shape)}"
    return got


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (4, 4), (8, 4), (6, 2), (8, 1), (16, 1), (20, 1), (34, 2)])
def test_decode_heads(thi, D, Hq, Hkv):
    """One token per request, every kind of group (one head, odd, more than a matrix tile holds); empty and one-position requests."""
    c = attention_case(Hq * 10 + D, Hq, Hkv, D, [130, 0, 1, 64], [1, 1, 1, 1])
    check_attention(thi, c, decode=True, what="decode")


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 191, 255, 257, 511, 513, 1025])
def test_decode_lengths(thi, n):
    c = attention_case(n, 4, 1, 128, [n], [1])
    check_attention(thi, c, decode=True, what="decode")


def test_decode_long_requests_next_to_short_ones(thi):
    """Requests that are cut into chunks next to ones that are not; a request's result does not depend on the others."""
    lens = [2200, 3, 700, 0, 1500, 64]
    c = attention_case(3, 4, 2, 64, lens, [1] * 6)
    got = check_attention(thi, c, decode=True, what="decode")
    order = [4, 3, 0, 5, 2, 1]
    d = dict(c, q=c["q"][order], table=c["table"][order], lens=c["lens"][order])
    assert np.array_equal(run_attention(thi, d, 64 ** -0.5, decode=True), got[order])


@pytest.mark.parametrize("Hq,Hkv,D", [(4, 4, 128), (8, 1, 128), (5, 1, 64), (3, 3, 64)])
@pytest.mark.parametrize("new", [2, 3, 5, 16, 17, 33])
def test_few_new_tokens(thi, Hq, Hkv, D, new):
    """Speculative tokens: several rows per request, some with as many positions as rows, some with fewer (rows that see nothing)."""
    c = attention_case(new * 7 + Hq, Hq, Hkv, D, [150, new, max(0, new - 2), 66], [new, new, new, 1])
    check_attention(thi, c, what="few")


@pytest.mark.parametrize("Hq,Hkv,D", [(2, 2, 128), (8, 2, 128), (3, 1, 64), (1, 1, 64)])
def test_prompts(thi, Hq, Hkv, D):
    """Whole prompts and chunks on a cache that is there, of odd lengths, next to a single token and a request without rows."""
    c = attention_case(Hq + D, Hq, Hkv, D, [300, 90, 64, 400, 200], [300, 1, 64, 129, 0])
    check_attention(thi, c, what="prompt")


def test_prompt_of_one_long_request(thi):
    c = attention_case(17, 2, 1, 128, [700], [700])
    check_attention(thi, c, what="prompt")


@pytest.mark.parametrize("new", [1, 4, 90])
def test_missing_pages(thi, new):
    """Entries that are no page (-1, past the pool, negative) are positions that are not there: at the front, in the middle, at the end, all of them."""
    c = attention_case(21, 4, 2, 128, [400, 400, 130, 400], [new] * 4)
    c["table"][0, [0, 3]] = [-1, 2 ** 31 - 1]
    c["table"][1, [1, 2, 6]] = [-5, len(c["pages"]), -2 ** 31]
    c["table"][2, :] = -1
    check_attention(thi, c, what="missing pages")


def test_lengths_outside_the_table(thi):
    """A length past the table's reach is the table's reach; a negative one is none."""
    c = attention_case(22, 2, 2, 64, [192, 192, 100], [1, 1, 1])
    c["lens"][:] = [2 ** 31 - 1, 193, -7]
    check_attention(thi, c, decode=True, what="lengths")


def test_dead_positions_and_foreign_pages_do_not_matter(thi):
    """Everything past a request's last position holds NaN scales (attention_case fills it so): no NaN comes through, also with weights of zero."""
    c = attention_case(23, 8, 2, 128, [65, 1, 129], [1, 1, 1])
    assert np.isfinite(check_attention(thi, c, decode=True)).all()
    c = attention_case(24, 8, 2, 128, [65, 40, 129], [40, 40, 40])
    assert np.isfinite(check_attention(thi, c)).all()


@pytest.mark.parametrize("new", [1, 70])
def test_nan_in_the_cache_reaches_the_rows_that_see_it(thi, new):
    c = attention_case(25, 2, 1, 128, [100, 100], [new, new])
    slot = int(c["table"][0, 0]) * PAGE + 60
    k = np.full((1, 128), np.nan)
    ref.store(c["pages"], slot, k, k)
    y, _, _ = ref.attention(c["q"], c["pages"], c["table"], c["lens"], None if new == 1 else c["offsets"], 0.1)
    got = run_attention(thi, c, 0.1, decode=new == 1)
    assert np.array_equal(np.isnan(got), np.isnan(y)) and np.isnan(y).any() and not np.isnan(y).all()


@pytest.mark.parametrize("new", [1, 3, 80])
def test_peaked_and_large_scores(thi, new):
    """Scores of some hundreds: one weight near 1, the others near 0; and a scale of zero: plain means."""
    c = attention_case(26, 4, 2, 128, [200, 90], [new, min(new, 90)], scale_of_q=60.0)
    check_attention(thi, c, what="peaked")
    check_attention(thi, c, scale=0.0, what="means")
    check_attention(thi, c, scale=-0.05, what="negative scale")


def test_pages_past_32_bits(thi):
    """A pool of more than 4 GiB, of which pages at both ends are used: byte offsets are 64-bit."""
    import torch
    Hkv, D = 8, 128
    P = (5 << 30) // thi.thi_kv4_page_bytes(Hkv, D)
    small = attention_case(27, 8, Hkv, D, [100, 150], [1, 1])
    big = torch.empty(P, Hkv, 68 * D, dtype=torch.uint8, device="cuda")
    far = P - len(small["pages"]) + np.arange(len(small["pages"]))
    far[0] = 1
    big[torch.from_numpy(far).cuda()] = dev(small["pages"])
    table = np.where(small["table"] >= 0, far[small["table"]], -1).astype(np.int32)
    ws = thi.Workspace(thi.thi_kv4_attention_workspace_bytes(2, 2, 8, Hkv, D, 1, table.shape[1]), init=False)
    out = torch.empty(2, 8, D, dtype=torch.float16, device="cuda")
    thi.thi_kv4_attention(dev(small["q"]), big, dev(table), dev(small["lens"]), None, 0.1, out, 1, ws)
    assert np.array_equal(host(out.double()), run_attention(thi, small, 0.1, decode=True))
    # append and read at the far end
    c = append_case(28, 5, 8, Hkv, D, 2)
    slots = ((P - 1) * PAGE + np.arange(5) * 7).astype(np.int32)
    q_out = torch.empty(5, 8, D, dtype=torch.float16, device="cuda")
    thi.thi_qk_norm_rope_kv4(dev(c["qkv"]), None, None, 1e-6, None, None, dev(slots), q_out, big)
    k_out, v_out = (torch.empty(5, Hkv, D, dtype=torch.float16, device="cuda") for _ in range(2))
    thi.thi_kv4_read(big, dev(slots), k_out, v_out)
    x = c["qkv"].astype(np.float64).reshape(5, -1, D)
    assert np.array_equal(host(k_out.double()), ref.quantise(x[:, 8:8 + Hkv])[2]) and np.array_equal(host(v_out.double()), ref.quantise(x[:, 8 + Hkv:])[2])


# ---- pages --------------------------------------------------------------------------------------------------------


def page_case(seed, rows, MP, P, most, words=64, layers=2):
    """Rows with random lengths and, here and there, pages beyond their length, shared whole pages, and references held elsewhere."""
    rng = np.random.default_rng(seed)
    table, lens, refs = np.full((rows, MP), -1, np.int32), np.zeros(rows, np.int32), np.zeros(P, np.int32)
    order = list(rng.permutation(P))
    for i in range(rows):
        lens[i] = rng.integers(0, most + 1)
        held = min(MP, -(-int(lens[i]) // PAGE) + int(rng.integers(0, 3)))
        for j in range(held):
            if j < lens[i] // PAGE and i and rng.random() < 0.3 and j < lens[i - 1] // PAGE and table[i - 1, j] >= 0:
                table[i, j] = table[i - 1, j]
            elif order and rng.random() < 0.97:
                table[i, j] = order.pop()
            if table[i, j] >= 0:
                refs[table[i, j]] += 1
    for p in order[:2]:
        refs[p] = 1                                                    # kept by somebody else
    used = table[table >= 0]
    if len(used):
        refs[rng.choice(used, max(1, len(used) // 10))] += 1
    pool = rng.integers(-2 ** 31, 2 ** 31, (layers, P, words), dtype=np.int32)
    return dict(table=table, lens=lens, refs=refs, pool=pool, rng=rng)


def run_fork(thi, c, parents, headroom):
    import torch
    N, (R, MP), P = len(parents), c["table"].shape, len(c["refs"])
    ws = thi.Workspace(thi.thi_kv4_pages_workspace_bytes(N, R, MP, P), init=False)
    ws.buffer.fill_(255)
    pool = dev(c["pool"])
    ins = [dev(c[k]) for k in ("refs", "table", "lens")]
    got = None
    for _ in range(2):                                                  # a pass can be repeated: it reads what it does not write
        outs = [torch.full(s, -99, dtype=torch.int32, device="cuda") for s in ((P,), (N, MP), (N,), (2,))]
        thi.thi_kv4_fork(*ins, dev(np.asarray(parents, np.int32)), None if headroom is None else dev(np.asarray(headroom, np.int32)), outs[0], outs[1], outs[2], outs[3],
                         pool, ws)
        now = [host(t) for t in outs] + [host(pool)]
        assert got is None or all(np.array_equal(a, b) for a, b in zip(got, now))
        got = now
    return got


def check_fork(thi, c, parents, headroom, what=""):
    P = len(c["refs"])
    say(f"[case] fork {what} rows {c['table'].shape} -> {len(parents)} pages {P}")
    refs, table, lens, info, copies = ref.fork(c["refs"], c["table"], c["lens"], parents, headroom, P)
    got = run_fork(thi, c, parents, headroom)
    pool = c["pool"].copy()
    for src, dst in copies:
        pool[:, dst] = c["pool"][:, src]
    for name, a, b in zip(("refs", "table", "lens", "info", "pool"), got, (refs, table, lens, np.array(info), pool)):
        assert np.array_equal(a, b), (what, name, np.argwhere(a != b)[:4].tolist())
    return copies


@pytest.mark.parametrize("seed,rows,out,MP,P", [(1, 1, 1, 1, 4), (2, 1, 4, 6, 20), (3, 5, 9, 8, 90), (4, 9, 5, 8, 90), (5, 64, 64, 12, 700), (6, 70, 200, 5, 900), (7, 300, 1500, 3, 4000)])
def test_fork(thi, seed, rows, out, MP, P):
    c = page_case(seed, rows, MP, P, MP * PAGE)
    rng = c["rng"]
    parents = rng.integers(-1, rows + 1, out)                           # -1 and rows: rows that start empty
    check_fork(thi, c, parents, rng.integers(-3, 200, out), "mixed")
    check_fork(thi, c, np.arange(out) % rows, None, "no headroom")
    check_fork(thi, c, np.full(out, rows - 1), np.ones(out, int), "one parent")


def test_fork_frees_and_grows(thi):
    c = page_case(9, 6, 10, 100, 300)
    check_fork(thi, c, [-1] * 6, None, "free all")
    check_fork(thi, c, [-1] * 3, [640, 64, 65], "new requests")
    check_fork(thi, c, np.arange(6), [700, 0, 1, 64, 128, 5], "grow in place")


def test_fork_runs_out_of_pages(thi):
    c = page_case(10, 8, 6, 34, 6 * PAGE)
    check_fork(thi, c, np.arange(24) % 8, np.full(24, 100), "short of pages")


def test_fork_of_many_free_pages(thi):
    """More counts than one step of the plan takes, free pages at the far end only."""
    c = page_case(11, 3, 4, 40, 200)
    P = 20000
    refs = np.ones(P, np.int32)
    refs[:40] = np.maximum(c["refs"], 1)
    refs[[9000, 15000, 19990, 19991, 19999]] = 0
    c["refs"], c["pool"] = refs, c["rng"].integers(0, 1 << 30, (1, P, 4), dtype=np.int32)
    check_fork(thi, c, [0, 0, 1, 1, 2, 2], [64] * 6, "far free pages")


def test_fork_ignores_entries_and_lengths_that_are_none(thi):
    c = page_case(12, 5, 6, 60, 300)
    c["table"][1, 0], c["table"][2, 1], c["table"][3, 5] = 60, 2 ** 31 - 1, -2 ** 31
    c["lens"][:] = [2 ** 31 - 1, -4, 6 * PAGE + 1, 100, 64]
    check_fork(thi, c, [0, 1, 2, 3, 4, 0, 3, 3, 4], [2 ** 31 - 1, 1, 1, 1, 1, -2 ** 31, 300, 0, 0], "odd entries")


def check_compact(thi, c, what=""):
    import torch
    P, (R, MP) = len(c["refs"]), c["table"].shape
    say(f"[case] compact {what} rows {R} pages {P}")
    refs, table, info, moves = ref.compact(c["refs"], c["table"], P)
    pool = c["pool"].copy()
    for src, dst in moves:
        pool[:, dst] = c["pool"][:, src]
    ws = thi.Workspace(thi.thi_kv4_pages_workspace_bytes(R, R, MP, P), init=False)
    ws.buffer.fill_(255)
    dp = dev(c["pool"])
    outs = [torch.full(s, -99, dtype=torch.int32, device="cuda") for s in ((P,), (R, MP), (2,))]
    thi.thi_kv4_compact(dev(c["refs"]), dev(c["table"]), *outs, dp, ws)
    for name, a, b in zip(("refs", "table", "info", "pool"), [host(t) for t in outs] + [host(dp)], (refs, table, np.array(info), pool)):
        assert np.array_equal(a, b), (what, name, np.argwhere(a != b)[:4].tolist())
    return moves


@pytest.mark.parametrize("seed,rows,MP,P,words", [(1, 1, 1, 1, 4), (2, 3, 5, 30, 4), (3, 20, 8, 300, 1088), (4, 40, 6, 1025, 12), (5, 200, 9, 9000, 4)])
def test_compact(thi, seed, rows, MP, P, words):
    c = page_case(seed, rows, MP, P, MP * PAGE, words=words, layers=3)
    assert check_compact(thi, c) or P == 1


def test_compact_nothing_to_move(thi):
    c = page_case(6, 3, 4, 30, 200)
    c["refs"][:] = 0
    check_compact(thi, c, "nothing live")
    c["refs"][:] = 2
    check_compact(thi, c, "all live")
    c["refs"][:] = 0
    c["refs"][-1] = 1
    check_compact(thi, c, "one at the end")
    c["table"][0, 0], c["table"][1, 0] = 30, -77
    check_compact(thi, c, "entries that are no page")


@pytest.mark.parametrize("MP", [9, 70, 200])
def test_fork_with_many_pages_behind_a_row(thi, MP):
    """Headroom and pages held beyond the length by the hundred, next to rows without: taken over, given up, taken fresh, until none is left."""
    c = page_case(40 + MP, 12, MP, 12 * MP + 40, 2 * PAGE, words=300)
    used = set(c["table"][c["table"] >= 0].tolist())
    spare = [p for p in range(len(c["refs"])) if c["refs"][p] == 0 and p not in used]
    c["table"][3, 3:MP - 1] = spare[:MP - 4]                             # held far beyond the length, by row 3 alone
    c["refs"][spare[:MP - 4]] = 1
    check_fork(thi, c, [3, 3, 0, -1, 5, 5, 11, 1], [MP * PAGE, 0, 1, 65 * PAGE, 3, 64 * PAGE + 1, 0, 2 ** 31 - 1], "long tails")
    check_fork(thi, c, list(range(12)) * 6, [MP * PAGE] * 72, "long tails, too few pages")


@pytest.mark.parametrize("words", [4, 252, 256, 300, 4100])
def test_page_sizes(thi, words):
    """Pages of 16 bytes, of a slice of the copy more or less, of some slices and a rest."""
    c = page_case(60, 30, 6, 260, 6 * PAGE, words=words, layers=3)
    assert check_fork(thi, c, np.arange(90) // 3, np.ones(90, int), "page sizes")
    assert check_compact(thi, c, "page sizes")


def test_compact_large_pool(thi):
    c = page_case(61, 200, 60, 20000, 60 * PAGE, words=4)
    assert check_compact(thi, c, "large pool")


# ---- streams and graphs -------------------------------------------------------------------------------------------


def test_on_a_stream_of_its_own_and_in_a_graph(thi):
    """Every operator on a side stream, then captured and replayed three times, with other work between the replays, against the eager results."""
    import torch
    Hq, Hkv, D, B = 8, 2, 128, 3
    c = attention_case(31, Hq, Hkv, D, [700, 66, 129], [1, 1, 1])
    pages = dev(c["pages"])
    table, lens, q = dev(c["table"]), dev(c["lens"]), dev(c["q"])
    a = append_case(32, B, Hq, Hkv, D, 2)
    slots = np.array([table.cpu().numpy()[b, (n - 1) // PAGE] * PAGE + (n - 1) % PAGE for b, n in enumerate(c["lens"])], np.int32)
    args = dict(qkv=dev(a["qkv"]), g=dev(a["q_gamma"]), pos=dev(a["positions"]), th=dev(a["theta"]), slots=dev(slots))
    q_out = torch.empty(B, Hq, D, dtype=torch.float16, device="cuda")
    k_out, v_out = (torch.empty(B, Hkv, D, dtype=torch.float16, device="cuda") for _ in range(2))
    out = torch.empty(B, Hq, D, dtype=torch.float16, device="cuda")
    refs = torch.zeros(len(c["pages"]), dtype=torch.int32, device="cuda")
    refs[table[table >= 0].long()] = 1
    parents, room = torch.tensor([0, 0, 2], dtype=torch.int32, device="cuda"), torch.ones(3, dtype=torch.int32, device="cuda")
    refs2, table2, lens2, info = torch.empty_like(refs), torch.empty_like(table), torch.empty_like(lens), torch.empty(2, dtype=torch.int32, device="cuda")
    refs3, table3, info3 = torch.empty_like(refs), torch.empty_like(table), torch.empty(2, dtype=torch.int32, device="cuda")
    ws = thi.Workspace(thi.thi_kv4_attention_workspace_bytes(B, B, Hq, Hkv, D, 1, table.shape[1]), init=False)
    wp = thi.Workspace(thi.thi_kv4_pages_workspace_bytes(3, 3, table.shape[1], len(refs)), init=False)
    outputs = (q_out, k_out, v_out, out, refs2, table2, lens2, info, refs3, table3, info3, pages)

    def step():
        thi.thi_qk_norm_rope_kv4(args["qkv"], args["g"], args["g"], 1e-6, args["pos"], args["th"], args["slots"], q_out, pages)
        thi.thi_kv4_read(pages, args["slots"], k_out, v_out)
        thi.thi_kv4_attention(q, pages, table, lens, None, 0.1, out, 1, ws)
        thi.thi_kv4_fork(refs, table, lens, parents, room, refs2, table2, lens2, info, pages.unsqueeze(0), wp)
        thi.thi_kv4_compact(refs2, table2, refs3, table3, info3, pages.unsqueeze(0), wp)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    # the state that a pass leaves, and the same pass again from there, are what a replay has to give
    step()
    want = [host(t).copy() for t in outputs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        for t in outputs[:-1]:
            t.fill_(7)
        torch.ones(1000, device="cuda").sum().item()
        graph.replay()
        for got, w in zip((host(t) for t in outputs), want):
            assert np.array_equal(got.view(np.uint8), w.view(np.uint8)), i
