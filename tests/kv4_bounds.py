"""How far attention over the 4-bit cache may be off, row by row, from the operator's definition (test infrastructure).

With scores off by d_j and weights off by a factor of 1 + w at most, the result is sum p_j f_j v_j / sum p_j f_j with |ln f_j| <= d_j + w, so it is
off by no more than  sum p_j |v_j - y| (exp(d_j + w) - 1) exp(max d_j + w),  whatever the signs."""
import numpy as np

from tests import kv4_reference as ref

PAGE = ref.PAGE
QUERY = 2.0 ** -16 / 3.75        # of a block's largest: what four e2m3 summands leave of 2^e, the largest being more than 3.75 * 2^e
ONE_SUMMAND, TWO_SUMMANDS = 2.0 ** -11, 2.0 ** -21


def held(c, b):
    """Positions of request b that have a page, and their keys and values [n, Hkv, D]."""
    P, MP = len(c["pages"]), c["table"].shape[1]
    n = int(min(max(c["lens"][b], 0), MP * PAGE))
    at = [p for p in range(n) if 0 <= c["table"][b, p // PAGE] < P]
    kv = [ref.load(c["pages"], int(c["table"][b, p // PAGE]) * PAGE + p % PAGE) for p in at]
    Hkv, D = c["pages"].shape[1], c["q"].shape[2]
    k, v = (np.stack([x[i] for x in kv]) if kv else np.zeros((0, Hkv, D)) for i in range(2))
    return n, np.array(at, int), k, v


def attention(c, scale, weight=TWO_SUMMANDS, query=QUERY, weights=None):
    """(out, tolerance) [T, Hq, D].  Roundings that are counted: the query's block (`query` of its largest, for each of a key's magnitudes), 32-bit sums of D products with
    the distance to the maximum (2^-24 of the magnitudes' sum for each product, 2^-18 for the rest), the exponential (2^-20), a weight (`weight` of it; 2^-33 where that is
    below what fp16 holds), 32-bit sums of the positions, the result (2^-11 of it, or 2^-25).  `weights`: what the definition's weights become before they are summed."""
    T, Hq, D = c["q"].shape
    Hkv = c["pages"].shape[1]
    q = c["q"].astype(np.float64)
    out, tol = np.zeros((T, Hq, D)), np.full((T, Hq, D), 2.0 ** -25)
    for b in range(len(c["lens"])):
        n, at, k, v = held(c, b)
        m = int(c["offsets"][b + 1] - c["offsets"][b])
        for i in range(m):
            seen = at <= n - m + i
            if not seen.any():
                continue
            t = int(c["offsets"][b]) + i
            for h in range(Hq):
                kk, vv, x = k[seen, h // (Hq // Hkv)], v[seen, h // (Hq // Hkv)], q[t, h]
                s = kk @ x * scale
                p = np.exp(s - s.max())
                p = p if weights is None else weights(p)
                p = p / p.sum()
                y = p @ vv
                largest = np.repeat(np.abs(x).reshape(-1, 32).max(-1), 32)
                d = abs(scale) * (np.abs(kk) @ (query * largest + (D + 8) * 2.0 ** -24 * np.abs(x))) + 2.0 ** -18 + 2.0 ** -20 + weight
                spread = np.abs(vv - y)
                out[t, h] = y
                tol[t, h] += 2.0 ** -11 * np.abs(y) + (p * np.expm1(d)) @ spread * np.exp(d.max()) + 2.0 ** -33 * np.abs(vv).sum(0) + 2 * (len(p) + 64) * 2.0 ** -24 * (p @ np.abs(vv))
    return out, tol


def far_queries(seed, Hq, Hkv, D, lens, new):
    """Queries with one large column in each block of 32, the others some 2^-12 of it; keys with one column each, not a large one, so that a score is one
    small column times 2^5 and shows what is left of it."""
    rng = np.random.default_rng(seed)
    B, T = len(lens), sum(new)
    pages, table = np.full((B + 2, Hkv, 68 * D), 255, np.uint8), rng.permutation(B + 2)[:B].astype(np.int32)[:, None]
    large = rng.integers(0, 32, D // 32)                              # the same columns for all rows
    small = np.ones(D, bool)
    small[np.arange(D // 32) * 32 + large] = False
    for b, n in enumerate(lens):
        assert n <= PAGE
        for pos in range(n):
            k = np.zeros((Hkv, D))
            if pos:
                k[np.arange(Hkv), rng.choice(np.flatnonzero(small), Hkv)] = 32.0
            ref.store(pages, int(table[b, 0]) * PAGE + pos, k, rng.standard_normal((Hkv, D)))
    q = 0.25 * rng.standard_normal((T, Hq, D))
    q[..., ~small] = rng.uniform(1024, 1945, (T, Hq, D // 32)) * rng.choice([-1, 1], (T, Hq, D // 32))
    return dict(q=q.astype(np.float16), pages=pages, table=table, lens=np.array(lens, np.int32), offsets=np.r_[0, np.cumsum(new)].astype(np.int32))


def whole_queries(c):
    """Queries that four summands hold exactly (multiples of 2^-10 below 2), and the scale that with log2 e is a power of two."""
    q = np.clip(np.round(c["q"].astype(np.float64) * 0.25 * 1024) / 1024, -1.9, 1.9)
    near = np.float32(0.125 / np.float32(1.44269504088896340736))
    scale = next(s for s in (near, np.nextafter(near, np.float32(0)), np.nextafter(near, np.float32(1))) if s * np.float32(1.44269504088896340736) == np.float32(0.125))
    return dict(c, q=q.astype(np.float16)), float(scale)
