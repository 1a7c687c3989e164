"""Plain implementations of the fp16 cache's operators in 64-bit numpy and plain Python, written from include/thi.h, with how far a kernel may be off (test
infrastructure).

Tolerances.  With scores off by d_j and weights off by a factor of 1 + w at most, a result is sum p_j f_j v_j / sum p_j f_j with |ln f_j| <= d_j + w, so it is
off by no more than  sum p_j |v_j - y| (exp(d_j + w) - 1) exp(max d_j + w),  whatever the signs; and a weight p_j by a factor of exp(d_j + max d)."""
from __future__ import annotations

import numpy as np

PAGE = 64
ONE_SUMMAND, TWO_SUMMANDS = 2.0 ** -11, 2.0 ** -21


def places(pos: int, D: int):
    """Where in a head's block the D keys and the D values of a position lie."""
    keys, values = np.zeros(D, int), np.zeros(D, int)
    for c in range(D):
        keys[c] = ((((pos // 16) * (D // 32) + c // 32) * 4 + c % 32 // 8) * 16 + pos % 16) * 8 + c % 8
        values[c] = 64 * D + (((((pos // 32) * (D // 16) + c // 16) * 4 + pos % 16 // 4) * 16 + c % 16) * 2 + pos % 32 // 16) * 4 + pos % 4
    return keys, values


_PLACES = {D: [places(p, D) for p in range(PAGE)] for D in (64, 128)}


def store(pages: np.ndarray, slot: int, k: np.ndarray, v: np.ndarray) -> None:
    """pages [P, Hkv, 128 D] fp16; k, v [Hkv, D]."""
    P, Hkv, n = pages.shape
    if not 0 <= slot < P * PAGE:
        return
    at_k, at_v = _PLACES[n // 128][slot % PAGE]
    pages[slot // PAGE][:, at_k] = k
    pages[slot // PAGE][:, at_v] = v


def load(pages: np.ndarray, slot: int):
    at_k, at_v = _PLACES[pages.shape[2] // 128][slot % PAGE]
    page = pages[slot // PAGE]
    return page[:, at_k].astype(np.float64), page[:, at_v].astype(np.float64)


def append(qkv, q_gamma, k_gamma, eps, positions, theta, Hq, Hkv, D):
    """(queries, keys, values, tolerances of queries and keys) [T, heads, D] in 64 bits."""
    T = len(qkv)
    x = qkv[:, : (Hq + 2 * Hkv) * D].astype(np.float64).reshape(T, -1, D)

    def one(y, gamma):
        size = np.abs(y)
        if gamma is not None:
            with np.errstate(all="ignore"):
                r = 1 / np.sqrt((y * y).mean(-1, keepdims=True) + float(np.float32(eps)))
                y, size = y * r * gamma.astype(np.float64), size * r * np.abs(gamma.astype(np.float64))
        a, b = y[..., 0::2], y[..., 1::2]
        if theta is not None:
            with np.errstate(all="ignore"):
                angle = positions.astype(np.float64)[:, None, None] * theta.astype(np.float64)
                y = np.stack([a * np.cos(angle) - b * np.sin(angle), b * np.cos(angle) + a * np.sin(angle)], -1).reshape(y.shape)
        pair = np.repeat(size[..., 0::2] + size[..., 1::2], 2, -1)
        # a sum of D squares, its root, two products; sine and cosine to 2^-22; two products and a sum: some 2^-20 of the pair; then the rounding to fp16
        return y, 2.0 ** -11 * np.abs(y) + 2.0 ** -25 + (D / 8 + 24) * 2.0 ** -24 * pair

    q, tq = one(x[:, :Hq], q_gamma)
    k, tk = one(x[:, Hq: Hq + Hkv], k_gamma)
    return q, k, x[:, Hq + Hkv:], tq, tk


def attention(c, scale, window=0, sinks=0, weight=TWO_SUMMANDS, weights_in=None):
    """(out, tolerance [T, Hq, D]; weights, tolerance [B, Hkv, 64 MP], with NaN where nothing is written).

    Roundings that are counted: sums of D products in 32 bits with the distance to the maximum (2^-24 of the magnitudes' sum for each product, 2^-18 for the rest), the
    exponential (2^-20), a weight (`weight` of it; 2^-33 where that is below what fp16 holds), sums of the positions in 32 bits, the result
    (2^-11 of it, or 2^-25)."""
    T, Hq, D = c["q"].shape
    Hkv, P, (B, MP) = c["pages"].shape[1], len(c["pages"]), c["table"].shape
    q = c["q"].astype(np.float64)
    out, tol = np.zeros((T, Hq, D)), np.full((T, Hq, D), 2.0 ** -25)
    w, wtol = np.full((B, Hkv, MP * PAGE), np.nan), np.zeros((B, Hkv, MP * PAGE))
    for b in range(B):
        n = int(min(max(int(c["lens"][b]), 0), MP * PAGE))
        m = int(c["offsets"][b + 1] - c["offsets"][b])
        before = max(0, n - m)
        w[b, :, :n] = 0
        if weights_in is not None:
            w[b, :, :before] = weights_in[b, :, :before]
        at = np.array([p for p in range(n) if 0 <= c["table"][b, p // PAGE] < P], int)
        kv = [load(c["pages"], int(c["table"][b, p // PAGE]) * PAGE + p % PAGE) for p in at]
        k, v = (np.stack([x[i] for x in kv]) if kv else np.zeros((0, Hkv, D)) for i in range(2))
        got, off = np.zeros((Hkv, n)), np.zeros((Hkv, n))
        for i in range(m):
            here = n - m + i
            seen = at <= here
            if window:
                seen &= (at > here - window) | (at < sinks)
            if not seen.any():
                continue
            t = int(c["offsets"][b]) + i
            for h in range(Hq):
                g = h // (Hq // Hkv)
                kk, vv, x = k[seen, g], v[seen, g], q[t, h]
                with np.errstate(all="ignore"):
                    s = kk @ x * scale
                    p = np.exp(s - s.max())
                    p = p / p.sum()
                    d = abs(scale) * (np.abs(kk) @ np.abs(x)) * (D + 8) * 2.0 ** -24 + 2.0 ** -18 + 2.0 ** -20
                    y = p @ vv
                    e = d + weight
                    out[t, h] = y
                    tol[t, h] += (2.0 ** -11 * np.abs(y) + (p * np.expm1(e)) @ np.abs(vv - y) * np.exp(e.max()) + 2.0 ** -33 * np.abs(vv).sum(0)
                                  + 2 * (len(p) + 64) * 2.0 ** -24 * (p @ np.abs(vv)))
                    got[g, at[seen]] += p
                    off[g, at[seen]] += p * np.expm1(d + d.max() + (len(p) + 64) * 2.0 ** -24)
        w[b, :, :n] += got
        wtol[b, :, :n] = off + (m * Hq // Hkv + 2) * 2.0 ** -24 * got + 2.0 ** -23 * np.abs(w[b, :, :n]) + 1e-30
    return out, tol, w, wtol


def evict(c, budget, sinks, recent, headroom):
    """What thi_kv16_evict leaves: dict(refs, table, lens, weights (NaN where nothing is written), info, pages)."""
    table, refs, lens = c["table"], c["refs"], c["lens"]
    (R, MP), P, (L, _, Hkv, n_head) = table.shape, len(refs), c["pages"].shape
    D = n_head // 128
    free = [p for p in range(P) if refs[p] == 0]
    out = dict(refs=refs.copy(), table=table.copy(), lens=lens.copy(), weights=np.full(c["weights"].shape, np.nan, np.float32), pages=c["pages"].copy())
    used, stop, moved, stayed = 0, False, 0, 0
    for b in range(R):
        n = int(min(max(int(lens[b]), 0), MP * PAGE))
        out["lens"][b] = n
        live = [p for p in range(n) if 0 <= table[b, p // PAGE] < P]
        if n > budget:
            kept = min(budget, len(live))
            need = min(MP, -(-(kept + headroom) // PAGE))
            if stop or used + need > len(free):
                stop, stayed = True, stayed + 1
        if n <= budget or stop:
            out["weights"][:, b, :, :n] = c["weights"][:, b, :, :n]
            continue
        moved += 1
        fresh = free[used: used + need]
        used += need
        for e in table[b]:
            if 0 <= e < P:
                out["refs"][e] -= 1
        out["refs"][fresh] += 1
        out["table"][b] = -1
        out["table"][b, :need] = fresh
        out["lens"][b] = kept
        for layer in range(L):
            for g in range(Hkv):
                w = c["weights"][layer, b, g]
                guarded = [p for p in live if p < sinks or p >= n - recent]
                others = sorted((p for p in live if not (p < sinks or p >= n - recent)), key=lambda p: (np.isnan(w[p]), -w[p] if not np.isnan(w[p]) else 0, p))
                keep = sorted(guarded + others[: kept - len(guarded)])
                for i, p in enumerate(keep):
                    from_k, from_v = _PLACES[D][p % PAGE]
                    to_k, to_v = _PLACES[D][i % PAGE]
                    src, dst = c["pages"][layer, table[b, p // PAGE], g], out["pages"][layer, fresh[i // PAGE], g]
                    dst[to_k], dst[to_v] = src[from_k], src[from_v]
                    out["weights"][layer, b, g, i] = w[p]
    out["info"] = np.array([moved, stayed], np.int32)
    return out
