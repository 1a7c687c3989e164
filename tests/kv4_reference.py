"""Plain implementations of the 4-bit cache's operators in 64-bit numpy and plain Python (test infrastructure), written from include/thi.h:
the byte layout through explicit index loops, the codes by nearest search, the page operators row by row."""
from __future__ import annotations

import numpy as np

PAGE = 64
GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=np.float64)


def block_exponent(big: float) -> int:
    """The smallest e in [-23, 13] with big <= 7 * 2^e (13 if there is none)."""
    for e in range(-23, 14):
        if big <= 7.0 * 2.0 ** e:
            return e
    return 13


def quantise(x: np.ndarray):
    """x [..., D] fp64 -> (codes [..., D], scale bytes [..., D/32], values [..., D])."""
    shape = x.shape
    x = np.asarray(x, np.float64).reshape(-1, 32)
    codes, bytes_, vals = np.zeros(x.shape, np.uint8), np.zeros(len(x), np.uint8), np.zeros(x.shape)
    for i, row in enumerate(x):
        if not np.isfinite(row).all():
            bytes_[i], vals[i] = 255, np.nan
            continue
        e = block_exponent(np.abs(row).max())
        y = np.abs(row) / 2.0 ** e
        dist = np.abs(y[:, None] - GRID)
        order = np.array([0, 2, 4, 6, 1, 3, 5, 7])            # of two equally near codes the even one
        c = order[dist[:, order].argmin(-1)]
        codes[i] = c + 8 * np.signbit(row)
        bytes_[i] = e + 127
        vals[i] = np.where(np.signbit(row), -GRID[c], GRID[c]) * 2.0 ** e
    lead = shape[:-1]
    return codes.reshape(shape), bytes_.reshape(*lead, -1), vals.reshape(shape)


def value_of(code: int, byte: int) -> float:
    if byte == 255:
        return float("nan")
    v = GRID[code & 7] * 2.0 ** (int(byte) - 127)
    return -v if code & 8 else v


def places(pos: int, D: int):
    """(byte, shift) of each column's key and value codes and byte of each column's scales, within a head's block."""
    c = np.arange(D)
    key = pos * (D // 2) + c // 2
    key_scale = 32 * D + (c // 32) * 64 + (pos % 16) * 4 + pos // 16
    value = 34 * D + (c // 32) * 1024 + (pos % 16 // 4) * 256 + (c % 32 // 2) * 16 + (pos // 16) * 4 + pos % 4
    value_scale = 66 * D + (c // 32) * 64 + (pos % 16 // 4) * 16 + (pos // 16) * 4 + pos % 4
    return key, key_scale, value, value_scale


_TABLE = np.array([[value_of(c, b) for b in range(256)] for c in range(16)])


def store(pages: np.ndarray, slot: int, k: np.ndarray, v: np.ndarray) -> None:
    """k, v [Hkv, D] into pages [P, Hkv, 68 D] (uint8) at slot."""
    P, Hkv, block = pages.shape
    D = block // 68
    if not 0 <= slot < P * PAGE:
        return
    key, ks, value, vs = places(slot % PAGE, D)
    kc, kb, _ = quantise(k)
    vc, vb, _ = quantise(v)
    for h in range(Hkv):
        out = pages[slot // PAGE, h]
        for at, scale_at, codes, bytes_ in ((key, ks, kc[h], kb[h]), (value, vs, vc[h], vb[h])):
            out[at[0::2]] = codes[0::2] | codes[1::2] << 4
            out[scale_at[0::32]] = bytes_


def load(pages: np.ndarray, slot: int):
    """(k, v) [Hkv, D] fp64 at slot."""
    P, Hkv, block = pages.shape
    D = block // 68
    if not 0 <= slot < P * PAGE:
        return np.zeros((Hkv, D)), np.zeros((Hkv, D))
    key, ks, value, vs = places(slot % PAGE, D)
    shift = 4 * (np.arange(D) % 2)
    b = pages[slot // PAGE]
    return tuple(_TABLE[(b[:, at] >> shift) & 15, b[:, scale_at]] for at, scale_at in ((key, ks), (value, vs)))


def norm_rope(x, gamma, eps, position, theta):
    """x [H, D] -> RMSNorm per head, then neighbouring pairs turned, fp64."""
    x = np.asarray(x, np.float64)
    if gamma is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + float(np.float32(eps))) * np.asarray(gamma, np.float64)
    if theta is not None:
        ang = float(position) * np.asarray(theta, np.float64)
        z = (x[:, 0::2] + 1j * x[:, 1::2]) * (np.cos(ang) + 1j * np.sin(ang))
        x = np.stack([z.real, z.imag], -1).reshape(x.shape)
    return x


def attention(q, pages, table, lens, offsets, scale):
    """(out [T,Hq,D], S [T,Hq,D] = sum p |v|, E [T,Hq] = largest sum |q k| scale of a row) in fp64."""
    T, Hq, D = q.shape
    P, Hkv, _ = pages.shape
    q = np.asarray(q, np.float64)
    out, S, E = np.zeros(q.shape), np.zeros(q.shape), np.zeros((T, Hq))
    B, MP = table.shape
    offsets = np.arange(B + 1) if offsets is None else offsets
    for b in range(B):
        n = int(min(max(lens[b], 0), MP * PAGE))
        held = [(pos, load(pages, int(table[b, pos // PAGE]) * PAGE + pos % PAGE)) for pos in range(n) if 0 <= table[b, pos // PAGE] < P]
        if not held:
            continue
        at = np.array([h[0] for h in held])
        k, v = np.stack([h[1][0] for h in held]), np.stack([h[1][1] for h in held])
        m = int(offsets[b + 1] - offsets[b])
        for i in range(m):
            seen = at <= n - m + i
            if not seen.any():
                continue
            t = int(offsets[b]) + i
            for h in range(Hq):
                g = h // (Hq // Hkv)
                s = k[seen, g] @ q[t, h] * scale
                E[t, h] = (np.abs(k[seen, g]) @ np.abs(q[t, h])).max() * abs(scale)
                p = np.exp(s - s.max())
                p /= p.sum()
                out[t, h], S[t, h] = p @ v[seen, g], p @ np.abs(v[seen, g])
    return out, S, E


def attention_tolerance(y, S, E, D, positions):
    """How far a kernel may be off: one fp16 rounding of the result (half a step: 2^-11 of it, 2^-25 absolute); a weight rounded to fp16
    (2^-11 of it) and the exponential (2^-20 is more than the instruction is off); a score's fp32 sum over D products (2^-24 of the sum of
    their magnitudes each, and as much for the scaling and the distance to the maximum), which moves a weight and the total it is divided by; fp32 sums of
    `positions` terms."""
    score = (D + 8) * 2.0 ** -24 * E[..., None]
    return 2.0 ** -11 * np.abs(y) + 2.0 ** -25 + S * (2.0 ** -11 + 2.0 ** -20 + 2 * score + 2 * (positions + 64) * 2.0 ** -24)


def fork(refs, table, lens, parents, headroom, P):
    """Row by row, as include/thi.h words it: (refs, table, lens, info, copies [(src, dst)])."""
    R, MP = table.shape
    N = len(parents)
    free = [p for p in range(P) if refs[p] == 0]
    out, lens_out = np.full((N, MP), -1, np.int32), np.zeros(N, np.int32)
    refs_out, copies, taken, missing = refs.copy(), [], 0, 0
    seen = set()
    for i in range(N):
        p = int(parents[i])
        alive = 0 <= p < R
        n = min(max(int(lens[p]), 0), MP * PAGE) if alive else 0
        first = alive and p not in seen
        if alive:
            seen.add(p)
        lens_out[i] = n
        whole, used = n // PAGE, -(-n // PAGE)
        want = min(MP, -(-(n + max(0, int(headroom[i]) if headroom is not None else 0)) // PAGE))
        for j in range(max(used, want)):
            src = int(table[p, j]) if alive and 0 <= table[p, j] < P else -1
            if j < whole:
                out[i, j] = src
                continue
            partly = j < used
            if src >= 0 and first and refs[src] == 1:
                out[i, j] = src
            elif not partly or src >= 0:
                if free:
                    out[i, j] = free.pop(0)
                    taken += 1
                    if partly:
                        copies.append((src, int(out[i, j])))
                else:
                    missing += 1
    for t, by in ((table, -1), (out, 1)):
        for e in t.reshape(-1):
            if 0 <= e < P:
                refs_out[e] += by
    return refs_out, out, lens_out, (taken, missing), copies


def compact(refs, table, P):
    live = [p for p in range(P) if refs[p] > 0]
    L = len(live)
    holes = [p for p in range(L) if refs[p] <= 0]
    movers = [p for p in live if p >= L]
    to = {p: p for p in live}
    to.update(zip(movers, holes))
    out = np.array([to.get(int(e), -1) for e in table.reshape(-1)], np.int32).reshape(table.shape)
    refs_out = np.zeros_like(refs)
    for p in live:
        refs_out[to[p]] = refs[p]
    return refs_out, out, (L, len(movers)), list(zip(movers, holes))
