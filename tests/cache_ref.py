"""Plain references of the operators of a quantised paged cache: NumPy in 64 bits,
from the definitions in include/asymspec_cache.h."""

import numpy as np


def levels(bits):
    """What the codes without a sign stand for (e4m3: without the last, which is no number)."""
    exp, man, bias = (4, 3, 7) if bits == 8 else (2, 1, 1)
    got = []
    for e in range(1 << exp):
        for m in range(1 << man):
            got.append(2.0 ** (1 - bias) * m / (1 << man) if e == 0 else 2.0 ** (e - bias) * (1 + m / (1 << man)))
    return np.array(got[:-1] if bits == 8 else got)


def encode(x, bits):
    """(codes one a byte [..., D], scale bytes [..., D / 32]) of fp64 values."""
    lv = levels(bits)
    x = x.reshape(x.shape[:-1] + (-1, 32))
    most = np.abs(x).max(-1)
    bad = ~np.isfinite(x).all(-1) | (most > lv[-1] * 2.0 ** (119 if bits == 8 else 125))
    x = np.where(bad[..., None], 0.0, x)
    most = np.where(bad, 0.0, most)
    e = np.full(most.shape, -100)
    for k in range(-99, 128):
        e = np.where(most > lv[-1] * 2.0 ** (k - 1), k, e)
    y = np.abs(x) / 2.0 ** e[..., None].astype(np.float64)
    hi = np.searchsorted(lv, y).clip(0, len(lv) - 1)
    lo = (hi - 1).clip(0)
    up, down = lv[hi] - y, y - lv[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    code = code + (128 if bits == 8 else 8) * np.signbit(x)
    code = np.where(bad[..., None], 0, code)
    return code.reshape(code.shape[:-2] + (-1,)).astype(np.uint8), np.where(bad, 255, e + 127).astype(np.uint8)


def packed(codes, bits):
    return codes if bits == 8 else (codes[..., 0::2] | (codes[..., 1::2] << 4)).astype(np.uint8)


def decode(data, scales, bits):
    """fp64 values of packed codes."""
    lv = np.append(levels(bits), [np.nan] if bits == 8 else [])
    if bits == 4:
        data = np.stack([data & 15, data >> 4], -1).reshape(data.shape[:-1] + (-1,))
    half = 128 if bits == 8 else 8
    v = np.where(data >= half, -1.0, 1.0) * lv[data % half]
    s = np.where(scales > (246 if bits == 8 else 252), np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return v * np.repeat(s, 32, -1)


def write(cache, k, v, slots, bits):
    """Into the four arrays, in place; k, v: fp64 [tokens, heads, D]."""
    N, H, S = cache[0].shape[:3]
    for part, x in ((0, k), (2, v)):
        codes, scales = encode(x, bits)
        data = packed(codes, bits)
        for t, s in enumerate(slots):
            if 0 <= s < N * S:
                cache[part][s // S, :, s % S] = data[t]
                cache[part + 1][s // S, :, s % S] = scales[t]


def rows_of(cache, part, table, positions, bits):
    """(fp64 values [n, heads, D], which positions there are) of a request's positions."""
    N, H, S = cache[0].shape[:3]
    D = cache[1].shape[3] * 32
    out = np.zeros((len(positions), H, D))
    ok = np.zeros(len(positions), bool)
    for i, p in enumerate(positions):
        page = p // S
        if p >= 0 and page < len(table) and 0 <= table[page] < N:
            out[i] = decode(cache[part][table[page], :, p % S], cache[part + 1][table[page], :, p % S], bits)
            ok[i] = True
    return out, ok


def read(cache, table, lengths, width, first, bits):
    got = []
    for part in (0, 2):
        rows = []
        for b in range(len(table)):
            p = (0 if first is None else int(first[b])) + np.arange(width)
            p = np.where(p < lengths[b], p, -1)
            rows.append(rows_of(cache, part, table[b], p, bits)[0])
        got.append(np.stack(rows))
    return got


def attend(q, cache, table, lengths, new_tokens, scale, window, bits):
    """(out, lse, bound on out's error, on lse's) in fp64 for q [B, R, H, D].

    The bounds count fp32 roundings, u = 2^-24.  A score sums D exact products, and the
    partial sums of an instruction may be cut rather than rounded: it is off by at
    most 2 (D + 4) u sum |q k|, and times the scale by as much more.  A probability is
    off by that, by its exponent's rounding (2 u of it), by the exponential (2 u) and by
    the parts it is split into; sums of n terms by 2 n u of the terms' magnitudes.

    Bounds are infinite, and the row may be anything, where a product's or a sum's
    magnitude passes 2^127 or a scaled score's times log2 e does: fp32 ends at 2^128, so
    that an evaluation there may meet an infinity, and the difference of two."""
    B, R, H, D = q.shape
    N, Hk, S = cache[0].shape[:3]
    u = 2.0 ** -24
    out, lse = np.zeros((B, R, H, D)), np.full((B, R, H), -np.inf)
    err, lerr = np.zeros((B, R, H, D)), np.zeros((B, R, H))
    for b in range(B):
        n = max(0, int(lengths[b]))
        fresh = R if new_tokens is None else int(np.clip(new_tokens[b], 0, R))
        if fresh == 0:
            continue
        lo, hi = (max(0, n - window + 1) if window else 0), min(n + fresh, table.shape[1] * S)
        p = np.arange(lo, max(lo, hi))
        k, ok = rows_of(cache, 0, table[b], p, bits)
        v, _ = rows_of(cache, 2, table[b], p, bits)
        for r in range(fresh):
            see = ok & (p <= n + r) & ((p > n + r - window) if window else True)
            if not see.any():
                continue
            for h in range(H):
                kh, vh = k[see, h // (H // Hk)], v[see, h // (H // Hk)]
                with np.errstate(all="ignore"):
                    t = kh @ q[b, r, h] * scale
                    far = np.abs(kh) @ np.abs(q[b, r, h]) * abs(scale)
                    m = np.nanmax(t) if not np.isnan(t).all() else 0.0
                    w = np.exp(t - m)
                    w = np.where(np.isnan(t), np.nan, w)
                    out[b, r, h] = (w[:, None] * vh).sum(0) / w.sum()
                    lse[b, r, h] = m + np.log(w.sum())
                    rel = 2 * (D + 8) * u * far + 2 * u * np.abs(t - m) + 4 * u + (2.0 ** -17 if q.dtype == np.float32 else u)
                    share = w / w.sum()
                    many = 2 * see.sum() * u + 8 * u
                    err[b, r, h] = (share * (rel + (share * rel).sum() + many)) @ np.abs(vh) + 2 * many * np.abs(out[b, r, h])
                    raw = np.abs(kh) @ np.abs(q[b, r, h])
                    top = max(np.nanmax(raw, initial=0), 1.5 * np.nanmax(far, initial=0), np.nanmax(np.abs(vh), initial=0) * 256 * see.sum())
                    if top > 2.0 ** 127:
                        err[b, r, h], lerr[b, r, h] = np.inf, np.inf
                        continue
                    lerr[b, r, h] = (share * rel).sum() + many + 4 * u * abs(lse[b, r, h]) + 2 * u * abs(m)
    return out, lse, err, lerr
