"""The 8-bit cache and the log probabilities in 64 bits (numpy), row by row from their definitions."""
import numpy as np

QMAX = {"e4m3": 448.0, "int8": 127.0}
EXP_MIN, EXP_MAX = -117, 119


def e4m3_values():
    """The value of each of the 256 codes (0x7f and 0xff are NaN)."""
    c = np.arange(256)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e > 0, np.ldexp(1.0 + m / 8.0, e - 7), np.ldexp(m / 8.0, -6))
    v = np.where(c & 128, -v, v)
    v[[0x7F, 0xFF]] = np.nan
    return v


def to_codes(y, fmt):
    """y (64 bits, in units of the scale) to code bytes: the nearest value, ties to the even code, saturating."""
    y = np.asarray(y, np.float64)
    if fmt == "int8":
        return np.clip(np.rint(y), -127, 127).astype(np.int8).view(np.uint8)
    mag = np.abs(np.clip(y, -448.0, 448.0))
    _, ex = np.frexp(np.maximum(mag, 2.0 ** -6))
    step = np.ldexp(1.0, ex - 4)
    r = np.rint(mag / step) * step
    grid = e4m3_values()[:127]
    code = np.searchsorted(grid, r)
    assert np.array_equal(grid[code], r)
    return (code | np.where(np.signbit(y), 128, 0)).astype(np.uint8)


def values(codes, fmt):
    return codes.view(np.int8).astype(np.float64) if fmt == "int8" else e4m3_values()[codes]


def least_exp(amax, fmt):
    e = EXP_MIN
    while e < EXP_MAX and amax > QMAX[fmt] * 2.0 ** e:
        e += 1
    return e


def append(codes, exps, rows, L, fmt, block):
    """rows [n, H, D] (64 bits) behind position L of codes [Lmax, H, D] uint8 / exps [NB, H], in place; the new length."""
    Lmax, H, _ = codes.shape
    n = min(len(rows), Lmax - L)
    rows = rows[:n]
    for h in range(H):
        at = 0
        while at < n:
            blk = (L + at) // block
            lo, hi = blk * block, min((blk + 1) * block, L + n)
            x = rows[at:hi - L, h]
            x = np.where(np.isnan(x), 0.0, x)
            e = least_exp(np.abs(x).max(), fmt)
            if lo < L:
                e = max(e, int(exps[blk, h]))
                if e > exps[blk, h]:
                    codes[lo:L, h] = to_codes(np.ldexp(values(codes[lo:L, h], fmt), int(exps[blk, h]) - e), fmt)
            codes[L + at:hi, h] = to_codes(np.ldexp(x, -e), fmt)
            exps[blk, h] = e
            at = hi - L
    return L + n


def attention(q, K, V, Ld, dk, dv, see, scale):
    """One sequence: q [N,Hq,D], K/V [rows,H,D] (values), Ld visible rows, see [N,N] bool
    -> out [N,Hq,D], sum p |v| [N,Hq,D], the largest scale * sum |q k| of a visible key [N,Hq,1]."""
    N, Hq, D = q.shape
    H = K.shape[1]
    G = Hq // H
    out, mean_abs, size = np.zeros((N, Hq, D)), np.zeros((N, Hq, D)), np.zeros((N, Hq, 1))
    for h in range(Hq):
        c = h // G
        k, v = np.concatenate((K[:Ld, c], dk[:, c])), np.concatenate((V[:Ld, c], dv[:, c]))
        s = q[:, h] @ k.T * scale
        s[:, Ld:][~see] = -np.inf
        seen = np.isfinite(s).any(1)
        size[:, h, 0] = np.where(np.isfinite(s), np.abs(q[:, h]) @ np.abs(k).T * scale, 0.0).max(1, initial=0.0)
        m = np.where(seen, s.max(1, initial=-np.inf), 0.0)
        p = np.exp(s - m[:, None])
        p /= np.where(seen, p.sum(1), 1.0)[:, None]
        out[:, h], mean_abs[:, h] = p @ v, p @ np.abs(v)
    return out, mean_abs, size


def logprobs(x, t, k):
    """(log p_t, entropy, top indices, their log p) of one row."""
    x = np.asarray(x, np.float64)
    m = x.max()
    lse = m + np.log(np.exp(x - m).sum())
    lp = x - lse
    p = np.exp(lp)
    order = np.lexsort((np.arange(len(x)), -x))[:k]
    return lp[t], -(p[p > 0] * lp[p > 0]).sum(), order, lp[order]
