"""Plain 64-bit numpy forms of the per-head norm with rotation and of the 8-bit KV cache (test infrastructure only)."""
from __future__ import annotations

import numpy as np

BLOCK, TOP, KMIN, KMAX = 32, 448.0, -40, 40


def e4m3_values() -> np.ndarray:
    """Value of every code 0..255: sign, 4 exponent bits (bias 7), 3 mantissa bits; 0x7f and 0xff are NaN."""
    out = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        v = (1 + m / 8) * 2.0 ** (e - 7) if e else m / 8 * 2.0 ** -6
        out[c] = np.nan if (c & 127) == 127 else (-v if c > 127 else v)
    return out


VALUES = e4m3_values()


def decode(codes: np.ndarray) -> np.ndarray:
    return VALUES[codes]


def encode(x: np.ndarray) -> np.ndarray:
    """Nearest code, ties to the even one, beyond the range to +-448 (infinities too), NaN to NaN; the sign of zero stays."""
    pos = VALUES[:127]                                    # codes 0..126 ascend
    a = np.minimum(np.abs(x), TOP)
    hi = np.clip(np.searchsorted(pos, np.nan_to_num(a)), 1, 126)
    lo = hi - 1
    mid = (pos[lo] + pos[hi]) / 2
    code = np.where(a < mid, lo, np.where(a > mid, hi, np.where(lo % 2 == 0, lo, hi)))
    code = np.where(np.isnan(x), 127, code)
    return (code + 128 * np.signbit(x)).astype(np.uint8)


def scale_exponent(amax: float) -> int:
    """Smallest k in [KMIN, KMAX] with amax <= 448 * 2^k (KMAX if there is none)."""
    for k in range(KMIN, KMAX + 1):
        if amax <= TOP * 2.0 ** k:
            return k
    return KMAX


def norm_rope(x: np.ndarray, gain, eps: float, pos: np.ndarray, theta: float) -> np.ndarray:
    """x [M, heads, dh] -> RMS norm over dh with gain (None: no norm), pairs (j, j + dh/2) turned by pos theta^(-2j/dh)."""
    x = x.astype(np.float64)
    if gain is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(gain, np.float64)
    half = x.shape[-1] // 2
    ang = pos[:, None].astype(np.float64) * theta ** (-2.0 * np.arange(half) / x.shape[-1])
    c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
    a, b = x[..., :half], x[..., half:]
    return np.concatenate([a * c - b * s, b * c + a * s], -1)


def write(codes: np.ndarray, scales: np.ndarray, rows, new: np.ndarray):
    """codes [blocks, heads, 32, dh], scales [blocks, heads] -> after the write.  rows: (t0, n, base, at, had) per row;
    new [M, heads, dh]."""
    codes, scales = codes.copy(), scales.astype(np.float64).copy()
    for t0, n, base, at, had in rows:
        if n == 0:
            continue
        for b in range(at // BLOCK, (at + n - 1) // BLOCK + 1):
            blk = base // BLOCK + b
            pos = b * BLOCK + np.arange(BLOCK)
            fresh = (pos >= at) & (pos < at + n)
            kept = (pos < had) & ~fresh
            for h in range(codes.shape[1]):
                x = decode(codes[blk, h]) * scales[blk, h]
                x[fresh] = new[t0 + pos[fresh] - at, h]
                valid = fresh | kept
                mag = np.abs(x[valid])
                amax = mag[np.isfinite(mag)].max(initial=0.0)
                k = scale_exponent(amax)
                codes[blk, h][valid] = encode(x[valid] / 2.0 ** k)
                scales[blk, h] = 2.0 ** k
    return codes, scales


def span(codes: np.ndarray, scales: np.ndarray, base: int, at: int, n: int) -> np.ndarray:
    """[n, heads, dh] values of cache positions [at, at + n) of the slab at `base`."""
    p = base + at + np.arange(n)
    return decode(codes[p // BLOCK, :, p % BLOCK]) * scales[p // BLOCK][:, :, None]


def attention(q: np.ndarray, k: np.ndarray, v: np.ndarray):
    """q [n, hq, dh], k / v [vis, hkv, dh] -> (out [n, hq, dh], sum_j p_j |v_j|, largest sum_d |q_d k_jd| / sqrt(dh),
    largest max_d |q_d| sum_d |k_jd| / sqrt(dh))."""
    n, hq, dh = q.shape
    out, mag, dot, flat = np.zeros(q.shape), np.zeros(q.shape), 0.0, 0.0
    if len(k) == 0:
        return out, mag, dot, flat
    g = hq // k.shape[1]
    for h in range(hq):
        z = q[:, h] @ k[:, h // g].T / np.sqrt(dh)
        dot = max(dot, float((np.abs(q[:, h]) @ np.abs(k[:, h // g]).T).max() / np.sqrt(dh)))
        flat = max(flat, float(np.abs(q[:, h]).max() * np.abs(k[:, h // g]).sum(1).max() / np.sqrt(dh)))
        p = np.exp(z - z.max(1, keepdims=True))
        p /= p.sum(1, keepdims=True)
        out[:, h], mag[:, h] = p @ v[:, h // g], p @ np.abs(v[:, h // g])
    return out, mag, dot, flat
