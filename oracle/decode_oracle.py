"""64-bit reference of the operators between a hidden state and a committed token: 8-bit row codes, products of codes, the
rules of constrained decoding and the confidence under them.  Plain numpy; test infrastructure only."""
from __future__ import annotations

import numpy as np

LEAST_SCALE = 2.0 ** -126


def quant(x, gain=None, eps=0.0):
    """(y, codes as floats, scale) of rows x in float64: y = x or its RMS norm; the scale is the fp32
    product of max |y| and 1 / 127, the codes are the exact quotients rounded half to even.  Rows with an infinite or NaN element: scale NaN, codes 0."""
    x = np.asarray(x, np.float64)
    with np.errstate(all="ignore"):
        y = x if gain is None else x * gain / np.sqrt((x * x).mean(1, keepdims=True) + eps)
        scale = np.maximum((np.abs(y).max(1).astype(np.float32) * np.float32(1 / 127)).astype(np.float64), LEAST_SCALE)
        bad = ~np.isfinite(x).all(1)
        codes = np.rint(y / scale[:, None])
    codes[bad] = 0
    scale[bad] = np.nan
    return y, codes, scale


def gemm(a, sa, w, sw):
    """Products of codes and scales: the integer sums are exact in 64 bits."""
    acc = np.asarray(a, np.float64) @ np.asarray(w, np.float64).T
    return acc * np.asarray(sw, np.float64) * np.asarray(sa, np.float64)[:, None]


def rules(z, row_req, vocab, mask_id=-1, ctx=None, begin=None, gen=None, end=None, repetition=None, presence=None,
          frequency=None, bias_at=None, bias_tok=None, bias_val=None, allowed=None, row_mask=None):
    """The logits z (fp32 values [rows, vocab]) after the rules, with every step rounded to fp32 as the definition has it."""
    one = np.float32
    y = np.array(z, np.float32)
    with np.errstate(all="ignore"):
        for r, i in enumerate(row_req):
            if i >= 0 and ctx is not None:
                count, seen = {}, set()
                for k in range(begin[i], end[i]):
                    t = int(ctx[k])
                    if t == mask_id or not 0 <= t < vocab:
                        continue
                    seen.add(t)
                    if k >= gen[i]:
                        count[t] = count.get(t, 0) + 1
                rho = one(1 if repetition is None else repetition[i])
                alpha, phi = one(0 if presence is None else presence[i]), one(0 if frequency is None else frequency[i])
                for t in seen:
                    y[r, t] = y[r, t] / rho if y[r, t] > 0 else y[r, t] * rho
                    if t in count:
                        y[r, t] = y[r, t] - (phi * one(count[t]) + alpha)
            if i >= 0 and bias_at is not None:
                for k in range(bias_at[i], bias_at[i + 1]):
                    y[r, bias_tok[k]] = y[r, bias_tok[k]] + one(bias_val[k])
            if allowed is not None and row_mask[r] >= 0:
                bits = np.unpackbits(np.ascontiguousarray(allowed[row_mask[r]]).view(np.uint8), bitorder="little")[:vocab]
                y[r, bits == 0] = -np.inf
            if mask_id >= 0:
                y[r, mask_id] = -np.inf
    return y


def confidence(y):
    """(tok, conf) of rows y: lowest argmax of the numbers, exp(max - logsumexp) in 64 bits; -1 and 0 where nothing is left."""
    tok, conf = [], []
    for row in np.asarray(y, np.float64):
        nan, real = np.isnan(row).any(), np.where(np.isnan(row), -np.inf, row)
        top = real.max()
        if top == -np.inf:
            tok.append(-1)
            conf.append(np.nan if nan else 0.0)
            continue
        tok.append(int(np.argmax(real)))
        with np.errstate(all="ignore"):
            share = np.where(real == top, 1.0, np.exp(real - top)).sum() if np.isfinite(top) else (real == top).sum()
        conf.append(np.nan if nan else 1.0 / share)
    return np.array(tok), np.array(conf)
