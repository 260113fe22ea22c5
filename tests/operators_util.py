"""64-bit references of the operators of a beam search on 4-bit operands, in numpy.

Quantisation is a definition (no rounding freedom), so codes, scales and values are compared bit for bit.
"""
from __future__ import annotations

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}


def up(n, to):
    return -(-n // to) * to


def quantize(x):
    """x [rows, cols] float64 -> codes [rows, cols] (0..15), biased exponents [rows, blocks], values."""
    rows, cols = x.shape
    nb = -(-cols // 32)
    b = np.zeros((rows, nb * 32))
    b[:, :cols] = x
    b = b.reshape(rows, nb, 32)
    finite = np.isfinite(b).all(-1)
    f = np.where(finite[..., None], b, 0.0)
    top = np.abs(f).max(-1)
    m, e = np.frexp(top)                       # top = m 2^e, m in [0.5, 1); 6 = 0.75 * 2^3
    k = np.where(top > 0, np.where(m > 0.75, e - 2, e - 3), 0)
    k = np.clip(k, -127, 127)
    t = np.abs(f) * np.exp2(-k.astype(np.float64))[..., None]
    # nearest of the grid, ties to the even code
    d = np.abs(t[..., None] - GRID)
    best = d.min(-1, keepdims=True)
    near = d == best
    lo = near.argmax(-1)
    hi = 7 - near[..., ::-1].argmax(-1)
    mag = np.where((lo != hi) & (lo % 2 == 1), hi, lo)
    code = mag | (np.signbit(f).astype(np.int64) << 3)
    val = np.where(np.signbit(f), -GRID[mag], GRID[mag]) * np.exp2(k.astype(np.float64))[..., None]
    val = np.where(finite[..., None], val, np.nan)
    code = np.where(finite[..., None], code, 0)
    scale = np.where(finite, k + 127, 255)
    return code.reshape(rows, -1)[:, :cols], scale, val.reshape(rows, -1)[:, :cols]


def layout(code, scale):
    """The bytes of codes and scales as the library lays them out."""
    rows, cols = code.shape
    R, Cc, Sc = up(rows, 16), up(cols, 128), up(cols, 512)
    c = np.zeros((R, Cc), np.uint8)
    c[:rows, :cols] = code
    s = np.full((R, Sc // 32), 127, np.uint8)
    s[:rows, :scale.shape[1]] = scale
    codes = np.zeros((R // 16, Cc // 128, 1024), np.uint8)
    scales = np.zeros((R // 16, Sc // 512, 256), np.uint8)
    for b in range(4):
        for r in range(16):
            for i in range(16):
                at = (b * 16 + r) * 16 + i
                codes[:, :, at] = c[r::16, b * 32 + 2 * i::128] | c[r::16, b * 32 + 2 * i + 1::128] << 4
            for t in range(4):
                scales[:, :, (b * 16 + r) * 4 + t] = s[r::16, t * 4 + b::16]
    return codes.reshape(-1), scales.reshape(-1)


def totals(logits, scores, finished=None, end=0):
    """[B, beams, V] float64 scores of all candidates; -inf where there is none."""
    x, s = logits.astype(np.float64), scores.astype(np.float64)[..., None]
    with np.errstate(all="ignore"):
        top = x.max(-1, keepdims=True)
        # (beside a largest logit of 1e38 the logarithm would be lost: the difference of the logits comes first)
        t = (s - np.log(np.exp(x - top).sum(-1, keepdims=True))) + (x - top)
    t = np.where(np.isnan(t), -np.inf, t)
    if finished is not None:
        f = np.full_like(t, -np.inf)
        f[:, :, end] = np.where(np.isnan(scores), -np.inf, scores)
        t = np.where(finished.astype(bool)[..., None], f, t)
    return t


def select(t, x, n):
    """(scores, tokens, parents) of the n best: by total, those of one beam by logit, ties by the lower place."""
    B, beams, V = t.shape
    out_s = np.full((B, n), -np.inf)
    out_v, out_k = np.full((B, n), -1), np.full((B, n), -1)
    for b in range(B):
        flat = t[b].reshape(-1)
        at = np.flatnonzero(flat > -np.inf)
        order = np.lexsort((at, -x[b].reshape(-1)[at].astype(np.float64) if beams == 1 else np.zeros(len(at)), -flat[at]))
        at = at[order][:n]
        out_s[b, :len(at)], out_v[b, :len(at)], out_k[b, :len(at)] = flat[at], at % V, at // V
    return out_s, out_v, out_k


# A sum over the vocabulary in 32-bit exponentials: relative error of a term 2^-22 at most (an argument rounded to
# 2^-24 of at most 88 only where the term itself is below e^-88, and one unit of the exponential), so the logarithm is
# off by less than 2^-22, and a score by that: candidates of different hypotheses nearer than twice that may change
# places.
GAP = 2.0 ** -21


def check_selection(got, t, x, n):
    """got: (scores, tokens, parents) as numpy; t, x: totals and logits in 64 bits."""
    s, v, k = got
    ws, wv, wk = select(t, x, n)
    B, beams, V = t.shape
    assert s.shape == v.shape == k.shape == (B, n)
    for b in range(B):
        there = ws[b] > -np.inf
        assert np.array_equal(np.isfinite(s[b]), there), (b, s[b], ws[b])
        assert (v[b][~there] == -1).all() and (k[b][~there] == -1).all() and (s[b][~there] == -np.inf).all()
        tol = GAP + HALF_STEP["f32"] * np.abs(ws[b][there])
        assert (np.abs(s[b][there] - ws[b][there]) <= tol).all(), (b, s[b], ws[b])
        if np.array_equal(v[b], wv[b]) and np.array_equal(k[b], wk[b]):
            continue
        # other candidates in these places: as good to within the gap, none twice, and exactly in order within a beam
        m = int(there.sum())
        assert len(set(zip(k[b][:m], v[b][:m]))) == m
        assert (np.abs(t[b][k[b][:m], v[b][:m]] - ws[b][:m]) <= GAP).all(), (b, v[b], wv[b])
        for h in set(k[b][:m]):
            mine = [(-float(x[b, h, c]), int(c)) for c in v[b][:m][k[b][:m] == h]]
            assert mine == sorted(mine), (b, h)
