"""Whether a selection is one of those that the definition allows, whatever the roundings of its sums.

The order of an utterance's candidates is by score, then hypothesis, then logit, then token.  Scores of one hypothesis
rise with its logits in every rounding, so whatever it puts among the winners are its own first ones, by logit and then token.
Between hypotheses only what the sums may be off by is open, and nothing at all where a score is so large that logits
are lost in it: there the scores of hypotheses are what they were before."""
from __future__ import annotations

import numpy as np

from operators_util import HALF_STEP, totals

UNIT = 2.0 ** -24


def log_error(V):
    """What the logarithm of a sum over V logits may be off by.  A term exp(x - ref), d below the row's largest one, is off by
    at most (relative; in units of 2^-24)
      2 d + 1      rounded arguments of the exponential: a difference rounded by half a step, at most d units, times log2(e), rounded by as much; or one
                   rounding of x log2(e) - shift, at most d + 0.35
      0.23 d + 0.1 log2(e) as a 32-bit constant: 1.34e-8 d
      2            the exponential: one unit in the last place of a value in (0.5, 2)
    and sums of up to eight of them before they go to 64 bits by at most 8.  The logarithm is off by the mean of that with
    the terms' shares p = exp(-d) / Z of their sum Z, and the mean of d is at most ln V: the entropy of the shares is
    sum p d + ln Z, at most ln V, and Z is at least the largest term, 1."""
    return (2.25 * np.log(V) + 11.5) * UNIT


def check_order(got, logits, scores, n, finished=None, end=0):
    """got: (scores, tokens, parents); logits [B, beams, V] and scores [B, beams] in 64 bits, of the values that the call was given."""
    s, v, k = got
    B, beams, V = logits.shape
    t = totals(logits, scores, finished, end)
    done = np.zeros((B, beams), bool) if finished is None else finished.astype(bool)
    off = log_error(V)
    assert s.shape == v.shape == k.shape == (B, n)
    for b in range(B):
        m = min(n, int((t[b] > -np.inf).sum()))
        assert (v[b, m:] == -1).all() and (k[b, m:] == -1).all() and (s[b, m:] == -np.inf).all(), (b, m, v[b], k[b], s[b])
        if m == 0:
            continue
        vb, kb = v[b, :m], k[b, :m]
        assert (vb >= 0).all() and (vb < V).all() and (kb >= 0).all() and (kb < beams).all(), (b, vb, kb)
        mine = t[b, kb, vb]
        assert (mine > -np.inf).all(), (b, vb, kb)
        # roundings of sums in 64 bits: a few steps of the numbers that are added
        live = ~done[b] & (t[b] > -np.inf).any(-1)
        x = np.where(t[b] > -np.inf, logits[b], 0.0)
        reach = np.where(live, np.abs(x).max(-1) + np.log(V) + 1, 0.0)
        size = np.abs(np.where(np.isfinite(scores[b]), scores[b], 0.0)) + 2 * reach
        slack = np.where(live, off, 0.0) + 8 * np.spacing(size)
        # (a hypothesis whose score does not change by all that its logits are away from it; an ended one's is its own)
        fixed = done[b] | (8 * reach < np.spacing(np.abs(scores[b])) / 2)
        tol = slack[kb] + HALF_STEP["f32"] * np.abs(mine) * 1.01
        assert (np.abs(s[b, :m].astype(np.float64) - mine) <= tol).all(), (b, s[b], mine)
        assert (np.diff(s[b, :m]) <= 0).all(), (b, s[b])
        last = mine[-1]
        for h in range(beams):
            took = vb[kb == h]
            if done[b, h]:
                assert list(took) in ([], [end]), (b, h, took)
                first = np.array([end] if np.isfinite(t[b, h, end]) else [], int)
            else:
                first = np.flatnonzero(t[b, h] > -np.inf)
                first = first[np.lexsort((first, -logits[b, h, first]))][:n + 1]
            assert np.array_equal(took, first[:len(took)]), (b, h, took, first)
            # what it has next would not have been among the winners
            if len(took) < len(first) and h != kb[-1]:
                rest = t[b, h, first[len(took)]]
                if fixed[h] and fixed[kb[-1]]:
                    assert (rest, -h) < (last, -kb[-1]), (b, h, rest, last)
                else:
                    assert rest <= last + slack[h] + slack[kb[-1]], (b, h, rest, last)
        for i in range(m - 1):
            if kb[i] == kb[i + 1]:
                continue
            if fixed[kb[i]] and fixed[kb[i + 1]]:
                assert (mine[i], -kb[i]) > (mine[i + 1], -kb[i + 1]), (b, i, vb, kb)
            else:
                assert mine[i] >= mine[i + 1] - slack[kb[i]] - slack[kb[i + 1]], (b, i, vb, kb)
