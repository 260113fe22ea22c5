"""The check of a selection's order against right and wrong selections made by hand, no GPU needed."""
import numpy as np
import pytest

from operators_order import check_order
from operators_util import totals


def _best(x, scores, n, finished=None, end=0):
    """The definition: by score, hypothesis, logit, token."""
    t = totals(x, scores, finished, end)
    B, beams, V = t.shape
    s, v, k = np.full((B, n), -np.inf), np.full((B, n), -1), np.full((B, n), -1)
    for b in range(B):
        at = np.flatnonzero(t[b].reshape(-1) > -np.inf)
        logit = np.where((finished[b] if finished is not None else np.zeros(beams, bool))[:, None], 0.0, x[b]).reshape(-1)
        order = np.lexsort((at % V, -logit[at], at // V, -t[b].reshape(-1)[at]))[:n]
        at = at[order]
        s[b, :len(at)], v[b, :len(at)], k[b, :len(at)] = t[b].reshape(-1)[at], at % V, at // V
    return s.astype(np.float32), v, k


def _wrong(got, x, scores, n, *rest):
    with pytest.raises(AssertionError):
        check_order(got, x, scores, n, *rest)


@pytest.mark.parametrize("seed", range(4))
def test_right_selections_pass_and_wrong_ones_do_not(seed):
    g = np.random.default_rng(seed)
    B, beams, V, n = 3, 4, 60, 7
    x = g.standard_normal((B, beams, V)) * 3
    x[:, :, 7] = x[:, :, 5]
    x[1, 2] = -np.inf
    x[2, 3, 9] = np.nan
    scores = -g.random((B, beams))
    scores[0, 3] = -np.inf
    done = g.random((B, beams)) < 0.3
    for rest in ((), (done, 11)):
        s, v, k = _best(x, scores, n, *rest)
        check_order((s, v, k), x, scores, n, *rest)
        for i in range(n - 1):
            for b in range(B):
                swap = np.arange(n)
                swap[[i, i + 1]] = i + 1, i
                w = [a.copy() for a in (s, v, k)]
                for a, o in zip(w[1:], (v, k)):
                    a[b] = o[b, swap]
                if not all(np.array_equal(a, o) for a, o in zip(w, (s, v, k))):      # (two places without a candidate)
                    _wrong(tuple(w), x, scores, n, *rest)
        for change in (lambda s, v, k: (s + 1e-4, v, k), lambda s, v, k: (s, v * 0 + v[:, :1], k), lambda s, v, k: (s[:, :-1], v[:, :-1], k[:, :-1]),
                       lambda s, v, k: (s, np.where(k == k[0, 0], (v + 1) % V, v), k), lambda s, v, k: (s * 0 - np.inf, v * 0 - 1, k * 0 - 1)):
            _wrong(change(s.copy(), v.copy(), k.copy()), x, scores, n, *rest)


def test_orders_where_scores_lose_the_logits():
    """Two hypotheses at -1e30: all candidates have that score, so the first hypothesis has all winners, by its logits."""
    g = np.random.default_rng(0)
    x = g.standard_normal((1, 2, 50))
    scores = np.full((1, 2), np.float64(np.float32(-1e30)))
    n, order = 5, np.argsort(-x[0], axis=-1, kind="stable")
    s = np.full((1, n), -1e30, np.float32)
    right = (s, order[0][None, :n], np.zeros((1, n), int))
    check_order(right, x, scores, n)
    assert all(np.array_equal(a, b) for a, b in zip(right, _best(x, scores, n)))
    _wrong((s, np.arange(n)[None], np.zeros((1, n), int)), x, scores, n)                   # its first tokens, whatever their logits
    _wrong((s, np.sort(order[0][:n])[None], np.zeros((1, n), int)), x, scores, n)          # the right ones in another order
    _wrong((s, order[1][None, -n:], np.ones((1, n), int)), x, scores, n)                   # the other one's worst
    _wrong((s, order[1][None, :n], np.ones((1, n), int)), x, scores, n)                    # the other one's best
    _wrong((s, np.array([[order[0][0], order[1][0], *order[0][1:4]]]), np.array([[0, 1, 0, 0, 0]])), x, scores, n)
    # the second hypothesis better: all its candidates come first
    scores = np.array([[np.float32(-1e30), np.float32(-9e29)]], np.float64)
    check_order((np.full((1, n), -9e29, np.float32), order[1][None, :n], np.ones((1, n), int)), x, scores, n)
    _wrong(right, x, scores, n)
    # one that has ended ties with them, behind the first and before the third
    x = g.standard_normal((1, 3, 4))
    scores = np.full((1, 3), np.float64(np.float32(-1e30)))
    done = np.array([[False, True, False]])
    o = np.argsort(-x[0], axis=-1, kind="stable")
    s = np.full((1, 7), -1e30, np.float32)
    check_order((s, np.array([[*o[0], 2, *o[2][:2]]]), np.array([[0] * 4 + [1] + [2] * 2])), x, scores, 7, done, 2)
    _wrong((s, np.array([[2, *o[0], *o[2][:2]]]), np.array([[1] + [0] * 4 + [2] * 2])), x, scores, 7, done, 2)
    _wrong((s, np.array([[*o[0], *o[2][:3]]]), np.array([[0] * 4 + [2] * 3])), x, scores, 7, done, 2)


def test_the_sums_error_allows_what_it_says():
    """A sum of many equal logits far below the largest one, in the arithmetic of the short rows with exact exponentials: within the bound,
    and beyond a bound that leaves out the arguments' rounding."""
    from operators_order import log_error
    f = np.float32
    worst = 0.0
    for low in np.linspace(-8, -4, 4001):
        low = f(low)
        arg = f(f(low - f(0)) * f(1.44269504))
        off = abs(np.log1p(1024 * np.exp2(np.float64(arg))) - np.log1p(1024 * np.exp(np.float64(low))))
        worst = max(worst, off)
    assert 2.0 ** -22 < worst < log_error(1025)
