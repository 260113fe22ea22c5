"""The operators of a beam search on 4-bit operands where their other tests do not go: sums that rise all along a row,
the largest values' own ways, states moved within themselves by every width, orders where scores lose the logits."""
import numpy as np
import pytest

from test_gpu_parity import pkg  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu


def _torch_type(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


@pytest.mark.parametrize("B,V,n,rise", [(1, 1 << 25, 40, 9.4e-5), (1, 1 << 25, 9, 2e-5), (4100, 65536, 40, 5.9e-4), (4100, 65536, 40, 0.0)])
def test_sums_of_rows_that_rise_all_along(pkg, B, V, n, rise):  # noqa: F811
    """Every 1024 logits are alike and a little above those before, so that whoever has them one after the other rescales a sum each
    time.  The logits of a step are all at most half a unit from a whole shift: an argument is off by 2^-25 of a factor of two, the constant
    log2(e) by 0.35 * 2^-26, an exponential by a unit, 2^-23, a sum of four alike by two roundings, 2^-23: together below 2^-21.8.  The scores
    are near 0 and lose nothing more when they are rounded; the sums in 64 bits, and their rescaling, lose nothing."""
    import torch
    steps = torch.arange(V // 1024, dtype=torch.float64) * rise
    steps = steps.float()
    x = steps.cuda().repeat_interleave(1024).view(1, 1, V).expand(B, 1, V)
    d = steps.double().numpy()
    total = d.max() + np.log(np.exp(d - d.max()).sum() * 1024)
    scores = torch.full((B, 1), float(total - d.max()))
    s, v, k = pkg.beam_select(x, scores.cuda(), n)
    first = V - 1024 if rise else 0
    right = bool((v.cpu().numpy() == np.arange(first, first + n)).all() and (k == 0).all())
    assert right
    want = scores.double().numpy() + d.max() - total
    off = float(np.abs(s.double().cpu().numpy() - want).max())
    assert off <= 2.0 ** -21


# an utterance in one launch without lists (one and two rows a wave), with lists, rows held whole, in pieces, in pieces by lists, and lists of many rows
ORDERS = [(3, 8, 300, 8), (2, 20, 1025, 30), (2, 40, 1025, 40), (3, 4, 4097, 4), (2, 3, 40000, 9), (2, 3, 40000, 40), (1400, 3, 2000, 33)]


def _ordered(pkg, x, scores, n, finished=None, end=0):  # noqa: F811
    from operators_order import check_order
    got = pkg.beam_select(x.cuda(), scores.cuda(), n, None if finished is None else finished.cuda(), end)
    check_order(tuple(t.cpu().numpy() for t in got), x.double().numpy(), scores.double().numpy(), n, None if finished is None else finished.numpy(), end)


@pytest.mark.parametrize("B,beams,V,n", ORDERS)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_orders_where_scores_lose_the_logits(pkg, B, beams, V, n, dtype):  # noqa: F811
    """Scores so large that all candidates of a hypothesis have the same: the hypothesis goes first, then the logit, then the token; and
    scores that lose a part of the logits, or none."""
    import torch
    g = torch.Generator().manual_seed(V + n)
    x = torch.randn((B, beams, V), generator=g) * 2
    x[:, :, V // 2:] = torch.randint(-4, 4, (B, beams, V - V // 2), generator=g).float()     # many ties
    x[0, 0, ::2] = -float("inf")
    x = x.to(_torch_type(dtype))
    finished = torch.rand((B, beams), generator=g) < 0.3
    for value in (-1e30, -1e10, -3.0):
        scores = torch.full((B, beams), value)
        _ordered(pkg, x, scores, n)
        _ordered(pkg, x, scores, n, finished, V - 1)
        scores[:, 1] = 1.1 * value
        scores[B - 1, beams - 1] = 0.9 * value
        _ordered(pkg, x, scores, n)


@pytest.mark.parametrize("B,beams,V,n", ORDERS[:-1])
def test_many_equal_logits_below_the_largest_one(pkg, B, beams, V, n):  # noqa: F811
    """All terms of the sum but one are off by the same: what the logarithm may be off by is nearly reached here."""
    import torch
    g = torch.Generator().manual_seed(V)
    for top in (0.0, 5.37, -811.3):
        x = torch.full((B, beams, V), top) - (3 + 9 * torch.rand((B, beams, 1), generator=g))
        x[:, :, V - 3] = top
        _ordered(pkg, x, -torch.rand((B, beams), generator=g), n)
