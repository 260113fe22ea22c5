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
