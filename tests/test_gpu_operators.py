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


@pytest.mark.parametrize("rows,cols,pad", [(16386, 512, 0), (4100, 2051, 0), (2051, 4608, 5), (33, 262150, 2), (9000, 1000, 1)])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_values_of_more_than_the_l2s_hold(pkg, rows, cols, pad, dtype):  # noqa: F811
    """Above 2^23 values they are stored past the L2s, 16 bytes a lane where a group of columns is whole: all values, codes and scales
    against a run that is not asked for values and what codes and scales stand for, some rows against the definition."""
    import torch
    from operators_util import layout, quantize
    assert rows * cols > 1 << 23
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    wide = torch.randn((rows, cols + pad), generator=g, device="cuda").to(_torch_type(dtype))
    wide[torch.rand((rows, cols + pad), generator=g, device="cuda") < 0.3] = 0
    x = wide[:, :cols]
    x[5, 3], x[rows - 1, cols - 1], x[17, cols // 2] = float("nan"), float("inf"), float("-inf")
    m, plain = pkg.Mx4Matrix(rows, cols, "cuda"), pkg.mx4_quantize(x)
    m.codes.fill_(0xAA), m.scales.fill_(0xAA)
    store = torch.full((rows + 2, cols), 7.0, device="cuda")
    m.quantize(x, values=store[1:rows + 1])
    assert torch.equal(m.codes, plain.codes) and torch.equal(m.scales, plain.scales)
    assert (store[0] == 7).all() and (store[rows + 1] == 7).all()
    # what the codes stand for, in the order of the rows
    R, C, S = -(-rows // 16) * 16, -(-cols // 128) * 128, -(-cols // 512) * 512
    both = torch.stack([m.codes & 15, m.codes >> 4], -1).view(R // 16, C // 128, 4, 16, 32).permute(0, 3, 1, 2, 4).reshape(R, C)
    scale = m.scales.view(R // 16, S // 512, 4, 16, 4).permute(0, 3, 1, 4, 2).reshape(R, S // 32)[:, :C // 32].float()
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device="cuda")
    unit = torch.where(scale == 255, float("nan"), torch.ldexp(torch.ones_like(scale), scale.int() - 127))
    for r in range(0, rows, 1024):
        part = slice(r, min(r + 1024, rows))
        want = (grid[both[part].int()].view(-1, C // 32, 32) * unit[part, :, None]).view(-1, C)[:, :cols]
        assert torch.equal(store[1:rows + 1][part].nan_to_num(123.0), want.nan_to_num(123.0))
    some = sorted({0, 5, 15, 16, 17, rows // 2, rows - 18, rows - 1})
    code, sc, val = quantize(x[some].double().cpu().numpy())
    got = store[1:rows + 1][some].cpu().numpy()
    assert np.array_equal(got, val.astype(np.float32), equal_nan=True)
    assert np.array_equal(np.signbit(got)[~np.isnan(got)], np.signbit(val)[~np.isnan(got)])
    assert np.array_equal(both[some][:, :cols].cpu().numpy(), code)
    c0, s0 = layout(*quantize(x[:16].double().cpu().numpy())[:2])
    assert np.array_equal(m.codes[:c0.size].cpu().numpy(), c0) and np.array_equal(m.scales[:s0.size].cpu().numpy(), s0)
    if dtype == "f32" and pad == 0:                        # the values may take the matrix' place
        again = pkg.Mx4Matrix(rows, cols, "cuda").quantize(wide, values=wide)
        assert torch.equal(again.codes, m.codes) and torch.equal(again.scales, m.scales)
        assert torch.equal(wide.nan_to_num(123.0), store[1:rows + 1].nan_to_num(123.0))


@pytest.mark.parametrize("M,N,K", [(4099, 4100, 300), (8200, 2050, 1290), (6200, 6200, 256)])
@pytest.mark.parametrize("a_type,y_type", [("f16", "f16"), ("mx4", "f16"), ("f32", "f32")])
def test_large_products_of_other_types(pkg, M, N, K, a_type, y_type):  # noqa: F811
    """Sizes that the largest tiles are chosen for, with fp16 results and operands of the types that the other test of them leaves out."""
    from test_gpu_mx4 import _products
    _products(pkg, M, N, K, a_type, y_type)


def _moved(src, parents):
    """src [..., B, beams, row], parents [B, beams_out], as numpy."""
    ok = (parents >= 0) & (parents < src.shape[-2])
    at = np.where(ok, parents, 0)
    out = np.take_along_axis(src, at.reshape((1,) * (src.ndim - 3) + at.shape + (1,)), axis=-2)
    return np.where(ok[..., None], out, 0).astype(src.dtype)


def _parents(g, B, beams, k):
    p = g.integers(-1, beams + 1, (B, k)).astype(np.int32)
    p[0, :] = np.arange(k) % beams                         # all stay
    if B > 1:
        p[1, :] = beams - 1 - np.arange(k) % beams         # all change places
    return p


@pytest.mark.parametrize("beams", [2, 9, 15, 16, 17, 20, 31, 32, 33, 63])
def test_states_within_themselves_by_every_width(pkg, beams):  # noqa: F811
    """Rows whose lengths and distances 16, 8, 4, 2 and 1 bytes divide, within themselves; rows beside them stay."""
    import torch
    g = np.random.default_rng(beams)
    B, p = 3, _parents(g, 3, beams, beams)
    host = [g.integers(0, 255, (2, B, beams, row + pad)).astype(np.uint8) for row, pad in ((4096, 16), (1000, 8), (996, 4), (998, 2), (333, 0), (16, 0), (5, 3), (1, 0))]
    dev = [torch.from_numpy(h).cuda() for h in host]
    pads = (16, 8, 4, 2, 0, 0, 3, 0)
    pkg.beam_reorder([(d[..., :d.shape[-1] - w],) * 2 for d, w in zip(dev, pads)], torch.from_numpy(p).cuda())
    for h, d, w in zip(host, dev, pads):
        row = h.shape[-1] - w
        assert np.array_equal(d.cpu().numpy()[..., :row], _moved(h[..., :row], p)), (h.shape, row)
        assert np.array_equal(d.cpu().numpy()[..., row:], h[..., row:])


@pytest.mark.parametrize("beams", [4, 16, 20, 64])
def test_states_within_themselves_beside_others_in_one_call(pkg, beams):  # noqa: F811
    """Sixteen tensors, in turn within themselves and to another place, long and short, of all widths."""
    import torch
    g = np.random.default_rng(beams)
    B, p = 2, _parents(g, 2, beams, beams)
    shapes = [((), 4096), ((2,), 640), ((), 1), ((3, 2), 33), ((), 9000), ((), 130), ((4,), 8), ((), 2048)] * 2
    types = [np.float32, np.int16, np.int64, np.uint8, np.uint8, np.float32, np.float32, np.int16] * 2
    host = [g.integers(0, 100, (*lead, B, beams, row)).astype(t) for (lead, row), t in zip(shapes, types)]
    dev = [torch.from_numpy(h).cuda() for h in host]
    to = [d if i % 2 == 0 else torch.full_like(d, 77) for i, d in enumerate(dev)]
    states = pkg.rnnt_beam_states(list(zip(dev, to)))
    pkg.beam_reorder(states, torch.from_numpy(p).cuda())
    for i, (h, d, o) in enumerate(zip(host, dev, to)):
        assert np.array_equal(o.cpu().numpy(), _moved(h, p)), (i, h.shape)
        assert i % 2 == 0 or np.array_equal(d.cpu().numpy(), h)


@pytest.mark.parametrize("B,beams,V,n", [(3, 1, 1500, 4), (3, 1, 1500, 5), (2, 1, 1025, 1), (2, 1, 1025, 2), (3, 2, 8192, 8), (3, 2, 8192, 9), (3, 2, 1088, 4), (3, 2, 1088, 5),
                                         (2, 4, 5000, 16), (2, 4, 5000, 17), (3, 16, 6144, 16), (3, 16, 6145, 16), (47, 16, 8000, 16), (48, 16, 8000, 16), (48, 9, 8193, 9)])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_where_rows_begin_to_be_held_whole(pkg, B, beams, V, n, dtype):  # noqa: F811
    """Both sides of what the way of a selection is chosen by: winners a wave, tiles a work-group, utterances."""
    import torch
    g = torch.Generator().manual_seed(B + V + n)
    x = (torch.randn((B, beams, V), generator=g) * 2).to(_torch_type(dtype))
    scores = -torch.rand((B, beams), generator=g)
    _ordered(pkg, x, scores, n)
    x[:, 0, V // 3:] = -float("inf")
    _ordered(pkg, x, scores, n, torch.rand((B, beams), generator=g) < 0.3, V - 1)
