"""Microscaled 4-bit matrices: quantisation bit for bit against its definition in 64 bits, products
against the 64-bit product of the values that the codes stand for."""
import numpy as np
import pytest

from operators_util import HALF_STEP, layout, quantize, up
from test_gpu_parity import pkg  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu
TYPES = ["f32", "bf16", "f16"]


def _torch_type(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


def _check_quantised(pkg, x, stride_pad=0):  # noqa: F811
    """x: a tensor on the CPU of any of the types."""
    import torch
    rows, cols = x.shape
    wide = torch.full((rows, cols + stride_pad), float("nan"), dtype=x.dtype)
    wide[:, :cols] = x
    dev = wide.cuda()[:, :cols]
    m = pkg.Mx4Matrix(rows, cols, "cuda")
    m.codes.fill_(0xAA)
    m.scales.fill_(0xAA)
    values = torch.full((rows, cols), 7.0, device="cuda")
    m.quantize(dev, values=values)
    code, scale, val = quantize(x.double().numpy())
    wc, ws = layout(code, scale)
    assert np.array_equal(m.scales.cpu().numpy(), ws)
    assert np.array_equal(m.codes.cpu().numpy(), wc)
    got = values.cpu().numpy()
    assert np.array_equal(got, val.astype(np.float32), equal_nan=True)
    assert np.array_equal(np.signbit(got)[~np.isnan(got)], np.signbit(val)[~np.isnan(got)])
    # without the values the same codes
    again = pkg.Mx4Matrix(rows, cols, "cuda").quantize(dev)
    assert torch.equal(again.codes, m.codes) and torch.equal(again.scales, m.scales)


@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (1, 31, 1), (16, 32, 0), (17, 33, 0), (5, 129, 7), (33, 511, 3), (40, 513, 0),
                                           (3, 1300, 4), (130, 640, 0), (7, 2049, 5), (64, 256, 8)])
@pytest.mark.parametrize("dtype", TYPES)
def test_quantised_matrices_bit_for_bit(pkg, rows, cols, pad, dtype):  # noqa: F811
    import torch
    g = torch.Generator().manual_seed(rows * 7 + cols)
    x = torch.randn((rows, cols), generator=g) * torch.exp2(torch.randint(-10, 10, (rows, 1), generator=g).float())
    x[torch.rand((rows, cols), generator=g) < 0.3] = 0
    _check_quantised(pkg, x.to(_torch_type(dtype)), pad)


@pytest.mark.parametrize("dtype", TYPES)
def test_ties_borders_and_the_smallest_and_largest_values(pkg, dtype):  # noqa: F811
    import torch
    t = _torch_type(dtype)
    mids = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    eps = torch.finfo(t).eps
    row = [6.0] + mids + [-m for m in mids]                       # all ties of a block whose unit is 1
    near = [6.0] + [m * (1 + eps) for m in mids] + [-m * (1 - eps) for m in mids]
    rows = []
    ks = range(-140, 126, 7) if dtype != "f16" else range(-24, 13)
    for k in ks:
        rows += [np.ldexp(np.array(row), k), np.ldexp(np.array(near), k)]
    # blocks whose largest value lies at a border of the unit, or at the ends of the type
    fi = torch.finfo(t)
    for v in (6.0, 6.0 * (1 + eps), 3.0, 3.0 * (1 + eps), 12.0 * (1 - eps / 2), fi.max, fi.tiny, fi.smallest_normal, float(torch.tensor(0.0, dtype=t)), -0.0):
        rows.append(np.array([v, -v / 3, v / 7, -0.0] * 8)[:31])
    x = torch.from_numpy(np.stack(rows)).to(t)
    # the type's own subnormals
    sub = torch.arange(1, 32, dtype=torch.float64) * float(torch.finfo(t).smallest_normal) * float(eps)
    x = torch.cat([x, sub.to(t)[None], -sub.to(t)[None] * 3])
    _check_quantised(pkg, x)


@pytest.mark.parametrize("dtype", TYPES)
def test_blocks_that_are_not_finite_are_nan_and_alone(pkg, dtype):  # noqa: F811
    import torch
    x = torch.randn((20, 300), generator=torch.Generator().manual_seed(1))
    x[3, 40] = float("inf")
    x[3, 299] = float("nan")
    x[19, 0] = float("-inf")
    x[0, 100:140] = float("nan")
    _check_quantised(pkg, x.to(_torch_type(dtype)))


def test_values_may_replace_the_matrix(pkg):  # noqa: F811
    import torch
    x = torch.randn((37, 411), generator=torch.Generator().manual_seed(2))
    _, _, val = quantize(x.double().numpy())
    d = x.cuda()
    pkg.Mx4Matrix(37, 411, "cuda").quantize(d, values=d)
    assert np.array_equal(d.cpu().numpy(), val.astype(np.float32))


def _check_product(got, qa, qw, bias, y_type, K):
    """got float64 [M, N]; qa, qw: values in 64 bits.  Products of two e2m1 values and two powers of two are exact; what a
    matrix instruction adds up (128 products and the sum so far) may be off by four units of the largest partial sum,
    whether it rounds or cuts, and a sum of parts by one more: (K / 128 + 8) * 2^-22 of the sum of magnitudes covers
    that.  Then one rounding to the type of y."""
    with np.errstate(invalid="ignore"):
        want, size = qa @ qw.T, np.abs(qa) @ np.abs(qw).T
        if bias is not None:
            want, size = want + bias, size + np.abs(bias)
        tol = (up(K, 128) // 128 + 8) * 2.0 ** -22 * size + HALF_STEP[y_type] * 1.01 * np.abs(want) + (2.0 ** -25 if y_type == "f16" else 0)
    nan = np.isnan(want)
    assert np.array_equal(np.isnan(got), nan)
    bad = ~nan & ~(np.abs(got - want) <= tol)
    assert not bad.any(), (np.argwhere(bad)[:5], got[bad][:5], want[bad][:5])


SHAPES = [(1, 1, 1), (1, 17, 32), (3, 5, 33), (8, 1025, 640), (16, 16, 128), (17, 33, 129), (33, 257, 511), (64, 130, 512), (70, 65, 700),
          (130, 96, 1024), (257, 300, 96), (300, 513, 1500), (31, 48, 2560), (512, 384, 640), (1030, 272, 160), (2100, 640, 1024),
          (1500, 1300, 1100), (700, 3001, 1000), (3000, 333, 2000), (5, 4097, 1000), (20, 300, 9000)]


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("a_type,y_type", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("mx4", "f32"), ("mx4", "bf16"), ("bf16", "f32")])
def test_products(pkg, M, N, K, a_type, y_type):  # noqa: F811
    _products(pkg, M, N, K, a_type, y_type)


def _products(pkg, M, N, K, a_type, y_type):  # noqa: F811
    import torch
    g = torch.Generator().manual_seed(M + 3 * N + 5 * K)
    a = torch.randn((M, K), generator=g) * torch.exp2(torch.randint(-3, 4, (M, 1), generator=g).float())
    w = (torch.rand((N, K), generator=g) - 0.5) * torch.exp2(torch.randint(-3, 2, (N, 1), generator=g).float())
    bias = torch.randn(N, generator=g) if (M + N) % 3 else None
    if a_type != "mx4":
        a = a.to(_torch_type(a_type))
    qa, qw = quantize(a.double().numpy())[2], quantize(w.double().numpy())[2]
    wm = pkg.mx4_quantize(w.cuda())
    pad = (M + K) % 4                                              # rows further apart than they are long
    if a_type == "mx4":
        am = pkg.mx4_quantize(a.cuda())
    else:
        wide = torch.full((M, K + pad), float("nan"), dtype=a.dtype)
        wide[:, :K] = a
        am = wide.cuda()[:, :K]
    out = torch.full((M + 1, N + pad), 99.0, dtype=_torch_type(y_type), device="cuda")
    got = wm.product(am, bias=None if bias is None else bias.cuda(), out=out[:M, :N])
    _check_product(got.double().cpu().numpy(), qa, qw, None if bias is None else bias.double().numpy(), y_type, K)
    assert (out[M:] == 99).all() and (out[:M, N:] == 99).all(), "nothing beyond the matrix is written"
    # the same bits from another call, with a workspace of the caller's full of other values
    need = pkg.rnnt_mx4_product_workspace(pkg.RNNT_TYPES[a_type], M, N, K)
    ws = torch.full((need + 16,), 0xFF, dtype=torch.uint8, device="cuda")
    again = wm.product(am, bias=None if bias is None else bias.cuda(), dtype=_torch_type(y_type), workspace=ws)
    assert torch.equal(again, got)


@pytest.mark.parametrize("M,N,K", [(4099, 4100, 300), (8200, 2050, 1290), (4000, 8000, 128), (4099, 4100, 129), (6200, 6200, 256), (6150, 6400, 520)])
@pytest.mark.parametrize("a_type,y_type", [("mx4", "f32"), ("bf16", "bf16")])
def test_large_products(pkg, M, N, K, a_type, y_type):  # noqa: F811
    """Sizes that the largest tiles are chosen for, with rows and columns that end inside one."""
    _products(pkg, M, N, K, a_type, y_type)


@pytest.mark.parametrize("M", [5, 300, 2050])
@pytest.mark.parametrize("a_type", ["f32", "bf16", "mx4"])
def test_what_is_not_finite_stays_in_its_row_and_column(pkg, M, a_type):  # noqa: F811
    import torch
    g = torch.Generator().manual_seed(M)
    N, K = (200, 300) if M < 2000 else (1700, 800)
    a, w = torch.randn((M, K), generator=g), torch.randn((N, K), generator=g)
    a[2, 299], a[M - 1, 5], w[7, 64], w[199, 299] = float("nan"), float("inf"), float("-inf"), float("nan")
    if a_type == "bf16":
        a = a.bfloat16()
    qa, qw = quantize(a.double().numpy())[2], quantize(w.double().numpy())[2]
    am = pkg.mx4_quantize(a.cuda()) if a_type == "mx4" else a.cuda()
    got = pkg.mx4_quantize(w.cuda()).product(am)
    _check_product(got.double().cpu().numpy(), qa, qw, None, "f32", K)


def test_very_large_and_very_small_scales(pkg):  # noqa: F811
    """Exponents of both sides far from 0, the sums in range: 2^100 * 2^-100, and blocks of zeros beside them."""
    import torch
    g = torch.Generator().manual_seed(5)
    a = torch.randn((40, 256), generator=g) * 2.0 ** 100
    w = torch.randn((50, 256), generator=g) * 2.0 ** -100
    a[:, 32:64] = 0
    w[:, 128:160] = 0
    a[7] = 0
    qa, qw = quantize(a.double().numpy())[2], quantize(w.double().numpy())[2]
    wm = pkg.mx4_quantize(w.cuda())
    _check_product(wm.product(a.cuda()).double().cpu().numpy(), qa, qw, None, "f32", 256)
    _check_product(wm.product(pkg.mx4_quantize(a.cuda())).double().cpu().numpy(), qa, qw, None, "f32", 256)


def test_products_of_nothing(pkg):  # noqa: F811
    import torch
    bias = torch.arange(5, dtype=torch.float32, device="cuda")
    w = pkg.Mx4Matrix(5, 0, "cuda")
    assert torch.equal(w.product(torch.empty((3, 0), device="cuda"), bias=bias), bias.expand(3, 5))
    assert torch.equal(w.product(torch.empty((3, 0), device="cuda")), torch.zeros((3, 5), device="cuda"))
    w = pkg.mx4_quantize(torch.randn((5, 64), device="cuda"))
    assert w.product(torch.empty((0, 64), device="cuda")).shape == (0, 5)
    assert pkg.Mx4Matrix(0, 64, "cuda").product(torch.randn((2, 64), device="cuda")).shape == (2, 0)
    pkg.Mx4Matrix(0, 64, "cuda").quantize(torch.empty((0, 64), device="cuda"))


def test_products_on_another_stream_and_from_a_graph(pkg):  # noqa: F811
    import torch
    g = torch.Generator().manual_seed(9)
    for M, N, K in ((8, 1025, 640), (300, 256, 640), (2100, 640, 1024)):
        w = pkg.mx4_quantize(torch.randn((N, K), generator=g).cuda())
        xs = [torch.randn((M, K), generator=g).cuda() for _ in range(3)]
        want = [w.product(x) for x in xs]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            assert torch.equal(w.product(xs[0]), want[0])
        torch.cuda.current_stream().wait_stream(side)
        x, y = xs[0].clone(), torch.empty_like(want[0])
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            w.product(x, out=y)
        for i in (1, 2, 0, 1):
            x.copy_(xs[i])
            y.fill_(0)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, want[i])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", [(3, 18, 97), (20, 40, 256), (2100, 640, 320), (1500, 1301, 450)])
def test_addresses_that_are_multiples_of_an_element_only(pkg, M, N, K, dtype):  # noqa: F811
    """Operands and results that begin one element behind an aligned address, with rows of odd and of even distances."""
    import torch
    g = torch.Generator().manual_seed(M + N + K)
    t = _torch_type(dtype)
    w = torch.randn((N, K), generator=g)
    for pad in (1, 2):
        a = torch.randn((M, K + pad), generator=g).to(t)
        part = a.cuda()[:, 1:K + 1] if pad > 1 else a.cuda().flatten()[1:].as_strided((M, K), (K + 1, 1))
        x = part.cpu().clone()
        code, scale, val = quantize(x.double().numpy())
        m = pkg.Mx4Matrix(M, K, "cuda").quantize(part)
        wc, ws = layout(code, scale)
        assert np.array_equal(m.codes.cpu().numpy(), wc) and np.array_equal(m.scales.cpu().numpy(), ws)
        out = torch.full((M, N + pad + 1), 99.0, dtype=t, device="cuda")
        got = pkg.mx4_quantize(w.cuda()).product(part, out=out[:, 1:N + 1])
        _check_product(got.double().cpu().numpy(), val, quantize(w.double().numpy())[2], None, dtype, K)
        assert (out[:, 0] == 99).all() and (out[:, N + 1:] == 99).all()


def test_rows_beyond_32_bit_offsets(pkg):  # noqa: F811
    """Rows 2^30 elements apart, of the operand and of the result: the last ones lie beyond 2^32 bytes and 2^31 elements."""
    import torch
    M, N, K, far = 4, 37, 300, 1 << 30
    g = torch.Generator().manual_seed(12)
    a, w = torch.randn((M, K), generator=g).bfloat16(), torch.randn((N, K), generator=g)
    store = torch.empty((M - 1) * far + 1024, dtype=torch.bfloat16, device="cuda")
    x, y = store.as_strided((M, K), (far, 1)), store.as_strided((M, N), (far, 1), 512)
    x.copy_(a)
    code, scale, val = quantize(a.double().numpy())
    assert np.array_equal(pkg.mx4_quantize(x).codes.cpu().numpy(), layout(code, scale)[0])
    pkg.mx4_quantize(w.cuda()).product(x, out=y)
    _check_product(y.double().cpu().numpy(), val, quantize(w.double().numpy())[2], None, "bf16", K)
    assert torch.equal(x.cpu(), a)


def test_a_large_product_from_a_graph_beside_eager_ones(pkg):  # noqa: F811
    """Large tiles, replayed while another stream computes products of its own with a workspace of its own."""
    import torch
    g = torch.Generator().manual_seed(13)
    M, N, K = 4200, 4100, 390
    w = pkg.mx4_quantize(torch.randn((N, K), generator=g).cuda())
    xs = [torch.randn((M, K), generator=g).cuda() for _ in range(2)]
    want = [w.product(x) for x in xs]
    x, y, z = xs[0].clone(), torch.empty_like(want[0]), torch.empty_like(want[0])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        w.product(x, out=y)
    for i in (1, 0, 1):
        x.copy_(xs[i])
        y.fill_(0), z.fill_(0)
        torch.cuda.synchronize()
        graph.replay()
        with torch.cuda.stream(side):
            w.product(xs[1 - i], out=z)
        torch.cuda.synchronize()
        assert torch.equal(y, want[i]) and torch.equal(z, want[1 - i])


def test_refusals_of_tensors_that_do_not_fit(pkg):  # noqa: F811
    import torch
    w = pkg.mx4_quantize(torch.randn((5, 64), device="cuda"))
    with pytest.raises(ValueError):
        w.product(torch.randn((3, 63), device="cuda"))
    with pytest.raises(ValueError):
        w.product(torch.randn((64, 3), device="cuda").t())
    with pytest.raises(ValueError):
        w.product(torch.randn((3, 64)))
    with pytest.raises(TypeError):
        w.product(torch.zeros((3, 64), device="cuda", dtype=torch.int32))
    with pytest.raises(ValueError):
        w.product(torch.randn((3, 64), device="cuda"), bias=torch.zeros(4, device="cuda"))
    with pytest.raises(ValueError):
        w.product(torch.randn((3, 64), device="cuda"), out=torch.zeros((3, 6), device="cuda"))
    for space in (torch.empty((1,), dtype=torch.uint8, device="cuda").expand(1 << 20), torch.empty((64,), device="cuda")):
        with pytest.raises(ValueError):
            w.product(torch.randn((3, 64), device="cuda"), workspace=space)
    with pytest.raises(ValueError):
        w.quantize(torch.randn((5, 65), device="cuda"))
