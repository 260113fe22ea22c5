"""What the operators refuse, and the calls that have nothing to do: decided on the host, no GPU needed.  Pointers are
never read on these paths, so made-up addresses do."""
import ctypes

import pytest

OK, NULL, SHAPE, UNSUPPORTED, SCRATCH = 0, -1, -2, -5, -6
P = 0x100000


@pytest.fixture(scope="module")
def lib():
    import paper_2406_03791_amd as pkg
    return pkg.load_library()


def test_sizes(lib):
    a, b = ctypes.c_int64(-1), ctypes.c_int64(-1)
    f = lambda r, c: (lib.rnnt_mx4_sizes(r, c, ctypes.byref(a), ctypes.byref(b)), a.value, b.value)  # noqa: E731
    assert f(1, 1) == (OK, 1024, 256)
    assert f(16, 512) == (OK, 4096, 256)
    assert f(17, 513) == (OK, 2 * 5 * 1024, 2 * 2 * 256)
    assert f(0, 100) == (OK, 0, 0) and f(100, 0) == (OK, 0, 0)
    assert f(2 ** 31 - 1, 2 ** 31 - 1)[0] == OK
    assert f(-1, 4)[0] == SHAPE and f(4, -1)[0] == SHAPE and f(2 ** 31, 4)[0] == UNSUPPORTED and f(4, 2 ** 31)[0] == UNSUPPORTED
    assert lib.rnnt_mx4_sizes(1, 1, None, ctypes.byref(b)) == NULL


def test_quantize(lib):
    def f(x=P, type=0, rows=4, cols=64, stride=64, codes=P, scales=P, values=None):
        return lib.rnnt_mx4_quantize(x, type, rows, cols, stride, codes, scales, values, None)
    assert f(rows=0) == OK and f(cols=0, stride=0) == OK and f(rows=0, x=None, codes=None) == OK
    assert f(x=None) == NULL and f(codes=None) == NULL and f(scales=None) == NULL
    assert f(type=3) == SHAPE and f(type=-1) == SHAPE and f(rows=-1) == SHAPE and f(cols=-1) == SHAPE and f(stride=63) == SHAPE
    assert f(x=P + 2) == SHAPE and f(x=P + 1, type=1) == SHAPE and f(codes=P + 8) == SHAPE and f(scales=P + 4) == SHAPE and f(values=P + 1) == SHAPE
    assert f(rows=2 ** 31) == UNSUPPORTED and f(rows=2 ** 31 - 1) == UNSUPPORTED and f(rows=2 ** 24, cols=2 ** 24, stride=2 ** 24) == UNSUPPORTED


def test_product(lib):
    def f(a=P, a_scales=P, a_type=3, a_stride=0, w=P, ws=P, bias=None, y=P, y_type=0, y_stride=64, M=8, N=64, K=128, space=None, space_bytes=0):
        return lib.rnnt_mx4_product(a, a_scales, a_type, a_stride, w, ws, bias, y, y_type, y_stride, M, N, K, space, space_bytes, None)
    assert f(M=0) == OK and f(N=0) == OK and f(M=0, a=None, w=None, y=None) == OK
    assert f(a=None) == NULL and f(a_scales=None) == NULL and f(w=None) == NULL and f(ws=None) == NULL and f(y=None) == NULL
    assert f(a_type=4) == SHAPE and f(y_type=3) == SHAPE and f(y_stride=63) == SHAPE and f(M=-1) == SHAPE and f(N=-1) == SHAPE and f(K=-1) == SHAPE
    assert f(a_type=0, a_stride=127) == SHAPE and f(space_bytes=-1) == SHAPE
    assert f(a=P + 8) == SHAPE and f(a_scales=P + 4) == SHAPE and f(w=P + 4) == SHAPE and f(ws=P + 8) == SHAPE and f(bias=P + 2) == SHAPE
    assert f(y=P + 2) == SHAPE and f(y=P + 1, y_type=1) == SHAPE and f(a=P + 2, a_type=0, a_stride=128) == SHAPE
    assert f(M=2 ** 31) == UNSUPPORTED and f(K=2 ** 31) == UNSUPPORTED
    assert f(M=2 ** 28, N=2 ** 20, y_stride=2 ** 20, K=0) == UNSUPPORTED and f(M=2 ** 31 - 1, N=2 ** 20, y_stride=2 ** 20) == UNSUPPORTED
    need = ctypes.c_int64(-1)
    g = lambda *k: (lib.rnnt_mx4_product_workspace(*k, ctypes.byref(need)), need.value)  # noqa: E731
    assert g(3, 8192, 8192, 8192) == (OK, 0) and g(0, 0, 5, 5) == (OK, 0) and g(0, 8, 5, 0) == (OK, 0)
    assert g(4, 1, 1, 1)[0] == SHAPE and g(0, -1, 1, 1)[0] == SHAPE and g(0, 2 ** 31, 1, 1)[0] == UNSUPPORTED
    assert lib.rnnt_mx4_product_workspace(0, 1, 1, 1, None) == NULL
    for shape in ((1 << 20, 8192, 8192), (11309, 640, 1024), (8, 1025, 640)):
        rc, n = g(1, *shape)
        assert rc == OK and n >= 0
        if n:
            k = dict(a_type=1, a_stride=shape[2], y_stride=shape[1], M=shape[0], N=shape[1], K=shape[2])
            assert f(**k) == SCRATCH and f(space=P, space_bytes=n - 1, **k) == SCRATCH and f(space=P + 8, space_bytes=n, **k) == SCRATCH


def test_select(lib):
    def f(x=P, type=0, batch=4000, beam=1000, scores=P, fin=None, B=2, beams=4, V=1000, n=4, end=0, s=P, t=P, p=P, space=P, space_bytes=1 << 40):
        return lib.rnnt_beam_select(x, type, batch, beam, scores, fin, B, beams, V, n, end, s, t, p, space, space_bytes, None)
    assert f(B=0) == OK and f(B=0, x=None, s=None) == OK
    for k in ("x", "scores", "s", "t", "p"):
        assert f(**{k: None}) == NULL
        assert f(**{k: P + 1}) == SHAPE
    assert f(type=3) == SHAPE and f(batch=-1) == SHAPE and f(beam=-1) == SHAPE and f(B=-1) == SHAPE and f(beams=0) == SHAPE and f(beams=65) == SHAPE
    assert f(V=0) == SHAPE and f(n=0) == SHAPE and f(n=65) == SHAPE and f(fin=P, end=1000) == SHAPE and f(fin=P, end=-1) == SHAPE and f(space_bytes=-1) == SHAPE
    assert f(V=2 ** 30) == UNSUPPORTED and f(B=2 ** 31 - 1) == UNSUPPORTED and f(B=2 ** 24, n=40) == UNSUPPORTED
    need = ctypes.c_int64(-1)
    g = lambda *k: (lib.rnnt_beam_select_workspace(*k, ctypes.byref(need)), need.value)  # noqa: E731
    assert g(2, 65, 10, 1)[0] == SHAPE and g(2, 1, 10, 0)[0] == SHAPE and g(2, 64, 2 ** 26, 1)[0] == UNSUPPORTED and g(0, 1, 1, 1) == (OK, 0)
    assert lib.rnnt_beam_select_workspace(1, 1, 1, 1, None) == NULL
    # enough for any type, where the one is done in one launch and the other in two
    assert g(4096, 1, 270000, 4) == (OK, 4096 * 9 * (4 * 8 + 64)) and g(4096, 1, 270000, 33) == (OK, 0)
    for B, beams, V, n in ((1, 4, 65535, 8), (128, 64, 65535, 64), (1, 1, 2 ** 31 - 1, 64)):
        rc, need_ = g(B, beams, V, n)
        assert rc == OK
        if need_:
            k = dict(B=B, beams=beams, V=V, n=n)
            assert f(space=None, **k) == SCRATCH and f(space_bytes=need_ - 1, **k) == SCRATCH and f(space=P + 8, **k) == SCRATCH


def test_reorder(lib):
    from paper_2406_03791_amd.binding import _BeamState

    def state(**kw):
        s = dict(src=P, dst=2 * P, outer=2, row_bytes=64, src_outer=1024, src_batch=256, src_beam=64, dst_outer=1024, dst_batch=256, dst_beam=64)
        s.update(kw)
        return _BeamState(*[s[k] for k, _ in _BeamState._fields_])

    def f(states=None, n=None, parents=P, B=2, k_in=4, k_out=4, **kw):
        states = [state(**kw)] if states is None else states
        return lib.rnnt_beam_reorder((_BeamState * max(1, len(states)))(*states), len(states) if n is None else n, parents, B, k_in, k_out, None)
    assert lib.rnnt_beam_reorder(None, 1, P, 1, 1, 1, None) == NULL
    assert f(B=0) == OK and f(outer=0) == OK and f(row_bytes=0) == OK and f(B=0, src=None, parents=None) == OK
    assert f(src=None) == NULL and f(dst=None) == NULL and f(parents=None) == NULL
    assert f(n=0) == SHAPE and f([state()] * 17) == SHAPE and f(B=-1) == SHAPE and f(parents=P + 2) == SHAPE
    assert f(k_in=0) == SHAPE and f(k_in=65) == SHAPE and f(k_out=0) == SHAPE and f(k_out=65) == SHAPE
    for k in ("outer", "row_bytes", "src_outer", "src_batch", "src_beam", "dst_outer", "dst_batch", "dst_beam"):
        assert f(**{k: -1}) == SHAPE
    assert f(dst_beam=63) == SHAPE and f(dst_batch=63) == SHAPE and f(dst_outer=63) == SHAPE and f(dst_batch=0) == SHAPE
    assert f(dst=P, src_batch=0, dst_batch=0) == SHAPE and f(dst=P, src_outer=0, dst_outer=0) == SHAPE
    assert f(B=0, dst_batch=0) == OK and f(outer=0, dst_outer=0) == OK
    assert f(dst=P, k_out=3) == SHAPE and f(dst=P, dst_batch=512) == SHAPE       # within itself: the same strides and beams
    assert f(outer=2 ** 31) == UNSUPPORTED and f(outer=2 ** 24) == UNSUPPORTED
