"""What the operators decide on the host, no GPU needed: refusals before anything is queued, and arguments that a C
integer would not hold."""
import ctypes

import pytest

OK, NULL, SHAPE, HIP, UNSUPPORTED, SCRATCH = 0, -1, -2, -4, -5, -6
P = 0x100000


@pytest.fixture(scope="module")
def lib():
    import paper_2406_03791_amd as pkg
    return pkg.load_library()


@pytest.mark.parametrize("a_type", [0, 1, 2, 3])
@pytest.mark.parametrize("M,N,K", [(1 << 24, 1 << 20, 512), (1 << 20, 1 << 24, 512), (1 << 24, 1 << 20, 128)])
def test_a_product_of_too_many_blocks_is_refused_before_its_operand_is_quantised(lib, a_type, M, N, K):
    """2^28 blocks and more of the result, a quantisation that is within its own limit: what has been queued by then would come
    back as an error of the HIP runtime here, where there is no device."""
    need = ctypes.c_int64(-1)
    assert lib.rnnt_mx4_product_workspace(a_type, M, N, K, ctypes.byref(need)) == OK and (need.value > 0) == (a_type != 3)
    assert lib.rnnt_mx4_product(P, P, a_type, K, P, P, None, P, 0, N, M, N, K, P, need.value, None) == UNSUPPORTED


WRAPS = 2 ** 32


class _Address:
    def data_ptr(self):
        return P


@pytest.mark.parametrize("by", [WRAPS, -WRAPS, 2 ** 31, 5 * WRAPS])
def test_counts_that_a_32_bit_argument_does_not_hold_are_refused(by):
    """Cut to 32 bits they would be ordinary calls: a vocabulary of 2^32 + 5 tokens one of 5.  (B = 0, so that a call that
    is not refused has nothing to do.)"""
    import paper_2406_03791_amd as pkg
    a = _Address()
    for at, few in ((0, 0), (1, 4), (2, 5), (3, 4)):
        k = [0, 4, 5, 4]
        k[at] = few + by
        with pytest.raises(pkg.RnntError):
            pkg.rnnt_beam_select_workspace(*k)
        with pytest.raises(pkg.RnntError):
            pkg.rnnt_beam_select(a, 0, 20, 5, a, None, *k, -1, a, a, a)
    with pytest.raises(pkg.RnntError):
        pkg.rnnt_beam_select(a, 0, 20, 5, a, a, 0, 4, 5, 4, 1 + by, a, a, a)
    states = pkg.rnnt_beam_states([])
    states.pairs, states.array = [None], (type(states.array)._type_ * 1)()
    for k in ((by, 4, 4), (0, 4 + by, 4), (0, 4, 4 + by)):
        with pytest.raises(pkg.RnntError):
            pkg.rnnt_beam_reorder(states, a, *k)
    pkg.rnnt_beam_reorder(states, a, 0, 4, 4)
    pkg.rnnt_beam_select(a, 0, 20, 5, a, None, 0, 4, 5, 4, -1, a, a, a)


def test_operands_that_a_gradient_is_wanted_for_are_refused():
    """There is no backward pass: a result without its gradient would train on without a word.  Refused before the tensors' device is
    looked at, so that CPU tensors do; codes alone are integers, which have none, and without gradients recorded nothing is refused
    for them (these calls go on to the refusal of tensors on the CPU)."""
    import torch
    import paper_2406_03791_amd as pkg
    m = pkg.Mx4Matrix(3, 64, "cpu")
    a, g = torch.zeros((2, 64)), torch.zeros((2, 64), requires_grad=True)
    b, bg, y, yg = torch.zeros(3), torch.zeros(3, requires_grad=True), torch.zeros((2, 3)), torch.zeros((2, 3), requires_grad=True)
    x, xg, v, vg = (torch.zeros((3, 64), requires_grad=r) for r in (False, True, False, True))
    z, zg = (torch.zeros((1, 2, 5), requires_grad=r) for r in (False, True))
    s, sg = (torch.zeros((1, 2), requires_grad=r) for r in (False, True))
    p, h, hg = torch.zeros((1, 2), dtype=torch.int32), torch.zeros((1, 2, 5)), torch.zeros((1, 2, 5), requires_grad=True)
    calls = [lambda: m.product(g), lambda: m.product(a, bias=bg), lambda: m.product(a, out=yg), lambda: m.product(g, bias=b, out=y),
             lambda: m.product(2 * g), lambda: m.quantize(xg, values=v), lambda: m.quantize(x, values=vg),
             lambda: pkg.beam_select(zg, s), lambda: pkg.beam_select(z, sg), lambda: pkg.beam_reorder([(hg, h)], p), lambda: pkg.beam_reorder([(h, hg)], p),
             lambda: pkg.beam_reorder(pkg.rnnt_beam_states([(h, hg)]), p)]
    for call in calls:
        with pytest.raises(ValueError, match="gradient"):
            call()
        with torch.no_grad(), pytest.raises(ValueError, match="GPU"):
            call()
    for call in (lambda: m.quantize(xg), lambda: pkg.mx4_quantize(xg), lambda: m.product(a), lambda: pkg.beam_select(z, s), lambda: pkg.beam_reorder([(h, h)], p)):
        with pytest.raises(ValueError, match="GPU"):
            call()


def test_what_two_sources_define_in_one_namespace_has_one_name_each():
    """Two definitions of one name in a namespace that units share break C++'s rule of one definition, whatever the linker makes of
    it; what both need is in a header."""
    import collections
    import os
    import re
    import paper_2406_03791_amd as pkg
    folder = os.path.join(os.path.dirname(pkg.__file__), "csrc")
    where = collections.defaultdict(set)
    for name in sorted(os.listdir(folder)):
        shared = False
        with open(os.path.join(folder, name)) as f:
            for line in f:
                if re.match(r"(}  // )?namespace", line):
                    shared = line.startswith("namespace rnnt")
                if not shared or line.rstrip().endswith(";"):
                    continue
                m = (re.match(r"(?:template <(?!>).*?> )?(?:struct|class|union|enum) (\w+)", line)
                     or re.match(r"(?:template <.*> )?(?:(?:__\w+__|static|inline|constexpr) )+[\w :]*?[\w>&*] ?[&*]?\b(?!__)(\w+)\(.*\)\s*(?:\{.*)?$", line))
                if m:
                    where[m.group(1)].add(name)
    assert "wave_sync" in where and "SelectArgs" in where and "aligned" not in where
    twice = {k: v for k, v in where.items() if len(v) > 1}
    assert not twice, twice


def test_what_is_no_matrix_is_refused_as_such():
    import torch
    import paper_2406_03791_amd as pkg
    m = pkg.Mx4Matrix(3, 64, "cpu")
    for shape in ((), (64,), (1, 2, 64)):
        for call in (lambda: pkg.mx4_quantize(torch.zeros(shape)), lambda: m.quantize(torch.zeros(shape)), lambda: m.product(torch.zeros(shape))):
            with pytest.raises(ValueError, match="matrix"):
                call()
