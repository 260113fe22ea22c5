"""Selection over beams and vocabulary against the scores of all candidates in 64 bits, and states that
follow the hypotheses, bit for bit."""
import numpy as np
import pytest

from operators_util import check_selection, totals
from test_gpu_parity import pkg  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu
TYPES = ["f32", "bf16", "f16"]


def _torch_type(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


def _run(pkg, x, scores, n, finished=None, end=0, workspace=None):  # noqa: F811
    import torch
    got = pkg.beam_select(x, scores, n, None if finished is None else finished, end, workspace)
    torch.cuda.synchronize()
    return tuple(t.cpu().numpy() for t in got)


def _check(pkg, x, scores, n, finished=None, end=0):  # noqa: F811
    """x: logits on the CPU, of any type."""
    f = None if finished is None else finished.numpy()
    t = totals(x.double().numpy(), scores.numpy(), f, end)
    got = _run(pkg, x.cuda(), scores.cuda(), n, None if finished is None else finished.cuda(), end)
    check_selection(got, t, x.double().numpy(), n)
    return got


CASES = [(1, 1, 1, 1), (1, 1, 5, 5), (2, 3, 7, 9), (1, 4, 1025, 4), (3, 8, 1025, 8), (2, 16, 257, 16), (5, 5, 64, 3), (1, 64, 130, 64), (2, 33, 1000, 33),
         (1, 2, 4096, 64), (2, 4, 8193, 10), (1, 1, 65535, 64), (3, 7, 20001, 12), (1, 64, 20000, 64), (130, 2, 100, 2), (1, 3, 3, 20),
         (1, 2, 8192, 5), (2, 1, 32769, 16), (3, 2, 65543, 4), (1, 1, 262145, 8), (1, 1, 524289, 3), (1050, 2, 9001, 2), (40, 30, 1030, 7),
         (3, 2, 9000, 32), (1, 3, 70000, 25), (2, 32, 3000, 32), (2, 3, 9000, 33), (4200, 1, 9000, 40)]


@pytest.mark.parametrize("B,beams,V,n", CASES)
@pytest.mark.parametrize("dtype", TYPES)
def test_selection(pkg, B, beams, V, n, dtype):  # noqa: F811
    import torch
    g = torch.Generator().manual_seed(B + 10 * beams + V + n)
    x = torch.randn((B, beams, V), generator=g) * 3
    x[:, :, V - 1] += 6
    scores = -torch.rand((B, beams), generator=g).cumsum(1) - 5
    if beams > 2:
        scores[:, 1] = -float("inf")
    _check(pkg, x.to(_torch_type(dtype)), scores, n)
    finished = (torch.rand((B, beams), generator=g) < 0.4).to(torch.uint8)
    _check(pkg, x.to(_torch_type(dtype)), scores, n, finished, end=V // 2)


@pytest.mark.parametrize("V,n", [(50, 10), (1025, 64), (9000, 64), (40000, 17), (9000, 10), (40000, 16), (1500, 9)])
def test_ties_go_to_the_lowest_place(pkg, V, n):  # noqa: F811
    """Few different values, equal rows and equal scores: the order is by value, then hypothesis, then token."""
    import torch
    g = torch.Generator().manual_seed(V)
    row = torch.randint(0, 3, (V,), generator=g).float()
    x = row.expand(2, 6, V).contiguous()
    scores = torch.zeros((2, 6))
    scores[1, 0] = scores[1, 3] = -1.0
    for t in TYPES:
        s, v, k = _run(pkg, x.to(_torch_type(t)).cuda(), scores.cuda(), n)
        for b in range(2):
            best = np.flatnonzero(row.numpy() == 2)
            live = [h for h in range(6) if scores[b, h] == 0]
            want = [(h, int(c)) for h in live for c in best][:n]
            assert list(zip(k[b], v[b]))[:len(want)] == want, (t, b)
    # all equal, and ascending and descending rows
    for x in (torch.zeros((1, 3, V)), torch.arange(V).float().expand(1, 3, V) / 64, -torch.arange(V).float().expand(1, 3, V) / 64):
        _check(pkg, x.contiguous(), torch.zeros((1, 3)), n)


@pytest.mark.parametrize("B,beams,V,n", [(2, 3, 1, 2), (3, 16, 1, 16), (2, 4, 63, 16), (3, 7, 1023, 11), (3, 16, 1024, 16), (2, 5, 1025, 1), (2, 16, 1087, 16),
                                         (2, 15, 1088, 16), (2, 16, 1089, 16), (2, 16, 1025, 17), (2, 17, 1025, 16), (300, 3, 40, 5),
                                         (2, 32, 1025, 32), (2, 31, 300, 20), (3, 4, 1088, 33), (2, 33, 1025, 32), (2, 20, 1024, 5), (2, 3, 500, 32),
                                         (3, 16, 4096, 16), (2, 8, 4097, 32), (2, 4, 8192, 16), (2, 5, 8000, 9), (2, 7, 1500, 12), (2, 8, 8193, 32), (260, 8, 3000, 4)])
@pytest.mark.parametrize("dtype", TYPES)
def test_short_rows(pkg, B, beams, V, n, dtype):  # noqa: F811
    """Around the lengths, hypotheses and winners up to which rows are short or held by one wave: random logits, few different ones, all the
    same but a few, masked ones, and magnitudes at which the scores lose the logits."""
    import torch
    g = torch.Generator().manual_seed(B + 10 * beams + V + n)
    scores = -torch.rand((B, beams), generator=g) * 8
    finished = torch.rand((B, beams), generator=g) < 0.3
    plain = torch.randn((B, beams, V), generator=g) * 2
    masked = plain.masked_fill(torch.rand((B, beams, V), generator=g) < 0.95, -float("inf"))
    masked[0, 1], masked[0, 2, V // 2], masked[B - 1] = -float("inf"), float("nan"), -float("inf")
    few = torch.randint(0, 3, (B, beams, V), generator=g).float()
    same = torch.zeros((B, beams, V))
    same[:, :, ::97] = 1
    peaks = plain.clone()
    peaks[:, 1, V - 1] += 30
    for x in (plain, masked, few, same, peaks, plain * 1e4):
        x = x.to(_torch_type(dtype))
        _check(pkg, x, scores, n)
        _check(pkg, x, scores, n, finished, end=V - 1)
    x = few.to(_torch_type(dtype))
    _check(pkg, x, torch.zeros((B, beams)), n)
    _check(pkg, x, scores * 1e4, n)
    far = scores.clone()
    far[:, 0], far[:, 2], far[0, 1] = -1e30, -1e38, -float("inf")
    _check(pkg, x, far, n)


@pytest.mark.parametrize("B,beams,V,n", [(256, 16, 1025, 16), (256, 16, 1500, 16), (64, 16, 4097, 16), (16, 16, 9000, 16), (16, 8, 40000, 40), (256, 4, 1500, 40)])
def test_equal_logits_of_a_row_stay_in_order(pkg, B, beams, V, n):  # noqa: F811
    """Logits of few bits beside scores of many: what a row has twice has one score, and the lower token comes first."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(V)
    x = (torch.randn((B, beams, V), generator=g, device="cuda") * 3).bfloat16()
    scores = torch.rand((B, beams), generator=g, device="cuda") * -20
    best, tokens, parents = pkg.beam_select(x, scores, n)
    at = x.gather(1, parents.long()[..., None].expand(-1, -1, V)).gather(2, tokens.long()[..., None])[..., 0]
    tie = (parents[:, 1:] == parents[:, :-1]) & (at[:, 1:] == at[:, :-1])
    assert int(tie.sum()) >= 3 and (best[:, 1:] == best[:, :-1])[tie].all() and (tokens[:, 1:] > tokens[:, :-1])[tie].all()


@pytest.mark.parametrize("B,beams,V,n", [(3, 5, 300, 5), (2, 40, 1025, 40), (2, 3, 30000, 3)])
def test_selection_and_reordering_on_another_stream_and_from_a_graph(pkg, B, beams, V, n):  # noqa: F811
    """Short rows, lists and two launches, replayed beside eager calls on another stream."""
    import torch
    g = torch.Generator().manual_seed(V)
    xs = [torch.randn((B, beams, V), generator=g).cuda() for _ in range(2)]
    scores, state = -torch.rand((B, beams), generator=g).cuda(), torch.randn((B, beams, 77), generator=g).cuda()

    def step(x, dst):
        best = pkg.beam_select(x, scores, n)
        pkg.beam_reorder([(state, dst)], best[2])
        return (*best, dst)
    want = [step(x, torch.empty_like(state)) for x in xs]
    for x, w in zip(xs, want):
        check_selection(tuple(t.cpu().numpy() for t in w[:3]), totals(x.double().cpu().numpy(), scores.cpu().numpy()), x.double().cpu().numpy(), n)
        assert np.array_equal(w[3].cpu().numpy(), _reorder(state.cpu().numpy(), w[2].cpu().numpy(), beams))
    side, x, dst = torch.cuda.Stream(), xs[0].clone(), torch.empty_like(state)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(x, dst)
    for i in (1, 0, 1, 1):
        x.copy_(xs[i])
        for t in out:
            t.fill_(5)
        torch.cuda.synchronize()
        graph.replay()
        with torch.cuda.stream(side):
            other = step(xs[1 - i], torch.empty_like(state))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want[i])) and all(torch.equal(a, b) for a, b in zip(other, want[1 - i]))


@pytest.mark.parametrize("V,n", [(40, 20), (1025, 4), (1025, 20), (3000, 9), (9000, 20), (30000, 5), (30000, 40)])
@pytest.mark.parametrize("dtype", TYPES)
def test_masks_of_finite_values(pkg, V, n, dtype):  # noqa: F811
    """Logits of the order of one beside masks of any size, and rows that are all mask, or all large."""
    import torch
    g = torch.Generator().manual_seed(V + n)
    most = float(torch.finfo(_torch_type(dtype)).max)
    values = [v for v in (1e4, 6e4, 1e7, 1e9, 1e10, 1e20, 1e30, 1e38) if v < most]
    x = torch.randn((2 * len(values), 3, V), generator=g)
    few = torch.rand((3, V), generator=g) < 0.98
    for i, v in enumerate(values):
        x[2 * i, 0] = torch.where(few[0], -v, x[2 * i, 0])
        x[2 * i, 1, : V - 1], x[2 * i, 2] = -v, -v
        x[2 * i + 1, 0, ::3], x[2 * i + 1, 1], x[2 * i + 1, 2, V // 2] = v, v, v
    scores = -torch.rand((2 * len(values), 3), generator=g)
    _check(pkg, x.to(_torch_type(dtype)), scores, n)


@pytest.mark.parametrize("dtype", TYPES)
def test_long_rows_whose_first_logits_say_nothing(pkg, dtype):  # noqa: F811
    """The largest logits far from the first ones, the first ones masked or very large, and values at the type's ends."""
    import torch
    g = torch.Generator().manual_seed(5)
    low, inf = float(torch.finfo(_torch_type(dtype)).min), float("inf")
    x = torch.randn((8, 2, 40000), generator=g)
    x[0, :, :600] = -inf
    x[1, :, :600] = low
    x[2, :, 20000:] += 200
    x[3, :, :8192] = -inf                                 # all of a piece and more
    x[4, :, 100:] = -inf
    x[5] = low
    x[6, :, :700] = -low
    x[7, :, ::3] = -low / 2
    scores = -torch.rand((8, 2), generator=g)
    _check(pkg, x.to(_torch_type(dtype)), scores, 9)


@pytest.mark.parametrize("V", [700, 1025, 3000, 8000, 40000])
@pytest.mark.parametrize("dtype", TYPES)
def test_one_logit_above_the_others(pkg, V, dtype):  # noqa: F811
    """By more and more, late in the row and early: what the terms of the sum are differences to is near their largest one."""
    import torch
    g = torch.Generator().manual_seed(V)
    x = torch.randn((12, 3, V), generator=g)
    for i in range(12):
        x[i, 0, V - 10], x[i, 1, V // 3], x[i, 2, 5] = 4 + 1.3 * i, 5 + 7.1 * i, 3 + 2.7 * i
    scores = -torch.rand((12, 3), generator=g)
    _check(pkg, x.to(_torch_type(dtype)), scores, 9)


def test_zeros_of_either_sign_tie(pkg):  # noqa: F811
    import torch
    x = torch.full((1, 1, 100), -1.0)
    x[0, 0, 10], x[0, 0, 20], x[0, 0, 30] = -0.0, 0.0, -0.0
    _, v, _ = _run(pkg, x.cuda(), torch.zeros((1, 1)).cuda(), 4)
    assert v[0].tolist() == [10, 20, 30, 0]


@pytest.mark.parametrize("V", [40, 1025, 12000, 30000])
def test_masks_infinities_and_nan(pkg, V):  # noqa: F811
    import torch
    inf, nan = float("inf"), float("nan")
    g = torch.Generator().manual_seed(V)
    n = 16 if V == 30000 else 20
    x = torch.randn((7, 4, V), generator=g)
    scores = -torch.rand((7, 4), generator=g)
    x[0, :, 3:] = -inf                                    # three tokens of each hypothesis are left
    x[1, 1] = -inf                                        # a hypothesis without any
    x[2, 0, V - 2] = nan
    x[2, 1, 1] = inf                                      # neither has a candidate
    x[3] = -inf                                           # an utterance without any
    scores[4] = -inf
    x[5] = torch.finfo(torch.float32).min                 # all at the type's lowest value
    x[5, 2, 7] = 0
    scores[6, 0], scores[6, 2] = nan, -1e30
    for t in TYPES:
        y = x.to(_torch_type(t))
        if t != "f32":
            y[5] = torch.finfo(y.dtype).min
            y[5, 2, 7] = 0
        got = _check(pkg, y, scores, n)
        assert (got[1][3] == -1).all() and (got[1][4] == -1).all()
    done = torch.zeros((7, 4), dtype=torch.bool)
    done[2], done[3, 1], done[4, 0] = True, True, True     # a finished hypothesis' logits do not matter; one that does not exist stays away
    _check(pkg, x, scores, n, done, end=V - 1)


def test_values_far_apart(pkg):  # noqa: F811
    """Logits of +-1e4 beside scores of -1e5: sums in 64 bits keep what 32 would lose."""
    import torch
    g = torch.Generator().manual_seed(3)
    x = torch.randn((4, 8, 700), generator=g) * 1e4
    scores = -1e5 - torch.rand((4, 8), generator=g)
    _check(pkg, x, scores, 30)
    x = torch.randn((4, 8, 700), generator=g) * 1e-3
    _check(pkg, x, scores, 64)


def test_strides_of_logits(pkg):  # noqa: F811
    import torch
    g = torch.Generator().manual_seed(4)
    big = torch.randn((5, 9, 1100), generator=g).cuda()
    scores = torch.randn((5, 9), generator=g)
    for x in (big[:, :, 3:1030], big[:, :, 1:18], big[:, 2:3, 5:900].expand(5, 9, 895), big[1:2, :, :64].expand(5, 9, 64), big.bfloat16()[:, :, 1:1000]):
        got = _run(pkg, x, scores.cuda(), 9)
        xd = x.double().cpu().numpy()
        check_selection(got, totals(xd, scores.numpy()), xd, 9)


def test_rows_behind_the_last_utterance_stay(pkg):  # noqa: F811
    import torch
    x, sc = torch.randn((3, 4, 1025), device="cuda"), torch.zeros((3, 4), device="cuda")
    need = pkg.rnnt_beam_select_workspace(2, 4, 1025, 5)
    ws = torch.full((need + 16,), 0xFF, dtype=torch.uint8, device="cuda")
    s, v, k = torch.full((3, 5), 7.0, device="cuda"), torch.full((3, 5), 7, device="cuda", dtype=torch.int32), torch.full((3, 5), 7, device="cuda", dtype=torch.int32)
    stream = torch.cuda.current_stream().cuda_stream
    pkg.rnnt_beam_select(x, pkg.RNNT_TYPE_F32, 4 * 1025, 1025, sc, None, 2, 4, 1025, 5, 0, s, v, k, ws, need, stream)
    pkg.rnnt_beam_select(x, pkg.RNNT_TYPE_F32, 4 * 1025, 1025, sc, None, 0, 4, 1025, 5, 0, None, None, None, None, 0, stream)
    torch.cuda.synchronize()
    assert (s[2] == 7).all() and (v[2] == 7).all() and (k[2] == 7).all()
    a = pkg.beam_select(x[:2], sc[:2], 5)
    assert torch.equal(a[0], s[:2]) and torch.equal(a[1], v[:2]) and torch.equal(a[2], k[:2])


def test_logits_beyond_32_bit_offsets(pkg):  # noqa: F811
    """Hypotheses 2^30 elements apart: the last one lies beyond 2^32 bytes and 2^31 elements."""
    import torch
    V, far = 300, 1 << 30
    store = torch.empty(2 * far + V, dtype=torch.bfloat16, device="cuda")
    x = torch.randn((1, 3, V), generator=torch.Generator().manual_seed(6)).bfloat16()
    view = store.as_strided((1, 3, V), (0, far, 1))
    view.copy_(x)
    got = _run(pkg, view, torch.zeros((1, 3)).cuda(), 12)
    xd = x.double().numpy()
    check_selection(got, totals(xd, np.zeros((1, 3), np.float32)), xd, 12)


def _reorder(src, parents, beams_in):
    ok = (parents >= 0) & (parents < beams_in)
    at = np.where(ok, parents, 0)
    out = np.take_along_axis(src, at.reshape((1,) * (src.ndim - 3) + at.shape + (1,)), axis=-2)
    return np.where(ok[..., None], out, 0)


@pytest.mark.parametrize("B,k_in,k_out,row", [(1, 1, 1, 1), (1, 4, 4, 640), (3, 8, 8, 33), (2, 1, 5, 641), (5, 16, 16, 100), (2, 20, 7, 1000), (2, 64, 64, 130),
                                              (3, 33, 40, 5000), (130, 2, 3, 7), (1, 8, 8, 70001)])
def test_states_follow_the_hypotheses(pkg, B, k_in, k_out, row):  # noqa: F811
    import torch
    g = np.random.default_rng(B + row)
    parents = g.integers(-1, k_in, (B, k_out)).astype(np.int32)
    parents[0, 0] = k_in                                  # outside: zeros
    lstm = g.standard_normal((4, B, k_in, row)).astype(np.float32)
    half = g.integers(0, 1 << 16, (B, k_in, row)).astype(np.uint16).view(np.int16)
    byte = g.integers(0, 255, (2, B, k_in, row)).astype(np.uint8)
    count = g.integers(0, 1 << 60, (B, k_in, 1))
    srcs = [lstm, half, byte, count]
    dev = [torch.from_numpy(s).cuda() for s in srcs]
    dst = [torch.full(s.shape[:-2] + (k_out + 1, row if s.shape[-1] > 1 else 1), 77, dtype=d.dtype, device="cuda") for s, d in zip(srcs, dev)]
    p = torch.from_numpy(parents).cuda()
    pkg.beam_reorder([(d, o[..., :k_out, :]) for d, o in zip(dev, dst)], p)
    torch.cuda.synchronize()
    for s, d, o in zip(srcs, dev, dst):
        assert np.array_equal(d.cpu().numpy(), s), "sources stay"
        assert np.array_equal(o[..., :k_out, :].cpu().numpy(), _reorder(s, parents, k_in))
        assert (o[..., k_out, :] == 77).all()
    if k_in == k_out:
        pkg.beam_reorder([(d, d) for d in dev], p)        # within themselves
        torch.cuda.synchronize()
        for s, d in zip(srcs, dev):
            assert np.array_equal(d.cpu().numpy(), _reorder(s, parents, k_in))


def test_large_states(pkg):  # noqa: F811
    """More than the L2s hold, out of place and within themselves, in rows of whole and of broken 16 bytes."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(1)
    for row, dtype in ((40000, torch.float32), (40001, torch.bfloat16)):
        src = torch.randn((2, 32, 8, row), generator=g, device="cuda").to(dtype)
        parents = torch.randint(-1, 8, (32, 8), generator=g, device="cuda", dtype=torch.int32)
        dst = torch.full_like(src, 5)
        pkg.beam_reorder([(src, dst)], parents)
        at = parents.clamp(min=0).long()
        want = src[:, torch.arange(32, device="cuda")[:, None], at] * (parents >= 0)[..., None]
        assert torch.equal(dst, want)
        pkg.beam_reorder([(src, src)], parents)
        assert torch.equal(src, want)


def test_states_with_strides_of_their_own(pkg):  # noqa: F811
    """Hidden and cell vectors in one buffer, double buffers side by side, one source for all utterances."""
    import torch
    g = np.random.default_rng(2)
    both = torch.from_numpy(g.standard_normal((2, 3, 6, 4, 90)).astype(np.float32)).cuda()     # [buffer, layer, B, beams, h and c]
    parents = g.integers(-1, 4, (6, 4)).astype(np.int32)
    p = torch.from_numpy(parents).cuda()
    before = both.clone()
    h, c = slice(0, 45), slice(45, 90)
    start = torch.arange(8, dtype=torch.int32, device="cuda").reshape(1, 1, 8).expand(6, 4, 8)
    labels = torch.zeros((6, 4, 8), dtype=torch.int32, device="cuda")
    pkg.beam_reorder([(both[0][..., h], both[1][..., h]), (both[0][..., c], both[1][..., c]), (start, labels)], p)
    torch.cuda.synchronize()
    assert torch.equal(both[0], before[0])
    assert np.array_equal(both[1].cpu().numpy(), _reorder(before[0].cpu().numpy(), parents, 4))
    assert np.array_equal(labels.cpu().numpy(), _reorder(start.cpu().numpy(), parents, 4))


def test_refusals_of_tensors_that_do_not_fit(pkg):  # noqa: F811
    import torch
    x, s = torch.randn((2, 3, 10), device="cuda"), torch.zeros((2, 3), device="cuda")
    for bad in (lambda: pkg.beam_select(x[0], s), lambda: pkg.beam_select(x, s[:1]), lambda: pkg.beam_select(x, s.double()),
                lambda: pkg.beam_select(x.transpose(1, 2), s), lambda: pkg.beam_select(x, s.cpu()), lambda: pkg.beam_select(x, s, finished=s),
                lambda: pkg.beam_select(x, s, workspace=torch.empty((1,), dtype=torch.uint8, device="cuda").expand(1 << 20)),
                lambda: pkg.beam_select(x, s, workspace=torch.empty((64,), device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        pkg.beam_select(x.double(), s)
    with pytest.raises(pkg.RnntError):
        pkg.beam_select(x, s, 65)
    with pytest.raises(pkg.RnntError):
        pkg.beam_select(x, s, finished=torch.zeros((2, 3), dtype=torch.bool, device="cuda"), end_token=10)
    p = torch.zeros((2, 3), dtype=torch.int32, device="cuda")
    for bad in (lambda: pkg.beam_reorder([(x, x.half())], p), lambda: pkg.beam_reorder([(x, x[:, :2])], p), lambda: pkg.beam_reorder([(x, x)], p.long()),
                lambda: pkg.beam_reorder([(x[..., ::2], x[..., ::2])], p), lambda: pkg.beam_reorder([(x[:1], x[:1])], p)):
        with pytest.raises(ValueError):
            bad()


def _cell(w, label, h, c):
    """One LSTM layer's step on labels [B, beams] and states [B, beams, H], elementary operations in 32 bits."""
    gates = w["emb"][label.long()] @ w["w_ih"].t() + h @ w["w_hh"].t() + w["b"]
    i, f, g, o = gates.chunk(4, -1)
    c = f.sigmoid() * c + i.sigmoid() * g.tanh()
    return o.sigmoid() * c.tanh(), c


@pytest.mark.parametrize("graph", [False, True])
def test_a_beam_search_over_a_transducer_with_4_bit_products(pkg, graph):  # noqa: F811
    """Alignment-length synchronous search: in every step each hypothesis is extended by the blank (its next frame) or
    by a label.  Product, selection and reordering follow one another as in a program; every step's selection is
    checked against the 64-bit scores of its own logits, the logits against the 64-bit product, and at the end every
    hypothesis' state against a walk of its own labels from the start, and its score against the sum of its steps'
    log-probabilities.  The second form is captured into a graph and replayed step by step."""
    import torch
    from operators_util import quantize, totals
    B, T, beams, H, V, steps, blank = 3, 9, 6, 64, 41, 14, 40
    g = torch.Generator().manual_seed(11)
    r = lambda *s: torch.randn(s, generator=g).cuda() * 0.3  # noqa: E731
    w = dict(emb=r(V, H) * 3, w_ih=r(4 * H, H), w_hh=r(4 * H, H), b=r(4 * H))
    w_out, b_out, w_pred, frames = r(V, H) * 2, r(V), r(H, H), r(B, T, H) * 3
    lens = torch.tensor([9, 1, 6], device="cuda")
    out_layer, pred_layer = pkg.mx4_quantize(w_out), pkg.mx4_quantize(w_pred)
    cap = steps
    S = dict(h=torch.zeros((B, beams, H), device="cuda"), c=torch.zeros((B, beams, H), device="cuda"),
             t=torch.zeros((B, beams, 1), dtype=torch.int32, device="cuda"), u=torch.zeros((B, beams, 1), dtype=torch.int32, device="cuda"),
             labels=torch.full((B, beams, cap), -1, dtype=torch.int32, device="cuda"))
    S["h"], S["c"] = _cell(w, torch.full((B, beams), blank, device="cuda"), S["h"], S["c"])
    scores = torch.full((B, beams), -float("inf"), device="cuda")
    scores[:, 0] = 0
    keep = pkg.rnnt_beam_states([(S[k], S[k]) for k in S])
    logits, z = torch.empty((B, beams, V), device="cuda"), torch.empty((B * beams, H), device="cuda")
    seen = {k: torch.empty_like(v) for k, v in dict(before=scores, after=scores).items()}
    seen["done"] = torch.empty((B, beams), dtype=torch.bool, device="cuda")
    seen["tokens"] = torch.empty((B, beams), dtype=torch.int32, device="cuda")
    seen["parents"] = torch.empty((B, beams), dtype=torch.int32, device="cuda")

    def step():
        done = (S["t"][..., 0] >= lens[:, None])
        at = torch.minimum(S["t"][..., 0], (lens - 1)[:, None]).long()
        q = pred_layer.product(S["h"].reshape(B * beams, H))
        z.copy_((frames[torch.arange(B, device="cuda")[:, None], at].reshape(B * beams, H) + q).relu())
        out_layer.product(z, bias=b_out, out=logits.view(B * beams, V))
        seen["before"].copy_(scores)
        seen["done"].copy_(done)
        best, tokens, parents = pkg.beam_select(logits, scores, beams, done, blank)
        pkg.beam_reorder(keep, parents)
        scores.copy_(best)
        seen["after"].copy_(best), seen["tokens"].copy_(tokens), seen["parents"].copy_(parents)
        was_done = torch.gather(done, 1, parents.clamp(min=0).long())
        label = (tokens >= 0) & (tokens != blank)
        h, c = _cell(w, tokens.clamp(min=0), S["h"], S["c"])
        S["h"].copy_(torch.where(label[..., None], h, S["h"]))
        S["c"].copy_(torch.where(label[..., None], c, S["c"]))
        S["labels"].copy_(torch.where((torch.arange(cap, device="cuda") == S["u"]) & label[..., None], tokens[..., None], S["labels"]))
        S["u"].add_(label[..., None].int())
        S["t"].add_(((tokens == blank) & ~was_done)[..., None].int())

    def check():
        n = lambda t: t.double().cpu().numpy()  # noqa: E731
        want = quantize(n(z))[2] @ quantize(n(w_out))[2].T + n(b_out)
        assert np.allclose(n(logits).reshape(-1, V), want, rtol=1e-5, atol=1e-5)
        x = n(logits)
        t = totals(x, n(seen["before"]), n(seen["done"]), blank)
        check_selection((seen["after"].cpu().numpy(), seen["tokens"].cpu().numpy(), seen["parents"].cpu().numpy()), t, x, beams)

    if graph:
        kept = {k: v.clone() for k, v in S.items()}
        kept_scores = scores.clone()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        for k in S:
            S[k].copy_(kept[k])
        scores.copy_(kept_scores)
        torch.cuda.synchronize()
        G = torch.cuda.CUDAGraph()
        with torch.cuda.graph(G):
            step()
        for k in S:
            S[k].copy_(kept[k])
        scores.copy_(kept_scores)
    history = []
    for i in range(steps):
        G.replay() if graph else step()
        torch.cuda.synchronize()
        check()
        history.append((seen["tokens"].cpu().numpy().copy(), seen["parents"].cpu().numpy().copy()))
    # hypotheses walked back: their labels, and their states from the start
    labels, u, t = S["labels"].cpu().numpy(), S["u"].cpu().numpy()[..., 0], S["t"].cpu().numpy()[..., 0]
    found = 0
    for b in range(B):
        for j in range(beams):
            if not torch.isfinite(scores[b, j]):
                continue
            k, path = j, []
            for tokens, parents in reversed(history):
                path.append(int(tokens[b, k]))
                k = int(parents[b, k])
            path = path[::-1]
            mine = [v for v in path if v != blank]
            assert labels[b, j, :u[b, j]].tolist() == mine and u[b, j] == len(mine)
            assert t[b, j] == min(int(lens[b]), path.count(blank))
            h = c = torch.zeros((1, 1, H), device="cuda")
            for v in [blank] + mine:
                h, c = _cell(w, torch.tensor([[v]], device="cuda"), h, c)
            assert torch.allclose(h[0, 0], S["h"][b, j], rtol=1e-4, atol=1e-5) and torch.allclose(c[0, 0], S["c"][b, j], rtol=1e-4, atol=1e-5)
            found += 1
    assert found > B * beams // 2
