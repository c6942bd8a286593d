"""GPU tests of vp_route and vp_route_backward against the definitions in 64 bits."""
import math
import os

import pytest
import torch

from tests import layer_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def vp():
    import paper_2609_34340_b200 as vp
    assert torch.cuda.is_available(), "these tests need a GPU"
    assert os.path.exists(vp.library_path()), "libvariopath.so has not been built"
    return vp


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _weight_bound(logits):
    """Relative error of a weight: an exponential's argument is off by half a unit of the logits' range, the function by 2^-21, a sum
    of 32 terms in a tree and the division by less than 16 units."""
    z = logits.double()
    z = z[torch.isfinite(z)]
    span = float(z.max() - z.min()) + float(z.abs().max()) if z.numel() else 0.0
    return (span + 24) * 2.0 ** -22


def _check(vp, p, logits, bias=None, view=None):
    T = logits.shape[0]
    z = logits.cuda() if view is None else view
    idx = torch.full((T + 3, p.topk), -9, dtype=torch.int32, device="cuda")
    w = torch.full((T + 3, p.topk), -9.0, device="cuda")
    vp.route(p, z, None if bias is None else bias.cuda(), idx[:T], w[:T])
    torch.cuda.synchronize()
    want_idx, want_w = ref.route(p, logits, bias)
    assert torch.equal(idx[:T].cpu(), want_idx)
    got = w[:T].cpu().double()
    assert ((got - want_w).abs() <= _weight_bound(logits) * want_w.abs() + 1e-37).all()
    assert (idx[T:] == -9).all() and (w[T:] == -9).all()            # nothing behind the last token
    return want_idx


SHAPES = [  # experts, topk, n_group, topk_group, group_top
    (1, 1, 1, 1, 1), (8, 2, 1, 1, 1), (16, 8, 4, 2, 2), (33, 33 - 1, 1, 1, 1), (60, 4, 1, 1, 1), (60, 6, 4, 2, 2), (64, 6, 8, 3, 1),
    (96, 8, 8, 4, 2), (128, 1, 1, 1, 1), (160, 6, 8, 3, 1), (160, 8, 8, 1, 2), (192, 6, 1, 1, 1), (256, 8, 8, 4, 2), (256, 8, 8, 4, 1),
    (256, 32, 32, 32, 2), (384, 8, 1, 1, 1), (512, 10, 16, 2, 2), (1024, 8, 8, 1, 2), (1000, 8, 5, 2, 2),
]


@pytest.mark.parametrize("experts,topk,n_group,topk_group,group_top", SHAPES)
@pytest.mark.parametrize("scoring,renormalise", [("softmax", False), ("softmax", True), ("sigmoid", True), ("sigmoid", False)])
@pytest.mark.parametrize("dtype,with_bias", [(torch.float32, True), (torch.bfloat16, False), (torch.bfloat16, True), (torch.float16, False)])
def test_route_matches_the_definition(vp, experts, topk, n_group, topk_group, group_top, scoring, renormalise, dtype, with_bias):
    g = _gen(experts * 31 + topk)
    p = vp.RouteParams(experts, topk, scoring, n_group, topk_group, group_top, renormalise, 2.5)
    logits = (torch.randn(45, experts, generator=g) * 2).to(dtype)
    bias = torch.round(torch.randn(experts, generator=g) * 20) / 1000 if with_bias else None
    _check(vp, p, logits, bias)


@pytest.mark.parametrize("T", [1, 2, 3, 5, 297, 1531])
def test_route_token_counts(vp, T):
    p = vp.RouteParams(64, 6, "sigmoid", 8, 4, 2, True, 1.0)
    _check(vp, p, torch.randn(T, 64, generator=_gen(T)), torch.randn(64, generator=_gen(1)) * 0.1)


def test_route_of_no_tokens_launches_nothing(vp):
    before = vp.kernel_launch_count()
    idx, w = vp.route(vp.RouteParams(64, 6), torch.zeros(0, 64, device="cuda"))
    grad = vp.route_backward(vp.RouteParams(64, 6), torch.zeros(0, 64, device="cuda"), idx, w)
    assert idx.shape == w.shape == (0, 6) and grad.shape == (0, 64) and vp.kernel_launch_count() == before


@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
@pytest.mark.parametrize("with_bias", [False, True])
@pytest.mark.parametrize("n_group,topk_group,group_top", [(1, 1, 1), (8, 4, 2), (4, 1, 1)])
def test_route_of_masked_experts_and_empty_rows(vp, scoring, with_bias, n_group, topk_group, group_top):
    g = _gen(7)
    p = vp.RouteParams(64, 8, scoring, n_group, topk_group, group_top, True, 1.0)
    z = torch.randn(40, 64, generator=g)
    z[:, torch.rand(64, generator=g) < 0.3] = -math.inf
    z[3] = -math.inf                                  # nothing to choose
    z[4] = math.nan
    z[5] = -math.inf
    z[5, 17] = 0.5                                    # one expert
    z[6, 20] = math.nan
    z[7, 9] = math.inf
    z[8] = torch.finfo(torch.float32).min             # the type's lowest value is a logit like any other
    z[9] = torch.finfo(torch.float32).max
    z[10] = -200.0 - torch.arange(64) * 0.25          # scores that vanish in 32 bits
    bias = None
    if with_bias:
        bias = torch.randn(64, generator=g) * 0.05
        bias[11], bias[12], bias[13] = -math.inf, math.nan, math.inf
    idx = torch.full((40, 8), 5, dtype=torch.int32, device="cuda")
    w = torch.full((40, 8), 5.0, device="cuda")
    vp.route(p, z.cuda(), None if bias is None else bias.cuda(), idx, w)
    want_bias = None if bias is None else torch.nan_to_num(bias, nan=-math.inf, posinf=math.inf, neginf=-math.inf)
    want_idx, want_w = ref.route(p, z, want_bias)
    assert torch.equal(idx.cpu(), want_idx)
    assert (idx[3:5] == -1).all() and (w[3:5] == 0).all() and torch.isfinite(w).all()
    rows = [t for t in range(40) if t not in (8, 9, 10)]
    assert ((w.cpu().double() - want_w)[rows].abs() <= 1e-5 * want_w[rows] + 1e-37).all()
    assert ((w.cpu().double() - want_w)[8:11].abs() <= 1e-4).all()


@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
@pytest.mark.parametrize("experts,n_group,topk_group,topk", [(32, 4, 2, 12), (60, 4, 2, 20), (60, 4, 3, 32), (256, 8, 4, 32), (1000, 5, 2, 32)])
def test_route_of_biases_of_the_lowest_value(vp, scoring, experts, n_group, topk_group, topk):
    """Experts kept out by the type's lowest value instead of -inf: they can still be chosen, after all others, and so can groups of
    nothing else, whose two best keys add up to less than 32 bits hold."""
    g = _gen(experts + topk)
    p = vp.RouteParams(experts, topk, scoring, n_group, topk_group, 2, True, 1.0)
    z = torch.randn(24, experts, generator=g)
    z[3] = -math.inf
    per, low = experts // n_group, torch.finfo(torch.float32).min
    for open_ in ([0], [n_group - 1], [], [1, 2], list(range(n_group))):
        bias = torch.full((experts,), low)
        for group in open_:
            bias[group * per:(group + 1) * per] = torch.randn(per, generator=g) * 0.05
        if len(open_) == n_group:
            bias[1::3] = low
            bias[:per] = torch.finfo(torch.float32).max
        _check(vp, p, z, bias)


@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
@pytest.mark.parametrize("n_group,topk_group,group_top", [(1, 1, 1), (8, 4, 2), (4, 2, 1)])
def test_route_of_infinite_biases(vp, scoring, n_group, topk_group, group_top):
    """An infinite bias is the largest number: its expert goes before finite ones, and in the order of indices beside that number itself."""
    g = _gen(21)
    top = torch.finfo(torch.float32).max
    for E in (8, 40, 96, 256):
        p = vp.RouteParams(E, min(E * topk_group // n_group, 9), scoring, n_group, topk_group, group_top, True, 1.0)
        for scale in (0.0, 1.0):
            z = torch.randn(12, E, generator=g) * scale
            bias = torch.randn(E, generator=g) * 0.02
            for share in (0.05, 0.5, 1.0):
                b = bias.clone()
                pick = torch.rand(E, generator=g)
                b[pick < share] = math.inf
                b[pick < share / 2] = top
                _check(vp, p, z, b)


@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
@pytest.mark.parametrize("n_group,topk_group,group_top", [(1, 1, 1), (8, 4, 2)])
def test_route_of_equal_logits_takes_the_lowest_index(vp, scoring, n_group, topk_group, group_top):
    p = vp.RouteParams(256, 8, scoring, n_group, topk_group, group_top, True, 1.0)
    for bias in (None, torch.zeros(256), torch.full((256,), 0.25)):
        idx = _check(vp, p, torch.full((9, 256), 0.75), bias)
        assert torch.equal(idx, torch.arange(8, dtype=torch.int32).expand(9, 8))
    coarse = torch.randint(0, 4, (60, 256), generator=_gen(3)).to(torch.bfloat16)     # many ties
    _check(vp, p, coarse, torch.zeros(256))
    _check(vp, p, coarse, torch.randint(0, 3, (256,), generator=_gen(4)) / 16)


@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
@pytest.mark.parametrize("n_group,topk_group,group_top", [(1, 1, 1), (8, 4, 2), (8, 3, 1)])
def test_route_chooses_as_64_bits_do(vp, scoring, n_group, topk_group, group_top):
    """Biases that make every key of a token nearly the same: the order hangs on digits that 32 bits do not hold."""
    g = _gen(11)
    p = vp.RouteParams(128, 8, scoring, n_group, topk_group, group_top, True, 1.0)
    z = torch.randn(1, 128, generator=g)
    _, s, _ = ref.scores(p, z)
    bias = (0.5 - s[0]).to(torch.float32)
    near = z + torch.randn(64, 128, generator=g) * 1e-7
    _check(vp, p, torch.cat([z, near]), bias)


@pytest.mark.parametrize("experts", [64, 256, 1000, 1024])
@pytest.mark.parametrize("apart", [3e-7, 1e-6, 4e-6, 1.2e-5])
def test_route_chooses_as_64_bits_do_where_the_softmax_sum_is_least_certain(vp, experts, apart):
    """One logit ahead and all others equally far behind, where the sum of the exponentials is off by most; biases that leave keys a step of
    about the error's bound apart, in a random order."""
    g = _gen(experts)
    p = vp.RouteParams(experts, 8, "softmax", 1, 1, 1, True, 1.0)
    far = 4.0
    for _ in range(50):                               # the distance at which the mean distance under the softmax, far - 1, is largest
        far = math.log((experts - 1) / (far - 1))
    z = torch.full((1, experts), -far) + torch.rand(1, experts, generator=g) * 1e-3
    z[0, experts // 3] = 0.0
    _, s, _ = ref.scores(p, z)
    bias = (0.5 - s[0] + torch.randperm(experts, generator=g).double() * apart / 4).to(torch.float32)
    near = z + torch.randn(40, experts, generator=g) * 1e-6
    _check(vp, p, torch.cat([z, near]), bias)


def test_route_of_strided_and_unaligned_logits(vp):
    g = _gen(5)
    p = vp.RouteParams(96, 6, "sigmoid", 4, 2, 2, True, 1.0)
    bias = torch.randn(96, generator=g) * 0.02
    for dtype in (torch.float32, torch.bfloat16):
        wide = torch.randn(50, 131, generator=g).to(dtype)
        for first in (0, 1, 3, 8, 35):
            _check(vp, p, wide[:, first:first + 96], bias, view=wide.cuda()[:, first:first + 96])
        _check(vp, p, wide[::3, :96], bias, view=wide.cuda()[::3, :96])


def _grad_check(vp, p, logits, idx, grad, view=None, out=None):
    z = logits.cuda() if view is None else view
    got = vp.route_backward(p, z, idx.cuda(), grad.cuda(), out)
    want, size = ref.route_backward(p, logits, idx, grad)
    dt = logits.dtype
    bound = (_weight_bound(logits) * 4 + 64 * 2.0 ** -24) * size + ref.HALF_STEP[dt] * want.abs() + ref.LEAST[dt]
    assert ((got.cpu().double() - want).abs() <= bound).all()
    return got


@pytest.mark.parametrize("experts,topk,n_group,topk_group,group_top", SHAPES)
@pytest.mark.parametrize("scoring,renormalise", [("softmax", False), ("softmax", True), ("sigmoid", True), ("sigmoid", False)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_route_backward_matches_the_formula(vp, experts, topk, n_group, topk_group, group_top, scoring, renormalise, dtype):
    g = _gen(experts + topk)
    p = vp.RouteParams(experts, topk, scoring, n_group, topk_group, group_top, renormalise, 2.5)
    logits = (torch.randn(21, experts, generator=g) * 2).to(dtype)
    idx, _ = ref.route(p, logits, None)
    _grad_check(vp, p, logits, idx, torch.randn(21, topk, generator=g))


@pytest.mark.parametrize("scoring,renormalise", [("softmax", False), ("softmax", True), ("sigmoid", True), ("sigmoid", False)])
def test_route_backward_matches_differences(vp, scoring, renormalise):
    g = _gen(2)
    p = vp.RouteParams(24, 5, scoring, 1, 1, 1, renormalise, 1.5)
    logits, grad = torch.randn(6, 24, generator=g), torch.randn(6, 5, generator=g)
    idx, _ = ref.route(p, logits, None)
    got = vp.route_backward(p, logits.cuda(), idx.cuda(), grad.cuda()).cpu().double()
    z, h = logits.double(), 1e-4
    for e in range(24):
        step = torch.zeros(24, dtype=torch.float64)
        step[e] = h
        up, down = ref.weights_of(p, z + step, idx), ref.weights_of(p, z - step, idx)
        slope = ((up - down) / (2 * h) * grad.double()).sum(dim=1)
        # h^2 / 6 times a third derivative (below 2 a weight), and the kernel's 32 bits
        assert ((got[:, e] - slope).abs() <= 1e-7 + 1e-5 * grad.double().abs().sum(dim=1)).all()


@pytest.mark.parametrize("scoring,renormalise", [("softmax", False), ("softmax", True), ("sigmoid", True), ("sigmoid", False)])
def test_route_backward_of_slots_that_count_for_nothing(vp, scoring, renormalise):
    """Dropped and foreign slots, masked experts, an expert named twice, strided rows on both sides."""
    g = _gen(9)
    p = vp.RouteParams(40, 6, scoring, 1, 1, 1, renormalise, 1.0)
    logits = torch.randn(30, 40, generator=g)
    logits[:, 5] = -math.inf
    logits[2] = -math.inf
    logits[3, 6] = math.nan
    idx = torch.stack([torch.randperm(40, generator=g)[:6] for _ in range(30)]).to(torch.int32)
    idx[0] = -1
    idx[1, 2], idx[1, 3] = 40, 1 << 30
    idx[4, 1] = idx[4, 4] = idx[4, 0]
    idx[5] = 5
    idx[3, 0] = 6
    grad = torch.randn(30, 6, generator=g)
    wide, out = torch.zeros(30, 45), torch.full((30, 47), 7.0, device="cuda")
    wide[:, 2:42] = logits
    clean = torch.where(torch.isnan(logits), -math.inf, logits)
    want, size = ref.route_backward(p, clean, idx, grad)
    vp.route_backward(p, wide.cuda()[:, 2:42], idx.cuda(), grad.cuda(), out[:, 3:43])
    got = out.cpu().double()
    assert ((got[:, 3:43] - want).abs() <= (_weight_bound(logits) * 4 + 64 * 2.0 ** -24) * size + 1e-37).all()
    assert (got[:, :3] == 7).all() and (got[:, 43:] == 7).all()


def test_route_on_another_stream_and_in_a_graph(vp):
    g = _gen(1)
    p = vp.RouteParams(256, 8, "sigmoid", 8, 4, 2, True, 2.5)
    a, b = torch.randn(200, 256, generator=g), torch.randn(200, 256, generator=g)
    bias = torch.randn(256, generator=g) * 0.02
    z, db = a.cuda(), bias.cuda()
    grad, out = torch.randn(200, 8, generator=g), torch.zeros(200, 256, device="cuda")
    dg = grad.cuda()
    idx, w = vp.route(p, z, db)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vp.route(p, z, db, idx, w)
        vp.route_backward(p, z, idx, dg, out)
    for logits in (b, a):
        z.copy_(logits)
        graph.replay()
        torch.cuda.synchronize()
        want, _ = ref.route(p, logits, bias)
        assert torch.equal(idx.cpu(), want)
        slope, size = ref.route_backward(p, logits, want, grad)
        assert ((out.cpu().double() - slope).abs() <= (_weight_bound(logits) * 4 + 64 * 2.0 ** -24) * size + 1e-37).all()
    other = torch.cuda.Stream()
    idx2 = torch.zeros_like(idx)
    other.wait_stream(torch.cuda.current_stream())
    vp.route(p, z, db, idx2, w, stream=other)
    other.synchronize()
    assert torch.equal(idx2, idx)


def test_route_refuses(vp):
    z = torch.zeros(4, 64, device="cuda")
    ok = dict(experts=64, topk=4, n_group=8, topk_group=2)
    for change in (dict(topk=0), dict(topk=17), dict(n_group=7), dict(topk_group=9), dict(topk_group=0), dict(group_top=3), dict(scale=math.inf)):
        with pytest.raises(vp.VpError) as e:
            vp.route(vp.RouteParams(**{**ok, **change}), z, None, torch.zeros(4, change.get("topk", 4), dtype=torch.int32, device="cuda"),
                     torch.zeros(4, change.get("topk", 4), device="cuda"))
        assert e.value.code == vp.E_BAD_ARG
    for experts, topk, groups in ((1025, 4, 1), (64, 33, 1), (64, 4, 64)):
        with pytest.raises(vp.VpError) as e:
            vp.route(vp.RouteParams(experts, topk, n_group=groups, topk_group=groups), torch.zeros(4, experts, device="cuda"))
        assert e.value.code == vp.E_UNSUPPORTED
    p = vp.RouteParams(**ok)
    idx, w = torch.zeros(4, 4, dtype=torch.int32, device="cuda"), torch.zeros(4, 4, device="cuda")
    for bad in (lambda: vp.route(vp.RouteParams(64, 4, "relu"), z), lambda: vp.route(p, z.double()), lambda: vp.route(p, z[:, :60]),
                lambda: vp.route(p, z.t()), lambda: vp.route(p, z, torch.zeros(63, device="cuda")), lambda: vp.route(p, z, torch.zeros(64)),
                lambda: vp.route(p, z, None, idx[:3], w), lambda: vp.route(p, z, None, idx.long(), w), lambda: vp.route(p, z, None, idx, w.half()),
                lambda: vp.route(p, z[:1].expand(4, 64)), lambda: vp.route_backward(p, z, idx, w, torch.zeros(4, 64, device="cuda").half()),
                lambda: vp.route_backward(p, z, idx[:2], w)):
        with pytest.raises(AssertionError):
            bad()
