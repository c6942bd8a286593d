"""GPU tests of vp_combine and vp_combine_backward against the definitions in 64 bits."""
import math
import os

import pytest
import torch

from tests import layer_reference as ref

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16, torch.float32]


@pytest.fixture(scope="module")
def vp():
    import paper_2609_34340_b200 as vp
    assert torch.cuda.is_available(), "these tests need a GPU"
    assert os.path.exists(vp.library_path()), "libvariopath.so has not been built"
    return vp


def _case(T, topk, H, dtype, seed, dropped=0.2):
    g = torch.Generator().manual_seed(seed)
    idx = torch.randint(0, 64, (T, topk), generator=g, dtype=torch.int32)
    idx[torch.rand(T, topk, generator=g) < dropped] = -1
    if T > 2:
        idx[1] = -1                                   # a token without copies
    w = torch.randn(T, topk, generator=g)
    rows = torch.randn(T * topk, H, generator=g).to(dtype)
    rows[(idx < 0).view(-1)] = math.nan               # what a dropped copy's row holds does not matter
    return idx, w, rows, torch.randn(T, H, generator=g).to(dtype)


def _finite(rows, idx):
    return torch.where((idx >= 0).view(-1, 1), rows, torch.zeros_like(rows))


SIZES = [(1, 1, 1), (1, 8, 7168), (3, 2, 7), (5, 6, 1000), (7, 8, 2048), (4, 3, 2056), (2, 40, 264), (300, 8, 96), (9, 9, 4104), (130, 4, 512)]


@pytest.mark.parametrize("T,topk,H", SIZES)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("with_base", [False, True])
def test_combine_matches_the_definition(vp, T, topk, H, dtype, with_base):
    idx, w, rows, base = _case(T, topk, H, dtype, T + topk + H)
    out = torch.full((T + 2, H), 3.0, dtype=dtype, device="cuda")
    vp.combine(rows.cuda(), idx.cuda(), w.cuda(), base.cuda() if with_base else None, out[:T])
    want, size = ref.combine(_finite(rows, idx), idx, w, base if with_base else None)
    bound = (topk + 1) * 2.0 ** -24 * size + ref.HALF_STEP[dtype] * want.abs() * (1 + 2.0 ** -8) + ref.LEAST[dtype]
    assert ((out[:T].cpu().double() - want).abs() <= bound).all()
    assert (out[T:] == 3).all()


@pytest.mark.parametrize("T,topk,H", SIZES)
@pytest.mark.parametrize("dtype", TYPES)
def test_combine_backward_matches_the_definition(vp, T, topk, H, dtype):
    idx, w, rows, grad = _case(T, topk, H, dtype, T + topk + H + 1)
    grad_rows, grad_weights = vp.combine_backward(grad.cuda(), rows.cuda(), idx.cuda(), w.cuda())
    here = (idx >= 0).unsqueeze(2)
    want = torch.where(here, w.double().unsqueeze(2) * grad.double().unsqueeze(1), 0.0).view(T * topk, H)
    assert ((grad_rows.cpu().double() - want).abs() <= (ref.HALF_STEP[dtype] * (1 + 2.0 ** -8) + 2.0 ** -24) * want.abs() + ref.LEAST[dtype]).all()
    terms = _finite(rows, idx).double().view(T, topk, H) * grad.double().unsqueeze(1)
    # a thread adds at most H / 256 vectors' values in a row, a tree of five and eight warps join them
    bound = (H / 256 + 32) * 2.0 ** -24 * terms.abs().sum(dim=2) + 1e-37
    assert ((grad_weights.cpu().double() - terms.sum(dim=2)).abs() <= bound).all()
    assert (grad_weights.cpu()[idx < 0] == 0).all()
    only_rows, only_weights = torch.zeros_like(grad_rows), torch.zeros_like(grad_weights)
    calls = vp.binding._calls
    assert calls.combine_backward(grad.cuda(), None, idx.cuda(), w.cuda(), only_rows, None, None) == 0
    assert calls.combine_backward(grad.cuda(), rows.cuda(), idx.cuda(), w.cuda(), None, only_weights, None) == 0
    assert torch.equal(only_rows, grad_rows) and torch.equal(only_weights, grad_weights)


@pytest.mark.parametrize("T,topk,H,first", [(5, 6, 96, 0), (30, 4, 1032, 0), (700, 8, 1032, 0), (3, 8, 4104, 0), (2, 11, 8200, 0), (6, 3, 50, 0), (9, 5, 64, 1)])
@pytest.mark.parametrize("dtype", TYPES)
def test_dropped_copies_have_no_gradient_whatever_the_tokens_gradient_holds(vp, T, topk, H, first, dtype):
    """An overflowed step: infinities and NaN in the gradient of tokens with dropped copies.  Short rows, long rows, rows of many tokens, rows
    that do not begin on 16-byte borders (first: values in front of them)."""
    idx, w, rows, grad = _case(T, topk, H, dtype, T + H, dropped=0.5)
    idx[0, 0], idx[0, 1] = 3, -1
    rows = torch.where((idx >= 0).view(-1, 1), torch.ones_like(rows), rows)
    grad[0, H // 2] = math.inf
    grad[2 % T, H - 1] = math.nan
    grad[T - 1, 0] = -math.inf
    flat = torch.zeros(T * topk * H + first, dtype=dtype, device="cuda")[first:].view(T * topk, H)
    flat.copy_(rows)
    grad_rows, grad_weights = (t.cpu() for t in vp.combine_backward(grad.cuda(), flat, idx.cuda(), w.cuda()))
    assert (grad_weights[idx < 0] == 0).all() and (grad_rows[(idx < 0).view(-1)] == 0).all()
    assert torch.equal(torch.isfinite(grad_weights), (idx < 0) | torch.isfinite(grad).all(dim=1, keepdim=True))


@pytest.mark.parametrize("dtype", TYPES)
def test_combine_backward_matches_differences(vp, dtype):
    """The sum is linear in rows and in weights: a difference is the derivative up to rounding."""
    T, topk, H = 3, 4, 40
    idx, w, rows, grad = _case(T, topk, H, dtype, 5)
    grad_rows, grad_weights = vp.combine_backward(grad.cuda(), rows.cuda(), idx.cuda(), w.cuda())
    rows = _finite(rows, idx)

    def loss(r, v):
        return (ref.combine(r, idx, v, None)[0] * grad.double()).sum()

    at = loss(rows.double(), w.double())
    for t in range(T):
        for s in range(topk):
            step = w.double().clone()
            step[t, s] += 1.0
            assert abs(float(loss(rows.double(), step) - at) - float(grad_weights[t, s])) <= 1e-4
            for h in (0, 17, H - 1):
                moved = rows.double().clone()
                moved[t * topk + s, h] += 1.0
                slope = float(loss(moved, w.double()) - at)
                assert abs(slope - float(grad_rows[t * topk + s, h])) <= 1.01 * ref.HALF_STEP[dtype] * abs(slope) + 1e-6


@pytest.mark.parametrize("topk", [1, 2, 3, 6, 8, 11])
@pytest.mark.parametrize("dtype", TYPES)
def test_gradients_do_not_depend_on_how_many_tokens_a_call_has(vp, topk, dtype):
    """The same tokens in a small batch and in a large one: the same bytes, whatever the row length."""
    for H in (64, 264, 520, 1032, 2048, 4088, 4096, 4104):
        g = torch.Generator(device="cuda").manual_seed(H + topk)
        T = 1300
        rows, grad = (torch.randn(n, H, device="cuda", generator=g).to(dtype) for n in (T * topk, T))
        idx = torch.randint(-1, 20, (T, topk), device="cuda", dtype=torch.int32, generator=g)
        w = torch.randn(T, topk, device="cuda", generator=g)
        large = vp.combine_backward(grad, rows, idx, w)
        for n in (1, 7, 300):
            small = vp.combine_backward(grad[:n], rows[:n * topk], idx[:n], w[:n])
            assert torch.equal(small[0], large[0][:n * topk]) and torch.equal(small[1], large[1][:n]), (H, n)


@pytest.mark.parametrize("dtype", TYPES)
def test_combine_of_unaligned_buffers_and_in_place(vp, dtype):
    T, topk, H = 6, 3, 64
    idx, w, rows, base = _case(T, topk, H, dtype, 8)
    want, size = ref.combine(_finite(rows, idx), idx, w, base)
    bound = 8 * 2.0 ** -24 * size + 1.01 * ref.HALF_STEP[dtype] * want.abs() + ref.LEAST[dtype]
    flat = torch.zeros(T * topk * H + 1, dtype=dtype, device="cuda")[1:].view(T * topk, H)
    flat.copy_(rows)
    assert flat.data_ptr() % 16 != 0
    got = vp.combine(flat, idx.cuda(), w.cuda(), base.cuda())
    assert ((got.cpu().double() - want).abs() <= bound).all()
    a, b = vp.combine_backward(base.cuda(), flat, idx.cuda(), w.cuda())
    c, d = vp.combine_backward(base.cuda(), rows.cuda(), idx.cuda(), w.cuda())
    assert torch.equal(a, c) and torch.allclose(b, d, rtol=1e-5, atol=1e-5)
    out = base.cuda()
    vp.combine(rows.cuda(), idx.cuda(), w.cuda(), out, out)
    assert ((out.cpu().double() - want).abs() <= bound).all()


def test_combine_of_no_tokens_launches_nothing(vp):
    before = vp.kernel_launch_count()
    rows, idx, w = torch.zeros(0, 64, device="cuda"), torch.zeros(0, 4, dtype=torch.int32, device="cuda"), torch.zeros(0, 4, device="cuda")
    assert vp.combine(rows, idx, w).shape == (0, 64)
    vp.combine_backward(rows, rows, idx, w)
    assert vp.kernel_launch_count() == before


def test_combine_gives_the_same_bytes_again_in_a_graph_and_on_another_stream(vp):
    idx, w, rows, base = (t.cuda() for t in _case(64, 8, 2048, torch.bfloat16, 3))
    first = vp.combine(rows, idx, w, base)
    grads = vp.combine_backward(base, rows, idx, w)
    out, gr, gw = torch.zeros_like(first), torch.zeros_like(grads[0]), torch.zeros_like(grads[1])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vp.combine(rows, idx, w, base, out)
        vp.combine_backward(base, rows, idx, w, gr, gw)
    for _ in range(2):
        out.zero_(), gr.zero_(), gw.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, first) and torch.equal(gr, grads[0]) and torch.equal(gw, grads[1])
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    out.zero_()
    other.wait_stream(torch.cuda.current_stream())
    vp.combine(rows, idx, w, base, out, stream=other)
    other.synchronize()
    assert torch.equal(out, first)


def test_combine_refuses(vp):
    rows, idx, w = torch.zeros(12, 64, device="cuda"), torch.zeros(3, 4, dtype=torch.int32, device="cuda"), torch.zeros(3, 4, device="cuda")
    for bad in (lambda: vp.combine(rows[:11], idx, w), lambda: vp.combine(rows.double(), idx, w), lambda: vp.combine(rows[:, ::2], idx, w),
                lambda: vp.combine(rows, idx.long(), w), lambda: vp.combine(rows, idx, w.half()), lambda: vp.combine(rows, idx, w[:, :3]),
                lambda: vp.combine(rows, idx, w, torch.zeros(3, 63, device="cuda")), lambda: vp.combine(rows, idx, w, None, torch.zeros(3, 64)),
                lambda: vp.combine(rows, idx, w, None, torch.zeros(3, 64, device="cuda").half()),
                lambda: vp.combine_backward(torch.zeros(3, 60, device="cuda"), rows, idx, w),
                lambda: vp.combine_backward(torch.zeros(3, 64, device="cuda").half(), rows, idx, w)):
        with pytest.raises(AssertionError):
            bad()
    with pytest.raises(vp.VpError) as e:
        vp.combine(torch.zeros(12, 0, device="cuda"), idx, w)
    assert e.value.code == vp.E_BAD_ARG
