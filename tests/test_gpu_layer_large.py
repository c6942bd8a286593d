"""The operators around the AlltoAllv on buffers of more than 2^31 elements: first and last rows against the definitions."""
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


def _rand(shape, seed, dtype=torch.bfloat16):
    return torch.randn(shape, device="cuda", dtype=dtype, generator=torch.Generator(device="cuda").manual_seed(seed))


def _ends(n, k=3):
    return list(range(k)) + list(range(n - k, n))


def test_route_of_many_tokens(vp):
    T, E = (1 << 31) // 1024 + 5, 1024
    p = vp.RouteParams(E, 4, "sigmoid", 8, 4, 2, True, 1.0)
    z = _rand((T, E), 1)
    bias = torch.round(torch.randn(E, generator=torch.Generator().manual_seed(2)) * 20) / 1000
    idx, w = vp.route(p, z, bias.cuda())
    rows = _ends(T)
    want, want_w = ref.route(p, z[rows].cpu(), bias)
    assert torch.equal(idx[rows].cpu(), want) and torch.allclose(w[rows].cpu().double(), want_w, rtol=1e-5)
    grad = _rand((T, 4), 3, torch.float32)
    out = vp.route_backward(p, z, idx, grad)
    slope, size = ref.route_backward(p, z[rows].cpu(), want, grad[rows].cpu())
    assert ((out[rows].cpu().double() - slope).abs() <= 1e-5 * size + 2.0 ** -8 * slope.abs() + 1e-37).all()


def test_route_of_as_many_tokens_as_there_may_be(vp):
    """One expert, 2^31 - 1 tokens: the launch's size is worked out without leaving 32 bits."""
    T = (1 << 31) - 1
    p = vp.RouteParams(1, 1, "sigmoid", 1, 1, 1, False, 1.0)
    z = torch.zeros(T, 1, device="cuda", dtype=torch.bfloat16)
    z[-2:] = 1.0
    idx, w = vp.route(p, z)
    s = 1 / (1 + torch.exp(torch.tensor(-1.0, dtype=torch.float64)))
    assert int(idx.view(-1)[::4097].abs().sum()) == 0 and (idx[-5:] == 0).all()
    assert torch.allclose(w[-5:].view(-1).cpu().double(), torch.tensor([0.5] * 3 + [float(s)] * 2, dtype=torch.float64), rtol=1e-6)
    out = vp.route_backward(p, z, idx, w.fill_(1.0))
    want = torch.tensor([0.25] * 3 + [float(s * (1 - s))] * 2, dtype=torch.float64)
    assert torch.allclose(out[-5:].view(-1).cpu().double(), want, rtol=2.0 ** -8)


def test_combine_of_many_rows(vp):
    T, topk, H = 4099, 64, 8200
    assert T * topk * H > 1 << 31
    rows, grad = _rand((T * topk, H), 1), _rand((T, H), 2)
    idx = torch.randint(-1, 8, (T, topk), device="cuda", dtype=torch.int32, generator=torch.Generator(device="cuda").manual_seed(3))
    w = _rand((T, topk), 4, torch.float32)
    out = vp.combine(rows, idx, w)
    grad_rows, grad_w = vp.combine_backward(grad, rows, idx, w)
    for t in _ends(T, 2):
        x, here = rows[t * topk:(t + 1) * topk].cpu(), (idx[t:t + 1] >= 0).cpu()
        want, size = ref.combine(x, idx[t:t + 1].cpu(), w[t:t + 1].cpu(), None)
        assert ((out[t:t + 1].cpu().double() - want).abs() <= 65 * 2.0 ** -24 * size + 1.01 * 2.0 ** -8 * want.abs()).all()
        g = grad[t].cpu().double()
        want = torch.where(here.view(-1, 1), w[t].cpu().double().unsqueeze(1) * g, 0.0)
        assert ((grad_rows[t * topk:(t + 1) * topk].cpu().double() - want).abs() <= 1.01 * 2.0 ** -8 * want.abs() + 1e-37).all()
        terms = torch.where(here.view(-1, 1), x.double() * g, 0.0)
        assert ((grad_w[t].cpu().double() - terms.sum(dim=1)).abs() <= (H / 256 + 32) * 2.0 ** -24 * terms.abs().sum(dim=1) + 1e-37).all()


def test_rows_of_4_bits_of_many_values(vp):
    R, K = 65600, 32768
    assert R * K > 1 << 31
    x = _rand((R, K), 1)
    codes, scales = vp.mxfp4_quantize(x)
    out = vp.mxfp4_dequantize(codes, scales)
    for r in _ends(R, 2):
        code, scale = ref.quantize(x[r:r + 1].float().cpu())
        assert torch.equal(ref.pack_codes(code), codes[r:r + 1].cpu()) and torch.equal(scale, scales[r:r + 1].cpu())
        assert torch.equal(out[r:r + 1].cpu(), ref.decode(ref.pack_codes(code), scale).bfloat16())


@pytest.mark.parametrize("rows_of", ["one expert", "many experts"])
def test_product_into_many_values(vp, rows_of):
    R, F, K = 65700, 32776, 64
    assert R * F > 1 << 31
    E = 1 if rows_of == "one expert" else 512            # (pairs of CTAs, and one CTA each: below 192 rows per expert)
    g = torch.Generator(device="cuda").manual_seed(5)
    byte = lambda *s: torch.randint(0, 256, s, device="cuda", dtype=torch.uint8, generator=g)  # noqa: E731
    scale = lambda *s: torch.randint(121, 134, s, device="cuda", dtype=torch.uint8, generator=g)  # noqa: E731
    xc, xs, wc, ws = byte(R, K // 2), scale(R, K // 32), byte(E, F, K // 2), scale(E, F, K // 32)
    off = (torch.arange(E + 1, device="cuda") * R // E).to(torch.int32)
    out, status = vp.mxfp4_product(xc, xs, wc, ws, off)
    assert int(status) == 0
    for r in _ends(R, 2) + [R // 2, (1 << 31) // F, (1 << 31) // F + 1]:
        e = int(torch.searchsorted(off[1:], torch.tensor([r], device="cuda", dtype=torch.int32), right=True))
        x, w = ref.decode(xc[r:r + 1].cpu(), xs[r:r + 1].cpu()), ref.decode(wc[e].cpu(), ws[e].cpu())
        want, size = x @ w.T, x.abs() @ w.abs().T
        assert ((out[r:r + 1].cpu().double() - want).abs() <= 20 * 2.0 ** -23 * size + 1.01 * 2.0 ** -8 * want.abs() + 1e-37).all()
