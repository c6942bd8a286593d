"""A mixture-of-experts layer from end to end on one GPU that plays every rank: router, demand, plan, rows in 4 bits, pack, exchange,
unpack, the experts' products, return, combine -- against the same layer from the definitions in 64 bits."""
import os

import numpy as np
import pytest
import torch

from tests import layer_reference as ref
from tests.exchange import deliver
from workloads import SchedParams as WParams, complete_catalog, tree_topology

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def vp():
    import paper_2609_34340_b200 as vp
    assert torch.cuda.is_available(), "these tests need a GPU"
    assert os.path.exists(vp.library_path()), "libvariopath.so has not been built"
    return vp


def _matrices(E, F, K, gen):
    code, scale = ref.quantize(torch.randn(E * F, K, generator=gen) / K ** 0.5)
    return ref.pack_codes(code).view(E, F, K // 2), scale.view(E, F, K // 32)


def _plan(vp, cat, D, row_bytes):
    w = WParams(granule_bytes=row_bytes).resolved(D.shape[0])
    dc = vp.load_catalog(cat.topology.blob(), cat.blob())
    p = vp.SchedParams(lambda_ns=w.lambda_ns, granule_bytes=w.granule_bytes, k_target=w.k_target, n_start=w.n_start, i_aa=w.i_aa, k_max=w.k_max)
    plan = vp.schedule_batch(dc, p, D.unsqueeze(0).cuda().contiguous())
    assert int(plan.status[0]) == 0
    return dc, plan, {k: (v[0] if isinstance(v, np.ndarray) else v) for k, v in plan.cpu().items()}


def _bytes(t):
    return t.cpu().contiguous().view(torch.uint8).numpy().reshape(t.shape[0], -1)


def test_layer_from_logits_to_output(vp):
    """Every rank's tokens through the experts of all ranks.  The reference takes each rounding where the layer does (rows to 4 bits, products and
    activations to bf16, hidden rows to 4 bits, the sum to bf16)."""
    cat = complete_catalog(tree_topology(1))
    N, T, topk, E, H, F, spare = 8, 60, 4, 32, 256, 96, 7
    epr = E // N
    g = torch.Generator().manual_seed(17)
    logits = torch.randn(N, T, E, generator=g)
    logits[2, 5] = -float("inf")                                 # a padding token
    bias = torch.round(torch.randn(E, generator=g) * 20) / 1000
    x = torch.randn(N, T, H, generator=g).to(torch.bfloat16)
    up, down = _matrices(E, 2 * F, H, g), _matrices(E, H, F, g)
    p = vp.RouteParams(E, topk, "sigmoid", 8, 4, 2, True, 2.5)
    idx, weights = zip(*(vp.route(p, logits[i].cuda(), bias.cuda()) for i in range(N)))
    for i in range(N):
        assert torch.equal(idx[i].cpu(), ref.route(p, logits[i], bias)[0])

    # dispatch: rows of codes with their scales behind them, as the pack sends them
    rb = vp.mxfp4_row_bytes(H)
    D = torch.zeros(N, N, dtype=torch.int64)
    for i in range(N):
        row, status = vp.demand_from_routing(idx[i].unsqueeze(0), epr, N, rb, src0=i)
        assert int(status) == 0
        D[i] = row[0].cpu()
    dc, plan, one = _plan(vp, cat, D, rb)
    staged, meta = {}, {}
    for i in range(N):
        rows = torch.zeros(T, rb, dtype=torch.uint8, device="cuda")
        vp.mxfp4_quantize(x[i].cuda(), *vp.mxfp4_rows(rows, H))
        n = int(D[i].sum()) // rb
        s, m = torch.zeros(n, rb, dtype=torch.uint8, device="cuda"), torch.full((n,), -1, dtype=torch.int32, device="cuda")
        assert int(vp.pack(plan, 0, i, idx[i], epr, rows, s, m)) == 0
        staged[i], meta[i] = s.cpu().numpy(), idx[i].view(-1).cpu().numpy()[m.cpu().numpy()] % epr

    # every rank's experts, and their rows back
    ob = 2 * H
    back_dc, back, back_one = _plan(vp, cat, (D // rb * ob).t().contiguous(), ob)
    returned = {}
    for j in range(N):
        recv, expert = deliver(one, j, staged, rb, meta)
        n, cap = recv.shape[0], recv.shape[0] + spare            # a buffer of fixed size, not full
        buf = torch.zeros(cap, rb, dtype=torch.uint8)
        buf[:n] = torch.from_numpy(recv)
        ids = torch.zeros(cap, dtype=torch.int32)
        ids[:n] = torch.from_numpy(expert.astype(np.int32))
        rows, src = torch.zeros(cap, rb, dtype=torch.uint8, device="cuda"), torch.zeros(cap, dtype=torch.int32, device="cuda")
        off, status = vp.unpack(plan, 0, j, buf.cuda(), ids.cuda(), epr, rows, out_src=src)
        assert int(status) == 0 and int(off[-1]) == n
        mine = slice(j * epr, (j + 1) * epr)
        h, st = vp.mxfp4_product(*vp.mxfp4_rows(rows, H), up[0][mine].cuda(), up[1][mine].cuda(), off)
        hc, hs = vp.mxfp4_quantize(h, gated=True, n_rows=off[-1:])
        y, st = vp.mxfp4_product(hc, hs, down[0][mine].cuda(), down[1][mine].cuda(), off, status=st)
        assert int(st) == 0
        s = torch.zeros(n, H, dtype=torch.bfloat16, device="cuda")
        assert int(vp.pack(back, 0, j, src[:n].view(n, 1).contiguous(), 1, y[:n], s)) == 0
        returned[j] = _bytes(s)

    # combine; what a rank routes to itself does not travel (the layer's owner handles it): those copies are dropped here
    xq = [ref.decode(*(lambda c, s: (ref.pack_codes(c), s))(*ref.quantize(x[i].float()))) for i in range(N)]
    wu, wd = ref.decode(*up), ref.decode(*down)
    for i in range(N):
        recv, _ = deliver(back_one, i, returned, ob)
        rows = torch.full((T * topk, H), float("nan"), dtype=torch.bfloat16, device="cuda")
        assert int(vp.unpack_tokens(back, 0, i, idx[i], epr, torch.from_numpy(recv).cuda().view(torch.bfloat16), rows)) == 0
        travels = torch.where((idx[i] >= 0) & (torch.div(idx[i], epr, rounding_mode="floor") != i), idx[i], -1)
        got = vp.combine(rows, travels, weights[i], x[i].cuda()).cpu().double()
        want, size = x[i].double(), x[i].double().abs()
        for t in range(T):
            for s in range(topk):
                e = int(travels[t, s])
                if e < 0:
                    continue
                h = (wu[e] @ xq[i][t]).to(torch.bfloat16).float()
                code, scale = ref.quantize((h[:F] / (1 + torch.exp(-h[:F])) * h[F:]).view(1, F))
                y = (wd[e] @ ref.decode(ref.pack_codes(code), scale)[0]).to(torch.bfloat16).double()
                want[t] += float(weights[i][t, s]) * y
                size[t] += float(weights[i][t, s]) * y.abs()
        assert torch.isfinite(got).all()
        # Half a step of bf16 for the sum and for each returned row.  A hidden value next to a border of a rounding (to bf16 or to 4 bits) may
        # fall to the other side, which moves an output by a step of that value times a weight: rare, and small in the norm.
        off = (got - want).abs()
        tight = off <= 2.0 ** -8 * (1 + 2.0 ** -6) * (want.abs() + size)
        assert tight.double().mean() > 0.98
        assert float(off.norm() / want.norm()) < 2.0 ** -7


def test_gradients_of_a_layer_agree_with_autograd_in_64_bits(vp):
    """Combine of given rows under router weights: the calls' gradients one after another against autograd of the same in 64 bits."""
    T, E, topk, H = 40, 16, 4, 128
    g = torch.Generator().manual_seed(3)
    for scoring in ("softmax", "sigmoid"):
        for renormalise in (False, True):
            p = vp.RouteParams(E, topk, scoring, 4, 2, 1, renormalise, 1.5)
            logits, rows, grad = torch.randn(T, E, generator=g), torch.randn(T * topk, H, generator=g), torch.randn(T, H, generator=g)
            idx, w = vp.route(p, logits.cuda())
            vp.combine(rows.cuda(), idx, w)
            grad_rows, grad_w = vp.combine_backward(grad.cuda(), rows.cuda(), idx, w)
            grad_logits = vp.route_backward(p, logits.cuda(), idx, grad_w)
            z, r = logits.double().requires_grad_(), rows.double().requires_grad_()
            out = (ref.weights_of(p, z, idx.cpu()).unsqueeze(2) * r.view(T, topk, H)).sum(dim=1)
            want_z, want_r = torch.autograd.grad((out * grad.double()).sum(), (z, r))
            assert torch.allclose(grad_rows.cpu().double(), want_r, rtol=1e-5, atol=1e-5)
            assert torch.allclose(grad_logits.cpu().double(), want_z, rtol=1e-4, atol=1e-4 * float(grad_w.abs().max()))
