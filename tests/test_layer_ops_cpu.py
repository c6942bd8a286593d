"""Refusals of the operators around the AlltoAllv that need no GPU: at the C entry points and in the binding."""
import ctypes as C

import pytest
import torch

BF16, F16, F32 = 0, 1, 2


@pytest.fixture(scope="module")
def lib():
    from paper_2609_34340_b200.build import build
    return C.CDLL(build())


class Params(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("experts", "topk", "scoring", "n_group", "topk_group", "group_top", "renormalise")] + [("scale", C.c_float)]


i64, P, null = C.c_int64, C.c_void_p, None
some = P(1 << 20)                                    # an address that nothing reads: every call below is refused or has no rows


def _params(**kw):
    return Params(**{**dict(experts=64, topk=4, scoring=1, n_group=8, topk_group=4, group_top=2, renormalise=1, scale=1.0), **kw})


def test_route_refusals(lib):
    def route(p, logits=some, dtype=F32, ld=64, T=3, idx=some, w=some):
        return lib.vp_route(C.byref(p) if p else null, logits, dtype, i64(ld), T, null, idx, w, null)

    def backward(p, logits=some, dtype=F32, ld=64, T=3, idx=some, g=some, out=some, out_ld=64):
        return lib.vp_route_backward(C.byref(p) if p else null, logits, dtype, i64(ld), T, idx, g, out, i64(out_ld), null)

    for fn in (route, backward):
        assert fn(None) == -1
        for bad in (dict(experts=0), dict(topk=0), dict(topk=65), dict(scoring=2), dict(n_group=0), dict(n_group=7), dict(topk_group=0),
                    dict(topk_group=9), dict(group_top=0), dict(group_top=3), dict(topk=10, topk_group=1), dict(scale=float("inf")),
                    dict(scale=float("nan"))):
            assert fn(_params(**bad)) == -1, bad
        for big in (dict(experts=1032), dict(topk=33, topk_group=8), dict(n_group=64, topk_group=64)):
            assert fn(_params(**big), ld=2000, **(dict(out_ld=2000) if fn is backward else {})) == -6, big
        assert fn(_params(), dtype=3) == -1 and fn(_params(), ld=63) == -1 and fn(_params(), T=-1) == -1
        assert fn(_params(), logits=null) == -1 and fn(_params(), idx=null) == -1 and fn(_params(), logits=P((1 << 20) + 2)) == -1
        assert fn(_params(topk=32, topk_group=8), T=1 << 26) == -6
        assert fn(_params(), T=0, logits=null) == 0
    odd = P((1 << 20) + 2)
    assert route(_params(), idx=odd) == -1 and route(_params(), w=odd) == -1 and backward(_params(), idx=odd) == -1 and backward(_params(), g=odd) == -1
    assert route(_params(), w=null) == -1 and backward(_params(), g=null) == -1 and backward(_params(), out=null) == -1
    assert backward(_params(), out_ld=63) == -1


def test_combine_refusals(lib):
    def combine(rows=some, dtype=BF16, idx=some, w=some, T=3, topk=2, H=64, base=null, out=some):
        return lib.vp_combine(rows, dtype, idx, w, T, topk, i64(H), base, out, null)

    def backward(grad=some, rows=some, dtype=BF16, idx=some, w=some, T=3, topk=2, H=64, gr=some, gw=some):
        return lib.vp_combine_backward(grad, rows, dtype, idx, w, T, topk, i64(H), gr, gw, null)

    for fn in (combine, backward):
        for bad in (dict(dtype=7), dict(dtype=-1), dict(T=-1), dict(topk=0), dict(H=0), dict(H=1 << 40), dict(idx=null), dict(w=null), dict(rows=null),
                    dict(rows=P((1 << 20) + 1))):
            assert fn(**bad) == -1, bad
        assert fn(T=1 << 30, topk=4) == -6
        assert fn(T=0, rows=null, idx=null) == 0
    odd = P((1 << 20) + 2)
    assert combine(idx=odd) == -1 and combine(w=odd) == -1 and backward(idx=odd) == -1 and backward(w=odd) == -1 and backward(gw=odd) == -1
    assert combine(topk=5000, T=1) == -6
    assert combine(out=null) == -1 and combine(base=P((1 << 20) + 1)) == -1
    assert backward(grad=null) == -1 and backward(gr=null, gw=null) == -1


def test_mxfp4_refusals(lib):
    def quantize(x=some, dtype=BF16, ld=64, R=3, K=64, gated=0, codes=some, cl=32, scales=some, sl=2):
        return lib.vp_mxfp4_quantize(x, dtype, i64(ld), i64(R), i64(K), gated, null, codes, i64(cl), scales, i64(sl), null)

    def dequantize(x=some, dtype=BF16, ld=64, R=3, K=64, codes=some, cl=32, scales=some, sl=2):
        return lib.vp_mxfp4_dequantize(codes, i64(cl), scales, i64(sl), i64(R), i64(K), null, x, dtype, i64(ld), null)

    for fn in (quantize, dequantize):
        for bad in (dict(dtype=3), dict(ld=63), dict(R=-1), dict(K=0), dict(K=48), dict(cl=31), dict(sl=1), dict(x=null), dict(codes=null),
                    dict(scales=null), dict(x=P((1 << 20) + 1))):
            assert fn(**bad) == -1, bad
        assert fn(R=1 << 31) == -6
        assert fn(R=0, x=null) == 0
    assert quantize(gated=1, ld=127) == -1

    def product(xc=some, xl=32, xs=some, sl=2, cap=8, wc=some, ws=some, E=2, F=16, K=64, off=some, out=some, dtype=BF16, ol=16, st=some):
        return lib.vp_mxfp4_product(xc, i64(xl), xs, i64(sl), i64(cap), wc, ws, E, i64(F), i64(K), off, out, dtype, i64(ol), st, null)

    for bad in (dict(dtype=5), dict(cap=-1), dict(E=0), dict(F=0), dict(K=0), dict(K=80), dict(ol=15), dict(xl=16), dict(xl=40), dict(sl=1),
                dict(xc=null), dict(xs=null), dict(wc=null), dict(ws=null), dict(off=null), dict(out=null), dict(st=null),
                dict(xc=P((1 << 20) + 8)), dict(wc=P((1 << 20) + 8)), dict(out=P((1 << 20) + 1)), dict(off=P((1 << 20) + 2))):
        assert product(**bad) == -1, bad
    assert product(E=1025) == -6 and product(K=1 << 21, xl=1 << 20, sl=1 << 16) == -6 and product(F=1 << 21, ol=1 << 21) == -6
    assert product(cap=1 << 31) == -6 and product(cap=0, xc=null) == 0


def test_binding_refuses_host_tensors_and_bad_settings():
    import paper_2609_34340_b200 as vp
    z, idx, w, rows = torch.zeros(3, 8), torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, 2), torch.zeros(6, 64)
    p = vp.RouteParams(8, 2)
    for call in (lambda: vp.route(p, z), lambda: vp.route(vp.RouteParams(8, 2, "other"), z), lambda: vp.route_backward(p, z, idx, w),
                 lambda: vp.combine(rows, idx, w), lambda: vp.combine_backward(rows[:3], rows, idx, w), lambda: vp.mxfp4_quantize(rows),
                 lambda: vp.mxfp4_quantize(rows[:, :40]), lambda: vp.mxfp4_dequantize(rows.byte()[:, :32], rows.byte()[:, :2]),
                 lambda: vp.mxfp4_product(rows.byte()[:, :32], rows.byte()[:, :2], torch.zeros(1, 4, 32, dtype=torch.uint8),
                                          torch.zeros(1, 4, 2, dtype=torch.uint8), torch.zeros(2, dtype=torch.int32))):
        with pytest.raises(AssertionError):
            call()


def test_wire_rows():
    import paper_2609_34340_b200 as vp
    for cols, want in ((32, 32), (64, 48), (1024, 544), (2048, 1088), (7168, 3808)):
        assert vp.mxfp4_row_bytes(cols) == want
        codes, scales = vp.mxfp4_rows(torch.zeros(2, want, dtype=torch.uint8), cols)
        assert codes.shape == (2, cols // 2) and scales.shape == (2, cols // 32)
        assert scales.data_ptr() - codes.data_ptr() == cols // 2


def test_reference_rounds_ties_to_the_even_code():
    from tests import layer_reference as ref
    x = torch.tensor([0, 0.25, 0.5, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 5.01, 7.9, -0.25, -0.75, -5.0, 4.0, 0.24] + [0.0] * 16).view(1, 32)
    code, scale = ref.quantize(x)
    assert int(scale) == 127
    values = ref.decode(ref.pack_codes(code), scale)[0, :16].tolist()
    assert values == [0, 0, 0.5, 1, 1, 2, 2, 4, 4, 6, 6, 0, -1, -4, 4, 0]
