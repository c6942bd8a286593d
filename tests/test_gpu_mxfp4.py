"""GPU tests of vp_mxfp4_quantize, vp_mxfp4_dequantize and vp_mxfp4_product against the definitions in 64 bits."""
import ctypes
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


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _unpack(codes):
    return torch.stack([codes % 16, codes // 16], dim=-1).flatten(-2)


# ---- rows to codes and back -----------------------------------------------------------------------------------------------

def _rows(R, K, dtype, seed):
    """Rows whose blocks range over many magnitudes, with every border of the rounding and odd blocks among them."""
    g = _gen(seed)
    x = torch.randn(R, K, generator=g) * torch.exp2(torch.randint(-12, 12, (R, K // 32), generator=g).float()).repeat_interleave(32, dim=1)
    borders = torch.tensor([0, 0.25, 0.5, 0.75, 1.0, 1.25, 1.5, 1.75, 2.0, 2.5, 3.0, 3.5, 4.0, 5.0, 6.0, 7.75])
    x[0, :32] = torch.cat([borders, -borders])
    if R > 1:
        x[1, :32] = 0
        x[1, 31] = -0.0
    return x.to(dtype)


@pytest.mark.parametrize("R,K", [(1, 32), (2, 64), (3, 96), (5, 2048), (129, 224), (700, 1408), (33, 7168)])
@pytest.mark.parametrize("dtype", TYPES)
def test_quantize_matches_the_definition(vp, R, K, dtype):
    x = _rows(R, K, dtype, R + K)
    buf = torch.full((R + 2, vp.mxfp4_row_bytes(K) + 16), 0xEE, dtype=torch.uint8, device="cuda")
    codes, scales = vp.mxfp4_rows(buf[:R], K)
    vp.mxfp4_quantize(x.cuda(), codes, scales)
    want_code, want_scale = ref.quantize(x.float())
    assert torch.equal(_unpack(codes.cpu()), want_code) and torch.equal(scales.cpu(), want_scale)
    assert (buf[R:] == 0xEE).all() and (buf[:R, K // 2 + K // 32:] == 0xEE).all()      # nothing else is written
    values = ref.decode(codes.cpu(), scales.cpu())
    for out_type in TYPES:
        out = torch.full((R + 1, K), 9.0, dtype=out_type, device="cuda")
        vp.mxfp4_dequantize(codes, scales, out[:R])
        assert torch.equal(out[:R].cpu(), values.to(out_type)) and (out[R:] == 9).all()
    own_codes, own_scales = vp.mxfp4_quantize(x.cuda())
    assert torch.equal(own_codes, codes) and torch.equal(own_scales, scales)
    assert torch.equal(vp.mxfp4_dequantize(own_codes, own_scales).cpu(), values.to(torch.bfloat16))


def test_quantize_of_extreme_blocks(vp):
    top, low = torch.finfo(torch.float32).max, 2.0 ** -149
    x = torch.zeros(10, 32)
    x[0, 0], x[0, 1] = top, -top
    x[1, :3] = torch.tensor([low, -3 * low, 2.0 ** -126])
    x[2, 4] = 2.0 ** -125
    x[3, 0], x[3, 1] = 2.0 ** -128, 2.0 ** -127 * 5.5
    x[4, 7] = math.inf
    x[5, 8] = -math.inf
    x[6, 9], x[6, 10] = math.nan, 1e30
    x[7] = math.nan
    x[8] = torch.linspace(-1, 1, 32)
    x[9, 31] = 1.0
    codes, scales = vp.mxfp4_quantize(x.cuda())
    want_code, want_scale = ref.quantize(x)
    assert torch.equal(_unpack(codes.cpu()), want_code) and torch.equal(scales.cpu(), want_scale)
    assert (scales[4:8] == 255).all() and (codes[4:8] == 0).all()
    out = vp.mxfp4_dequantize(codes, scales, torch.zeros(10, 32, device="cuda")).cpu()
    assert torch.isnan(out[4:8]).all() and torch.isfinite(out[:4]).all()
    assert torch.equal(out[:4].double(), ref.decode(codes.cpu(), scales.cpu())[:4])


@pytest.mark.parametrize("dtype", TYPES)
def test_quantize_of_strided_and_unaligned_rows(vp, dtype):
    x = _rows(20, 96, dtype, 3)
    want_code, want_scale = ref.quantize(x.float())
    wide = torch.zeros(20, 200, dtype=dtype, device="cuda")
    for first in (0, 1, 8, 17):
        wide[:, first:first + 96] = x.cuda()
        buf = torch.full((20, 101), 0xEE, dtype=torch.uint8, device="cuda")             # rows of an odd number of bytes
        codes, scales = buf[:, 3:51], buf[:, 60:63]
        vp.mxfp4_quantize(wide[:, first:first + 96], codes, scales)
        assert torch.equal(_unpack(codes.cpu()), want_code) and torch.equal(scales.cpu(), want_scale)
        rest = torch.ones(101, dtype=torch.bool)
        rest[3:51], rest[60:63] = False, False
        assert (buf[:, rest.cuda()] == 0xEE).all()
        out = torch.full((20, 113), 5.0, dtype=dtype, device="cuda")
        vp.mxfp4_dequantize(codes, scales, out[:, 7:103])
        assert torch.equal(out[:, 7:103].cpu(), ref.decode(codes.cpu(), scales.cpu()).to(dtype))
        assert (out[:, :7] == 5).all() and (out[:, 103:] == 5).all()


@pytest.mark.parametrize("n", [-5, 0, 1, 7, 40, 1000])
def test_rows_in_use_are_counted_on_the_device(vp, n):
    x = _rows(40, 64, torch.bfloat16, 4)
    x[max(n, 0):] = math.nan                          # behind the last sequence: whatever memory holds
    count = torch.tensor([n], dtype=torch.int32, device="cuda")
    codes = torch.full((40, 32), 0xEE, dtype=torch.uint8, device="cuda")
    scales = torch.full((40, 2), 0xEE, dtype=torch.uint8, device="cuda")
    vp.mxfp4_quantize(x.cuda(), codes, scales, n_rows=count)
    used = min(max(n, 0), 40)
    want_code, want_scale = ref.quantize(x.float())
    assert torch.equal(_unpack(codes.cpu())[:used], want_code[:used]) and torch.equal(scales.cpu()[:used], want_scale[:used])
    assert (codes[used:] == 0xEE).all() and (scales[used:] == 0xEE).all()
    out = torch.full((40, 64), 5.0, dtype=torch.bfloat16, device="cuda")
    vp.mxfp4_dequantize(codes, scales, out, n_rows=count)
    assert torch.equal(out[:used].cpu(), ref.decode(codes.cpu(), scales.cpu())[:used].bfloat16()) and (out[used:] == 5).all()


@pytest.mark.parametrize("R,K", [(1, 32), (7, 96), (130, 2048)])
@pytest.mark.parametrize("dtype", TYPES)
def test_gated_quantize(vp, R, K, dtype):
    """silu(first) * second in 32 bits: a value is off by at most 8 units in the last place (the exponential, two sums, a quotient,
    a product), so codes and scales are the definition's wherever it is not that near a border, and next to it elsewhere."""
    g = _gen(R + K)
    h = torch.randn(R, 2 * K, generator=g)
    h[:, ::7] *= 20
    h = h.to(dtype)
    gate, up = h[:, :K].double(), h[:, K:].double()
    v = gate / (1 + torch.exp(-gate)) * up
    codes, scales = vp.mxfp4_quantize(h.cuda(), gated=True)
    off = 8 * 2.0 ** -23
    lo, hi = ref.quantize(v * (1 - off)), ref.quantize(v * (1 + off))
    clear = (lo[1] == hi[1]).repeat_interleave(32, dim=1) & (lo[0] == hi[0])
    got = _unpack(codes.cpu())
    assert torch.equal(got[clear], lo[0][clear])
    assert (torch.isin(scales.cpu().int() - lo[1].int(), torch.tensor([0, 1])) | (scales.cpu() == hi[1])).all()
    assert clear.double().mean() > 0.99


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("far", [0, 1, 2])
def test_gated_quantize_over_the_whole_range_of_gates(vp, dtype, far):
    """A gate to a block, from the type's lowest value to its largest, both sides of -87.3 (where 1 + e^-x passes 2^126) and -88.7 (where e^-x
    leaves 32 bits), down to where the activation vanishes, infinities and NaN; times factors that bring it to every place between two codes.
    The activation is off by five units in the last place (an exponential 2, its correction, the sum and the product half a one each, the reciprocal 1)
    and its product with the factor by half a one, and what is not a normal number by half the smallest step, so the code is that of a value
    within these."""
    top = torch.finfo(dtype).max
    gates = torch.tensor([top, -top, top * 0.7, -top * 0.7, top / 4, 2.36e38, 2.37e38, -2.37e38, 1e30, -1e30, 130.0, 133.0, -130.0, -133.0, -200.0, -60.0,
                          -64.5, -66.0, -67.5, -87.0, -87.25, -87.5, -88.0, -88.5, -88.75, -89.0, -91.0, -95.0, -100.0, -104.0, -110.0, 87.5, 89.0, 40.0,
                          0.0, -0.0, 1e-30, -1e-30, 2.0 ** -20, -1.0, 1.0, -16.0, 16.0, -17.5, math.inf, -math.inf, math.nan], dtype=torch.float32)
    gates = torch.cat([gates[gates.abs() <= top], gates[-3:]]).to(dtype)
    up = torch.linspace(0.51, 0.99, 32).to(dtype) * (2.0 ** [0, -60 if dtype != torch.float16 else -4, 40 if dtype != torch.float16 else 10][far])
    h = torch.cat([gates.view(-1, 1).expand(-1, 32), up.to(dtype).expand(len(gates), 32)], dim=1).contiguous()
    codes, scales = (t.cpu() for t in vp.mxfp4_quantize(h.cuda(), gated=True))
    gate, f = h[:, :32].double(), h[:, 32:].double()
    a = gate / (1 + torch.exp(-gate))                 # (e^-x of 64 bits does not overflow before -709)
    a = torch.where(gate < -700, gate * 0, a)
    off, least = 5 * 2.0 ** -23, 2.0 ** -150
    lo, hi = a - (a.abs() * off + least), a + (a.abs() * off + least)
    lo, hi = lo * f, hi * f                           # (f > 0)
    lo, hi = lo - (lo.abs() * 2.0 ** -24 + least), hi + (hi.abs() * 2.0 ** -24 + least)
    beyond = torch.finfo(torch.float32).max
    bad = ~torch.isfinite(a * f).all(dim=1) | ((a * f).abs() > beyond).any(dim=1)
    assert torch.equal(scales.view(-1) == 255, bad) and (codes[bad] == 0).all() and int(bad.sum()) >= 3
    got = ref.decode(codes, scales)
    for r in torch.nonzero(~bad).view(-1).tolist():
        # The scale is one of those between the least and the largest magnitude that the block can have; under it the codes lie between the ends'.
        least_of = torch.where((lo[r] <= 0) & (hi[r] >= 0), 0.0, torch.minimum(lo[r].abs(), hi[r].abs()))
        ends = [float(m.max()) for m in (least_of, torch.maximum(lo[r].abs(), hi[r].abs()))]
        want = [max(math.frexp(m)[1] - 3, -127) if m > 0 else -127 for m in ends]
        e = int(scales[r, 0]) - 127
        assert want[0] <= e <= want[1], (float(gates[r]), e, want)
        step = 2.0 ** e
        at = [torch.tensor([_nearest(float(v) / step) for v in x[r]], dtype=torch.float64) * step for x in (lo, hi)]
        assert ((at[0] <= got[r]) & (got[r] <= at[1])).all(), float(gates[r])


def _nearest(x):
    """The value of the grid next to x: ties to even, magnitudes above 6 to 6."""
    a = min(abs(x), 6.0)
    step = 0.5 if a < 2 else (1.0 if a < 4 else 2.0)
    return math.copysign(round(a / step) * step, x)       # (Python rounds ties to even; a grid point's code is even where its quotient is)


def test_quantize_refuses(vp):
    x = torch.zeros(4, 64, device="cuda")
    codes, scales = torch.zeros(4, 32, dtype=torch.uint8, device="cuda"), torch.zeros(4, 2, dtype=torch.uint8, device="cuda")
    for bad in (lambda: vp.mxfp4_quantize(torch.zeros(4, 48, device="cuda")), lambda: vp.mxfp4_quantize(x.double(), codes, scales),
                lambda: vp.mxfp4_quantize(x, codes), lambda: vp.mxfp4_quantize(x, codes[:3], scales), lambda: vp.mxfp4_quantize(x, codes, scales[:, :1]),
                lambda: vp.mxfp4_quantize(x, codes.int(), scales), lambda: vp.mxfp4_quantize(x, codes, scales, gated=True),
                lambda: vp.mxfp4_quantize(x.t(), codes, scales), lambda: vp.mxfp4_quantize(x, codes.cpu(), scales),
                lambda: vp.mxfp4_quantize(x[:1].expand(4, 64), codes, scales), lambda: vp.mxfp4_quantize(x, codes[:1].expand(4, 32), scales),
                lambda: vp.mxfp4_quantize(x, codes, scales, n_rows=torch.zeros(1, dtype=torch.int64, device="cuda")),
                lambda: vp.mxfp4_dequantize(codes, scales, torch.zeros(4, 60, device="cuda")),
                lambda: vp.mxfp4_dequantize(codes, scales, torch.zeros(4, 64, device="cuda").double())):
        with pytest.raises(AssertionError):
            bad()
    before = vp.kernel_launch_count()
    vp.mxfp4_quantize(x[:0], codes[:0], scales[:0])
    vp.mxfp4_dequantize(codes[:0], scales[:0])
    assert vp.kernel_launch_count() == before


# ---- the experts' products ------------------------------------------------------------------------------------------------

def _operands(counts, F, K, seed, spare=0, first=0):
    """Rows of 4-bit values in wire format, matrices, offsets; scales range over 2^-6 .. 2^6."""
    g = _gen(seed)
    cap, E = first + sum(counts) + spare, len(counts)
    x_code, x_scale = torch.randint(0, 16, (cap, K), generator=g), torch.randint(121, 134, (cap, K // 32), generator=g)
    w_code, w_scale = torch.randint(0, 16, (E, F, K), generator=g), torch.randint(121, 134, (E, F, K // 32), generator=g)
    off = torch.tensor([first] + counts).cumsum(0).to(torch.int32)
    to8 = lambda t: t.to(torch.uint8)  # noqa: E731
    return dict(xc=ref.pack_codes(to8(x_code)), xs=to8(x_scale), wc=ref.pack_codes(to8(w_code)), ws=to8(w_scale), off=off, cap=cap, F=F, K=K)


def _wire(vp, o):
    buf = torch.full((o["cap"], vp.mxfp4_row_bytes(o["K"])), 0xEE, dtype=torch.uint8, device="cuda")
    codes, scales = vp.mxfp4_rows(buf, o["K"])
    codes.copy_(o["xc"])
    scales.copy_(o["xs"])
    return codes, scales


def _bound(o, size, want, dtype):
    """Products are exact, and so are sums of 32 of them under one pair of scales; each addition in 32 bits is off by at most a unit in
    the last place of what has been added up (K / 32 blocks, and their parts)."""
    return (o["K"] / 16 + 16) * 2.0 ** -23 * size + 1.01 * ref.HALF_STEP[dtype] * want.abs() + ref.LEAST[dtype]


def _near(o, got, want, size, dtype):
    """Within the bound; what fp16 does not hold (from 65,520 on) is an infinity of that sign."""
    bound = _bound(o, size, want, dtype)
    beyond = (want.abs() + bound >= 65520) & (got.double() == want.sign() * math.inf) & (dtype == torch.float16)
    return ((got.double() - want).abs() <= bound) | beyond


def _product(vp, o, dtype, wire=True, out=None, status=None):
    codes, scales = _wire(vp, o) if wire else (o["xc"].cuda(), o["xs"].cuda())
    if out is None:
        out = torch.full((o["cap"], o["F"]), 3.0, dtype=dtype, device="cuda")
    out, status = vp.mxfp4_product(codes, scales, o["wc"].cuda(), o["ws"].cuda(), o["off"].cuda(), out, status)
    torch.cuda.synchronize()
    return out.cpu(), int(status)


def _expected(o):
    return ref.product(ref.decode(o["xc"], o["xs"]), ref.decode(o["wc"], o["ws"]), o["off"].tolist(), o["cap"])


def _check(vp, o, dtype, **kw):
    got, status = _product(vp, o, dtype, **kw)
    want, size = _expected(o)
    assert status == 0
    first, last = int(o["off"][0]), int(o["off"][-1])
    inside = slice(first, last)
    assert _near(o, got, want, size, dtype)[inside].all()
    assert (got[:first] == 3).all() and (got[last:] == 3).all()


def test_product_of_one_block(vp):
    """One row, one feature, 32 values: the sum by hand."""
    o = _operands([1], 1, 32, 0)
    got, status = _product(vp, o, torch.float32)
    want, _ = _expected(o)
    assert status == 0 and float(got[0, 0]) == float(want[0, 0])


@pytest.mark.parametrize("u", range(8))
def test_product_takes_every_scale_from_its_own_place(vp, u):
    """Codes of 1, one block's scale apart from the others: rows, features and blocks of k are told apart."""
    o = _operands([128], 256, 256, u)
    o["xc"][:], o["wc"][:] = 0x22, 0x22
    o["xs"][:], o["ws"][:] = 127, 127
    o["xs"][:, u] = (torch.arange(128) % 13 + 121).to(torch.uint8)
    o["ws"][:, :, (u + 3) % 8] = (torch.arange(256) % 11 + 122).to(torch.uint8)
    got, status = _product(vp, o, torch.float32)
    want, _ = _expected(o)
    assert status == 0 and torch.equal(got.double(), want)


@pytest.mark.parametrize("counts", [[1], [127], [128], [129], [0, 3, 0, 0, 130, 1], [31, 32, 33, 64, 65]])
@pytest.mark.parametrize("F,K", [(8, 32), (1, 96), (100, 256), (256, 288), (257, 1056), (520, 2080)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_product_matches_the_definition(vp, counts, F, K, dtype):
    _check(vp, _operands(counts, F, K, F + K + len(counts), spare=3), dtype)


@pytest.mark.parametrize("counts,F,K", [([300] * 8, 4096, 512), ([2000, 0, 1, 900], 2048, 1024), ([4000], 2304, 768)])
@pytest.mark.parametrize("dtype", TYPES)
def test_product_of_many_tiles(vp, counts, F, K, dtype):
    """More tiles than SMs: both halves of tensor memory, features in tiles of 256."""
    _check(vp, _operands(counts, F, K, F + K, spare=5), dtype)


def test_product_does_not_depend_on_the_launch_shape(vp):
    """The same rows in a buffer of their own (one CTA to a tile) and in a large one (pairs of CTAs): the same bytes."""
    for F, K in ((2304, 768), (4096, 2080), (2048, 7168)):
        o = _operands([100], F, K, F + K, spare=3900)
        large, status = _product(vp, o, torch.float32)
        o["cap"], o["xc"], o["xs"] = 100, o["xc"][:100], o["xs"][:100]
        small, other = _product(vp, o, torch.float32)
        assert status == other == 0 and torch.equal(large[:100], small)


def test_product_of_long_rows(vp):
    _check(vp, _operands([5, 40], 300, 7168, 1), torch.bfloat16)


def test_product_of_contiguous_rows_and_offsets_that_do_not_begin_at_zero(vp):
    for K in (32, 64, 416, 1056):
        _check(vp, _operands([9, 0, 50], 130, K, K, spare=70, first=13), torch.float32, wire=False)


@pytest.mark.parametrize("K", [32, 416, 1024, 1056, 2080])
def test_product_of_scales_at_any_alignment(vp, K):
    """Rows of scales that begin at every byte of a sector and are any number of bytes apart; what lies around them is NaN."""
    o = _operands([130, 1, 30], 40, K, K)
    want, size = _expected(o)
    n = K // 32
    for first, width in ((0, n + 77), (1, n + 77), (2, n + 5), (3, n + 1), (16, n + 16), (29, n + 32)):
        flat = torch.full((162 * (n + 77),), 255, dtype=torch.uint8, device="cuda")
        scales = torch.as_strided(flat, (161, n), (width, 1), first)
        scales.copy_(o["xs"])
        out = torch.zeros(161, 40, device="cuda")
        vp.mxfp4_product(o["xc"].cuda(), scales, o["wc"].cuda(), o["ws"].cuda(), o["off"].cuda(), out)
        assert ((out.cpu().double() - want).abs() <= _bound(o, size, want, torch.float32)).all()


def test_product_of_a_thousand_experts(vp):
    g = _gen(6)
    counts = (torch.rand(1024, generator=g) < 0.3).long() * torch.randint(1, 4, (1024,), generator=g)
    _check(vp, _operands(counts.tolist(), 16, 64, 6), torch.bfloat16)


def test_product_without_rows(vp):
    o = _operands([0, 0, 0], 40, 64, 2, spare=9)
    got, status = _product(vp, o, torch.bfloat16)
    assert status == 0 and (got == 3).all()
    before = vp.kernel_launch_count()
    vp.mxfp4_product(o["xc"][:0].cuda(), o["xs"][:0].cuda(), o["wc"].cuda(), o["ws"].cuda(), o["off"].cuda())
    assert vp.kernel_launch_count() == before


@pytest.mark.parametrize("dtype", TYPES)
def test_product_into_strided_and_unaligned_rows(vp, dtype):
    o = _operands([40, 2], 72, 96, 4)
    want, size = _expected(o)
    for width, first in ((80, 0), (83, 5), (96, 8)):
        wide = torch.full((42, width), 3.0, dtype=dtype, device="cuda")
        _, status = _product(vp, o, dtype, out=wide[:, first:first + 72])
        got = wide.cpu()
        assert status == 0
        assert _near(o, got[:, first:first + 72], want, size, dtype).all()
        assert (got[:, :first] == 3).all() and (got[:, first + 72:] == 3).all()


def test_product_of_nan_scales_spoils_its_own_rows_and_features_only(vp):
    o = _operands([20, 20], 64, 128, 5)
    o["xs"][7, 1], o["ws"][1, 33, 0] = 255, 255
    got, status = _product(vp, o, torch.float32)
    want, size = _expected(o)
    spoilt = torch.isnan(want)
    assert status == 0 and spoilt[7].all() and spoilt[20:, 33].all() and int(spoilt.sum()) == 64 + 20
    assert torch.equal(torch.isnan(got), spoilt)
    assert ((got.double() - want).abs() <= _bound(o, size, want, torch.float32))[~spoilt].all()


def test_product_reports_offsets_that_fall_or_leave_the_buffer(vp):
    o = _operands([10, 10, 10], 32, 64, 7, spare=10)
    want, size = _expected(o)
    for off, rows in (([0, 10, 20, 41], (0, 20)), ([-3, 10, 20, 30], (0, 30)), ([0, 10, 5, 5], (0, 10)), ([50, 60, 70, 80], (0, 0))):
        o["off"] = torch.tensor(off, dtype=torch.int32)
        status = torch.full((1,), 4, dtype=torch.int32, device="cuda")
        got, st = _product(vp, o, torch.float32, status=status)
        assert st == 4 | vp.ST_PACK_MISMATCH              # OR-ed in
        inside = slice(*rows)
        assert ((got.double() - want).abs()[inside] <= _bound(o, size, want, torch.float32)[inside]).all()


def test_product_of_offsets_that_fall_gives_a_row_to_the_first_expert_that_reaches_it(vp):
    """Ranges that overlap as given: no row has two experts, and no row is summed twice."""
    o = _operands([50, 50, 30], 160, 320, 17, spare=70)
    for off, rows in (([0, 100, 50, 120], (100, 0, 20)), ([40, 10, 60, 50], (0, 20, 0)), ([0, 200, 0, 200], (200, 0, 0)), ([-7, 3, -9, 999], (3, 0, 197))):
        o["off"] = torch.tensor(off, dtype=torch.int32)
        at = min(max(off[0], 0), 200)
        want, size, used = torch.zeros(200, 160).double(), torch.zeros(200, 160).double(), torch.zeros(200, dtype=torch.bool)
        x, w = ref.decode(o["xc"], o["xs"]), ref.decode(o["wc"], o["ws"])
        for e, n in enumerate(rows):
            want[at:at + n], size[at:at + n], used[at:at + n] = x[at:at + n] @ w[e].T, x[at:at + n].abs() @ w[e].abs().T, True
            at += n
        got, status = _product(vp, o, torch.float32)
        assert status == vp.ST_PACK_MISMATCH
        assert ((got.double() - want).abs() <= _bound(o, size, want, torch.float32))[used].all() and (got[~used] == 3).all()


def test_product_of_many_experts_whose_offsets_fall(vp):
    """Offsets that fall again and again over several groups of 32 experts, behind groups whose offsets rise."""
    E = 100
    o = _operands([1] * E, 8, 32, 18, spare=28)
    off = list(range(40)) + [90 if e % 2 else 20 for e in range(40, E + 1)]
    o["off"] = torch.tensor(off, dtype=torch.int32)
    x, w = ref.decode(o["xc"], o["xs"]), ref.decode(o["wc"], o["ws"])
    expert = [e for e in range(39)] + [40] * (90 - 39)                # (expert 39 has none: its end is before its beginning)
    want = torch.stack([x[r] @ w[e].T for r, e in enumerate(expert)])
    size = torch.stack([x[r].abs() @ w[e].abs().T for r, e in enumerate(expert)])
    got, status = _product(vp, o, torch.float32)
    assert status == vp.ST_PACK_MISMATCH
    assert ((got[:90].double() - want).abs() <= _bound(o, size, want, torch.float32)).all() and (got[90:] == 3).all()


def test_product_in_a_graph_and_on_two_streams(vp):
    o, q = _operands([300, 200], 512, 512, 8), _operands([70, 430], 512, 512, 9)
    dev = {k: (v.cuda() if torch.is_tensor(v) else v) for k, v in o.items()}
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = torch.zeros(500, 512, device="cuda")
    call = lambda to, stream=None: vp.mxfp4_product(dev["xc"], dev["xs"], dev["wc"], dev["ws"], dev["off"], to, status, stream=stream)  # noqa: E731
    call(out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out)
    for other in (q, o):                              # new rows, matrices and offsets in the same buffers
        for k in ("xc", "xs", "wc", "ws", "off"):
            dev[k].copy_(other[k])
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        want, size = _expected(other)
        assert ((out.cpu().double() - want).abs() <= _bound(other, size, want, torch.float32)).all()
    streams, outs = [torch.cuda.Stream() for _ in range(2)], [torch.zeros_like(out) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(3):
        for s, to in zip(streams, outs):
            call(to, s)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], out) and torch.equal(outs[1], out) and int(status) == 0


@pytest.mark.parametrize("counts,F,K", [([1], 520, 7168), ([60, 20, 3], 600, 1056), ([2100], 2304, 2080), ([3000, 500], 4096, 1024)])
def test_product_whose_waits_run_out_reports_it_and_leaves_the_device_as_it_was(vp, counts, F, K):
    """Waits of few polls: the call ends, the status says so, rows outside the offsets keep what they hold, and the next call is right."""
    o = _operands(counts, F, K, F, spare=9)
    want, size = _expected(o)
    codes, scales = _wire(vp, o)
    wc, ws, off = o["wc"].cuda(), o["ws"].cuda(), o["off"].cuda()
    n, gave_up = sum(counts), 0
    fn = vp.binding._load().vp_mxfp4_product_polls
    for polls in (0, 1, 2, 3, 5, 8, 20, 60, 200, 1000, 1 << 22):
        out = torch.full((o["cap"], F), 3.0, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        i64, P = ctypes.c_int64, ctypes.c_void_p
        rc = fn(P(codes.data_ptr()), i64(codes.stride(0)), P(scales.data_ptr()), i64(scales.stride(0)), i64(o["cap"]), P(wc.data_ptr()), P(ws.data_ptr()),
                len(counts), i64(F), i64(K), P(off.data_ptr()), P(out.data_ptr()), 2, i64(F), P(status.data_ptr()),
                P(torch.cuda.current_stream().cuda_stream), ctypes.c_uint(polls))
        assert rc == 0
        torch.cuda.synchronize()
        assert int(status) in (0, vp.ST_INTERNAL_TIMEOUT) and (out[n:] == 3).all()
        if int(status) == 0:
            assert ((out.cpu().double() - want).abs() <= _bound(o, size, want, torch.float32))[:n].all()
        gave_up += int(status) != 0
        _check(vp, o, torch.float32)
    assert gave_up > 0 and int(status) == 0


def test_product_refuses(vp):
    o = _operands([4, 4], 16, 64, 1)
    d = {k: (v.cuda() if torch.is_tensor(v) else v) for k, v in o.items()}
    args = lambda **kw: [kw.get(k, d[k]) for k in ("xc", "xs", "wc", "ws", "off")]  # noqa: E731
    for bad in (dict(xc=d["xc"][:7]), dict(xs=d["xs"][:, :1]), dict(wc=d["wc"][:, :, :16]), dict(ws=d["ws"][:1]), dict(off=d["off"][:2]),
                dict(off=d["off"].long()), dict(xc=d["xc"].cpu()), dict(wc=d["wc"].transpose(0, 1)), dict(ws=d["ws"].int())):
        with pytest.raises(AssertionError):
            vp.mxfp4_product(*args(**bad), torch.zeros(8, 16, device="cuda"))
    for out in (torch.zeros(8, 15, device="cuda"), torch.zeros(7, 16, device="cuda"), torch.zeros(8, 16), torch.zeros(8, 16, device="cuda").double()):
        with pytest.raises(AssertionError):
            vp.mxfp4_product(*args(), out)
    odd = torch.zeros(8, 40, dtype=torch.uint8, device="cuda")
    for codes in (odd[:, :32], torch.zeros(8, 48, dtype=torch.uint8, device="cuda")[:, 8:40]):    # a stride, a start off 16 bytes
        with pytest.raises(vp.VpError) as e:
            vp.mxfp4_product(*args(xc=codes))
        assert e.value.code == vp.E_BAD_ARG
