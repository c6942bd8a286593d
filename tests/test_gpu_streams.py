"""Calls on a stream that is not the current one, with outputs that the call allocates: they belong to that stream."""
import os

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def vp():
    import paper_2609_34340_b200 as vp
    assert torch.cuda.is_available(), "these tests need a GPU"
    assert os.path.exists(vp.library_path()), "libvariopath.so has not been built"
    return vp


def _product_args(off):
    byte = lambda *s: torch.randint(0, 256, s, device="cuda", dtype=torch.uint8)  # noqa: E731
    scale = lambda *s: torch.full(s, 127, device="cuda", dtype=torch.uint8)  # noqa: E731
    return byte(40, 32), scale(40, 2), byte(2, 64, 32), scale(2, 64, 2), torch.tensor(off, device="cuda", dtype=torch.int32)


def test_a_status_is_cleared_on_the_calls_stream(vp):
    args = _product_args([0, 30, 20])                     # an offset falls
    vp.mxfp4_product(*args)                               # (loading a kernel waits for the whole device)
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(100_000_000)                        # the current stream is busy for some 50 ms
    _, status = vp.mxfp4_product(*args, stream=other)
    torch.cuda.synchronize()
    assert int(status) == vp.ST_PACK_MISMATCH


def _calls(vp):
    g = torch.Generator().manual_seed(1)
    p = vp.RouteParams(64, 4)
    z = torch.randn(500, 64, generator=g).cuda()
    idx, w = vp.route(p, z)
    rows, grad = torch.randn(2000, 256, generator=g).cuda(), torch.randn(500, 256, generator=g).cuda()
    codes, scales = vp.mxfp4_quantize(rows)
    args = _product_args([0, 10, 40])
    torch.cuda.synchronize()
    return {
        "route": lambda s: vp.route(p, z, stream=s),
        "route_backward": lambda s: [vp.route_backward(p, z, idx, w, stream=s)],
        "combine": lambda s: [vp.combine(rows, idx, w, stream=s)],
        "combine_backward": lambda s: vp.combine_backward(grad, rows, idx, w, stream=s),
        "mxfp4_quantize": lambda s: vp.mxfp4_quantize(rows, stream=s),
        "mxfp4_dequantize": lambda s: [vp.mxfp4_dequantize(codes, scales, stream=s)],
        "mxfp4_product": lambda s: vp.mxfp4_product(*args, stream=s),
    }


@pytest.mark.parametrize("name", ["route", "route_backward", "combine", "combine_backward", "mxfp4_quantize", "mxfp4_dequantize", "mxfp4_product"])
def test_memory_that_the_current_stream_still_writes_is_not_handed_out(vp, name):
    """Blocks of the outputs' sizes are freed while the current stream has not yet written to them: an output of a call on another stream
    in such a block would be overwritten."""
    call = _calls(vp)[name]
    want = [t.clone() for t in call(None)]
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(100_000_000)
    held = [torch.empty(((t.untyped_storage().nbytes() + 511) // 512 * 512,), dtype=torch.uint8, device="cuda") for t in want for _ in range(4)]
    for t in held:
        t.fill_(0x55)
    del held, t
    got = call(other)
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
