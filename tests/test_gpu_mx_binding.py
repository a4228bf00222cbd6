"""The block-scaled calls' binding on the device: a given amax in its forms, and what a refused call leaves to the next one."""
import pytest
import torch

from test_gpu_mx import check_quantized, draw, fmt_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(lib):
    c = lib.Context.for_mx(512, 512, 512)
    yield c
    c.close()


def test_a_refused_call_leaves_the_next_one_its_own_amax(lib, ctx):
    x, f = draw(40, 200, "bf16", 3), lib.FP4_MX_NVFP4
    q, small = lib.MXTensor(40, 200, "cuda", f, True, True), torch.tensor([1e-3], device="cuda")
    for bad in (x[:39], x[:, :199], x.double(), x.cpu(), draw(200, 40, "bf16", 3).t()):
        with pytest.raises(AssertionError):
            lib.fp4_mx_quantize(ctx, bad, f, out=q, amax=small)
        check_quantized(lib.fp4_mx_quantize(ctx, x, f, out=q), x, "nvfp4")


def test_a_given_amax_in_its_forms(lib, ctx):
    x, f = draw(40, 200, "bf16", 4), lib.FP4_MX_NVFP4
    for amax in (torch.tensor([2.0], device="cuda"), torch.tensor(2.0, device="cuda"), torch.tensor([[2.0]], dtype=torch.float64), torch.tensor([9.0, 2.0], device="cuda")[1],
                 torch.tensor(2.0, dtype=torch.bfloat16, device="cuda", requires_grad=True)):
        q = lib.fp4_mx_quantize(ctx, x, f, True, True, amax=amax)
        assert float(q.amax) == 2.0 and q.struct.flags == 0
        check_quantized(q, x, "nvfp4", amax=2.0)
        check_quantized(lib.fp4_mx_quantize(ctx, x, f, out=q, amax=q.amax), x, "nvfp4", amax=2.0)      # the operand's own
        check_quantized(lib.fp4_mx_quantize(ctx, x, f, out=q), x, "nvfp4")


def test_a_flag_that_the_caller_set_stays(lib, ctx):
    x, f = draw(40, 200, "bf16", 5), lib.FP4_MX_NVFP4
    q = lib.MXTensor(40, 200, "cuda", f, True, True)
    q.struct.flags = 1
    q.amax.fill_(0.5)
    check_quantized(lib.fp4_mx_quantize(ctx, x, f, out=q, amax=torch.tensor([4.0], device="cuda")), x, "nvfp4", amax=4.0)
    assert q.struct.flags == 1
    check_quantized(lib.fp4_mx_quantize(ctx, x, f, out=q), x, "nvfp4", amax=4.0)


def test_a_given_amax_in_a_captured_call(lib, ctx):
    x, f = draw(40, 200, "bf16", 6), lib.FP4_MX_NVFP4
    q, amax, stream = lib.MXTensor(40, 200, "cuda", f, True, True), torch.tensor([1.0], device="cuda"), torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        lib.fp4_mx_quantize(ctx, x, f, out=q, amax=amax)
        stream.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            lib.fp4_mx_quantize(ctx, x, f, out=q, amax=amax)
    for a in (3.0, 0.25):
        amax.fill_(a)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        check_quantized(q, x, "nvfp4", amax=a)


@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4"])
def test_a_backward_pass_with_the_operand_it_reads(lib, ctx, fmt):
    f, M, K, N = fmt_of(lib, fmt), 70, 200, 130
    x, w, dy = draw(M, K, "bf16", 7), draw(K, N, "bf16", 8), draw(M, N, "bf16", 9)
    _, sx, sw = lib.fp4_mx_linear_fwd(ctx, x, w, f)
    dx, dw = lib.fp4_mx_linear_bwd(ctx, dy, sx, sw)
    only, none = lib.fp4_mx_linear_bwd(ctx, dy, None, sw, want_dw=False)
    assert none is None and torch.equal(only, dx)
    none, only = lib.fp4_mx_linear_bwd(ctx, dy, sx, None, want_dx=False)
    assert none is None and torch.equal(only, dw)
    with pytest.raises(lib.Fp4Error):
        lib.fp4_mx_linear_bwd(ctx, dy, sx, None)
