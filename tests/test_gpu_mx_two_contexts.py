"""Two contexts on two streams at once, one each as documented: the same bits as one after the other, eagerly and from two graphs."""
import pytest
import torch

from test_gpu_mx import draw, fmt_of

pytestmark = pytest.mark.gpu


class Side:
    """A layer's passes, SwiGLU and a token's pass on a context of its own, into buffers that stay."""

    def __init__(self, lib, f, seed, M, K, N):
        self.lib, self.f, self.ctx, self.stream = lib, f, lib.Context.for_mx(M, K, N), torch.cuda.Stream()
        self.x, self.w, self.dy = draw(M, K, "bf16", seed, 3.0), draw(K, N, "bf16", seed + 1, 3.0), draw(M, N, "bf16", seed + 2, 3.0)
        self.sx, self.sw = lib.MXTensor(M, K, "cuda", f, True, True), lib.MXTensor(K, N, "cuda", f, True, True)
        self.token, self.st = draw(1, K, "bf16", seed + 3, 3.0), lib.MXTensor(1, K, "cuda", f)
        self.ckpt = lib.SwigluCheckpoint(M, N, "cuda")
        new = lambda r, c: torch.empty((r, c), dtype=torch.bfloat16, device="cuda")               # noqa: E731
        self.outs = [new(M, N), new(M, K), new(K, N), new(1, N), new(M, N), new(M, N), new(M, N)]

    def run(self):
        y, dx, dw, t, h, dg, du = self.outs
        lib, c = self.lib, self.ctx
        lib.fp4_mx_linear_fwd(c, self.x, self.w, self.f, self.sx, self.sw, out=y)
        lib.fp4_mx_linear_bwd(c, self.dy, self.sx, self.sw, dX=dx, dW=dw)
        lib.fp4_mx_linear_fwd(c, self.token, None, self.f, self.st, self.sw, reuse_w=True, out=t)
        lib.fp4_mx_swiglu_fwd(c, y, self.dy, out=h, checkpoint=self.ckpt)
        lib.fp4_mx_swiglu_bwd(c, self.dy, self.ckpt, dgate=dg, dup=du)

    def same(self, want):
        return [torch.equal(a, b) for a, b in zip(self.outs, want)]

    def clear(self):
        for o in self.outs:
            o.zero_()


@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4"])
@pytest.mark.parametrize("sizes", [((40, 2048, 512), (8, 4096, 1024)), ((1500, 1024, 2000), (300, 700, 900)), ((2048, 2048, 2048), (16, 4096, 4096))])
def test_two_contexts_at_once(lib, fmt, sizes):
    sides = [Side(lib, fmt_of(lib, fmt), 10 * i, *s) for i, s in enumerate(sizes)]
    wants = []
    for s in sides:
        s.run()
        torch.cuda.synchronize()
        wants.append([o.clone() for o in s.outs])
        s.clear()
    torch.cuda.synchronize()
    for _ in range(10):
        for s in sides:
            with torch.cuda.stream(s.stream):
                s.run()
    torch.cuda.synchronize()
    for s, w in zip(sides, wants):
        assert all(s.same(w)), s.same(w)
        s.clear()
    graphs = []
    for s in sides:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s.stream):
            s.run()
            s.run()
        graphs.append(g)
    torch.cuda.synchronize()
    for _ in range(5):
        for s, g in zip(sides, graphs):
            with torch.cuda.stream(s.stream):
                g.replay()
    torch.cuda.synchronize()
    for s, w in zip(sides, wants):
        assert all(s.same(w)), s.same(w)
        assert s.ctx.read_status() == 0
        s.ctx.close()
