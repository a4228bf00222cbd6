"""Block-scaled ("microscaled") operands, their product, and SwiGLU with an 8-bit checkpoint, as cases that can be timed.

Every kind of case has a plain form in elementary torch operations (`own` is false) and the calls that a program makes of
the package (`own` is true).  Kinds:

  quantize  a tensor to blocks along its rows and along its columns, and back to the values the codes stand for
  gemm      the product of two operands that are there
  serve     forward of a linear whose weight was quantised when it was loaded, from one token on
  step      forward and backward of a linear, weight included (training)
  act       SwiGLU of a few tokens (serving: nothing is kept)
  swiglu    SwiGLU forward, gate and up kept in 8 bits, and its backward from them (training)
  mlp       forward and backward of the three linears of a gated MLP with SwiGLU between them (training)

Formats: "mxfp4" is E2M1 in blocks of 32 with a power of two each, the least one that lets the block's largest magnitude
fit; "nvfp4" is E2M1 in blocks of 16 with an E4M3 scale each and one power of two for the tensor, the least one that lets
its largest magnitude fit 6 * 448; the checkpoint is E4M3 in blocks of 32 with a power of two each.  Elements and E4M3
scales are rounded to the nearest value of the format, ties to even.

Sizes are those of the LLaMA 1.3B / 7B / 13B linears and anything between; activations are heavy-tailed with a few outlier
channels, weights normal (0.02), output gradients normal (1e-3).
"""
import math

import torch

own = False

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def listed():
    return [
        # one token of a 7B model through the up projection: latency, and the weight's bytes
        dict(name="serve-1-7b-up", kind="serve", M=1, K=4096, N=11008, fmt="mxfp4", dtype="bf16"),
        # a small batch of decoded tokens, long contraction
        dict(name="serve-24-13b-down", kind="serve", M=24, K=13824, N=5120, fmt="nvfp4", dtype="bf16"),
        # a prompt whose length fills no tile
        dict(name="serve-1921-1.3b-down", kind="serve", M=1921, K=5504, N=2048, fmt="mxfp4", dtype="bf16"),
        # the product by itself at a square size
        dict(name="gemm-8192", kind="gemm", M=8192, K=8192, N=8192, fmt="mxfp4", dtype="bf16"),
        # odd sizes all round, result in fp32 (rows of the result start off any alignment)
        dict(name="gemm-odd-f32", kind="gemm", M=1003, K=4100, N=2729, fmt="nvfp4", dtype="fp32"),
        # smallest layer of the test configurations: launches count
        dict(name="step-fc1024", kind="step", M=256, K=1024, N=1024, fmt="mxfp4", dtype="bf16"),
        # 13B gate projection, one micro-batch
        dict(name="step-13b-gate", kind="step", M=8192, K=5120, N=13824, fmt="nvfp4", dtype="bf16"),
        # an activation for forward and weight gradient
        dict(name="quantize-act", kind="quantize", M=8192, K=4096, fmt="mxfp4", dtype="bf16"),
        # a tensor with odd sides whose scale for the whole tensor has to be found first
        dict(name="quantize-odd", kind="quantize", M=4097, K=5511, fmt="nvfp4", dtype="fp16"),
        # activation of one decoded token
        dict(name="act-1-7b", kind="act", M=1, K=11008, dtype="bf16"),
        # activation of the largest layer, forward and backward
        dict(name="swiglu-13b", kind="swiglu", M=16384, K=13824, dtype="bf16"),
        # the whole MLP of a 1.3B decoder layer
        dict(name="mlp-1.3b", kind="mlp", M=4096, K=2048, N=5504, fmt="mxfp4", dtype="bf16"),
    ]


def _size(rng, lo, hi):
    """Any whole number, spread evenly over the logarithm of [lo, hi]."""
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    kind = rng.choices(["quantize", "gemm", "serve", "step", "act", "swiglu", "mlp"], [4, 4, 5, 4, 2, 3, 2])[0]
    fmt, dtype = rng.choice(["mxfp4", "nvfp4"]), rng.choice(["bf16", "bf16", "fp16"])
    if kind == "quantize":
        return dict(kind=kind, M=_size(rng, 1, 16384), K=_size(rng, 16, 8192), fmt=fmt,
                    dtype=rng.choice(["bf16", "fp16", "fp32"]))
    if kind == "gemm":
        dtype = rng.choice(["bf16", "fp16", "fp32"])
        return dict(kind=kind, M=_size(rng, 1, 8192), K=_size(rng, 32, 4096 if dtype == "fp32" else 8192),
                    N=_size(rng, 64, 8192), fmt=fmt, dtype=dtype)
    if kind == "serve":
        return dict(kind=kind, M=_size(rng, 1, 2048), K=_size(rng, 512, 13824), N=_size(rng, 512, 13824), fmt=fmt, dtype=dtype)
    if kind == "step":
        return dict(kind=kind, M=_size(rng, 64, 8192), K=_size(rng, 512, 5120), N=_size(rng, 512, 13824), fmt=fmt, dtype=dtype)
    if kind == "act":
        return dict(kind=kind, M=_size(rng, 1, 64), K=_size(rng, 512, 13824), dtype=rng.choice(["bf16", "fp16", "fp32"]))
    if kind == "swiglu":
        return dict(kind=kind, M=_size(rng, 64, 16384), K=_size(rng, 512, 13824), dtype=dtype)
    return dict(kind=kind, M=_size(rng, 128, 4096), K=_size(rng, 512, 2048), N=_size(rng, 512, 5504), fmt="mxfp4", dtype="bf16")


# ------------------------------------------------------------------------------- inputs -------
def _activation(g, rows, cols, dtype):
    """Student-t with five degrees of freedom, one channel in two hundred thirty times larger."""
    x = torch.randn((rows, cols), device=DEV, generator=g)
    d = torch.zeros_like(x)
    t = torch.empty_like(x)
    for _ in range(5):
        t.normal_(generator=g)
        d.addcmul_(t, t)
    x.mul_(d.div_(5.0).rsqrt_())
    x[:, torch.randperm(cols, device=DEV, generator=g)[:max(1, cols // 200)]] *= 30.0
    return x.to(DTYPES[dtype])


def _normal(g, rows, cols, std, dtype):
    return torch.randn((rows, cols), device=DEV, generator=g).mul_(std).to(DTYPES[dtype])


def _inputs(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    M, K, N, dt = case["M"], case["K"], case.get("N", 0), case["dtype"]
    kind = case["kind"]
    if kind == "quantize":
        return {"x": _activation(g, M, K, dt)}
    if kind == "gemm":
        return {"a": _activation(g, M, K, "bf16"), "b": _normal(g, N, K, 0.02, "bf16")}
    if kind == "serve":
        return {"x": _activation(g, M, K, dt), "w": _normal(g, K, N, 0.02, dt)}
    if kind == "step":
        return {"x": _activation(g, M, K, dt), "w": _normal(g, K, N, 0.02, dt), "dy": _normal(g, M, N, 1e-3, dt)}
    if kind in ("act", "swiglu"):
        s = {"gate": _normal(g, M, K, 1.5, dt), "up": _normal(g, M, K, 1.0, dt)}
        if kind == "swiglu":
            s["dh"] = _normal(g, M, K, 1e-3, dt)
        return s
    return {"x": _normal(g, M, K, 1.0, dt), "wg": _normal(g, K, N, 0.02, dt), "wu": _normal(g, K, N, 0.02, dt),
            "wd": _normal(g, N, K, 0.02, dt), "dy": _normal(g, M, K, 1e-3, dt)}


# ------------------------------------------------------------------------------- plain form ---
def _pow2(e):
    """2^e in fp32 for whole e in [-127, 127]."""
    return torch.where(e == -127, torch.full_like(e, 1 << 22), (e + 127) << 23).view(torch.float32)


def _least_exponent(amax, mantissa, shift):
    """The least e in [-127, 127] with amax <= MAX 2^e, where MAX = mantissa 2^shift (mantissa in [1/2, 1))."""
    m, ex = torch.frexp(amax)
    e = ex - shift + (m > mantissa).to(torch.int32)
    return torch.where(amax == 0, -127, e.clamp(-127, 127)).to(torch.int32)


def _round_e2m1(v):
    a = v.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    return torch.copysign((torch.round(a / step) * step).clamp(max=6.0), v)


def _round_e4m3(v):
    return v.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).float()


def _blocks(x, size):
    rows, cols = x.shape
    return torch.nn.functional.pad(x.float(), (0, -cols % size)).view(rows, -1, size)


def _fake(x, fmt):
    """The values that the codes of `x`, in blocks along its rows, stand for."""
    rows, cols = x.shape
    if fmt == "nvfp4":
        b = _blocks(x, 16)
        amax = b.abs().amax(2, keepdim=True)
        k = _least_exponent(amax.max(), 0.65625, 12).clamp(min=-100)
        s = _round_e4m3(amax * _pow2(-k) / 6.0)
        v = _round_e2m1(torch.where(s > 0, b * _pow2(-k) / s, 0.0)) * s * _pow2(k)
    else:
        b = _blocks(x, 32)
        amax = b.abs().amax(2, keepdim=True)
        if fmt == "mxfp4":
            e = _least_exponent(amax, 0.75, 3)
            v = _round_e2m1(b * _pow2(-e)) * _pow2(e)
        else:
            e = _least_exponent(amax, 0.875, 9)
            v = _round_e4m3(b * _pow2(-e)) * _pow2(e)
    return v.view(rows, -1)[:, :cols]


def _fake_t(x, fmt):
    """The same in blocks along the columns: the transposed values."""
    return _fake(x.t().contiguous(), fmt)


def _swiglu(g, u, dtype):
    return (g / (1.0 + torch.exp(-g)) * u).to(dtype)


def _swiglu_grad(g, u, dh, dtype):
    s = 1.0 / (1.0 + torch.exp(-g))
    dh = dh.float()
    return (dh * u * s * (1.0 + g * (1.0 - s))).to(dtype), (dh * g * s).to(dtype)


def _plain_mlp(s):
    x, fmt, dt = s["x"], s["case"]["fmt"], s["x"].dtype
    xq = _fake(x, fmt)
    gate = (xq @ _fake_t(s["wg"], fmt).t()).to(dt)
    up = (xq @ _fake_t(s["wu"], fmt).t()).to(dt)
    h = _swiglu(gate.float(), up.float(), dt)
    y = (_fake(h, fmt) @ _fake_t(s["wd"], fmt).t()).to(dt)
    g, u = _fake(gate, "mxfp8"), _fake(up, "mxfp8")
    dh = (_fake(s["dy"], fmt) @ _fake(s["wd"], fmt).t()).to(dt)
    dgate, dup = _swiglu_grad(g, u, dh, dt)
    dwd = (_fake_t(_swiglu(g, u, dt), fmt) @ _fake_t(s["dy"], fmt).t()).to(dt)
    xt = _fake_t(x, fmt)
    dwg = (xt @ _fake_t(dgate, fmt).t()).to(dt)
    dwu = (xt @ _fake_t(dup, fmt).t()).to(dt)
    dx = (_fake(dgate, fmt) @ _fake(s["wg"], fmt).t()).to(dt)
    dx = (dx.float() + _fake(dup, fmt) @ _fake(s["wu"], fmt).t()).to(dt)
    return {"y": y, "dx": dx, "dwg": dwg, "dwu": dwu, "dwd": dwd}


def _plain(s):
    case = s["case"]
    kind, fmt, dt = case["kind"], case.get("fmt"), DTYPES[case["dtype"]]
    if kind == "quantize":
        return _fake(s["x"], fmt).to(torch.bfloat16), _fake_t(s["x"], fmt).to(torch.bfloat16)
    if kind == "gemm":
        return (s["a"] @ s["b"].t()).to(dt)
    if kind == "serve":
        return (_fake(s["x"], fmt) @ s["w"].t()).to(dt)
    if kind == "step":
        x, w, dy = s["x"], s["w"], s["dy"]
        return {"y": (_fake(x, fmt) @ _fake_t(w, fmt).t()).to(dt), "dx": (_fake(dy, fmt) @ _fake(w, fmt).t()).to(dt),
                "dw": (_fake_t(x, fmt) @ _fake_t(dy, fmt).t()).to(dt)}
    if kind == "act":
        return _swiglu(s["gate"].float(), s["up"].float(), dt)
    if kind == "swiglu":
        h = _swiglu(s["gate"].float(), s["up"].float(), dt)
        dgate, dup = _swiglu_grad(_fake(s["gate"], "mxfp8"), _fake(s["up"], "mxfp8"), s["dh"], dt)
        return {"h": h, "dgate": dgate, "dup": dup}
    return _plain_mlp(s)


# ------------------------------------------------------------------------------- own calls ----
def _own_buffers(s):
    """What a program that uses the package holds beside its tensors: a context and the buffers it calls with."""
    import paper_2501_17116_b200 as fp4
    case = s["case"]
    kind, M, K, N, dt = case["kind"], case["M"], case["K"], case.get("N", 0), DTYPES[case["dtype"]]
    fmt = fp4.FP4_MX_NVFP4 if case.get("fmt") == "nvfp4" else fp4.FP4_MX_E2M1
    s["ctx"] = fp4.Context.for_mx(M, K, N)
    new = lambda rows, cols, t=dt: torch.empty((rows, cols), dtype=t, device=DEV)                  # noqa: E731
    mx = lambda rows, cols, **kw: fp4.MXTensor(rows, cols, DEV, fmt=fmt, **kw)                     # noqa: E731
    if kind == "quantize":
        s.update(q=mx(M, K, codes_t=True), out=new(M, K, torch.bfloat16), out_t=new(K, M, torch.bfloat16))
    elif kind == "gemm":
        s.update(qa=fp4.fp4_mx_quantize(s["ctx"], s["a"], fmt=fmt), qb=fp4.fp4_mx_quantize(s["ctx"], s["b"], fmt=fmt), out=new(M, N))
    elif kind == "serve":
        s.update(sx=mx(M, K), out=new(M, N), sw=fp4.fp4_mx_quantize(s["ctx"], s["w"], fmt=fmt, codes=False, codes_t=True))
        del s["w"]
    elif kind == "step":
        s.update(sx=mx(M, K, codes_t=True), sw=mx(K, N, codes_t=True), y=new(M, N), dx=new(M, K), dw=new(K, N))
    elif kind == "act":
        s.update(h=new(M, K))
    elif kind == "swiglu":
        s.update(h=new(M, K), ckpt=fp4.SwigluCheckpoint(M, K, DEV), dgate=new(M, K), dup=new(M, K))
    else:
        s.update(sx=mx(M, K, codes_t=True), sg=mx(K, N, codes_t=True), su=mx(K, N, codes_t=True), sd=mx(N, K, codes_t=True),
                 gate=new(M, N), up=new(M, N), ckpt=fp4.SwigluCheckpoint(M, N, DEV), hq=mx(M, N), hqt=mx(M, N, codes=False, codes_t=True),
                 dyq=mx(M, K, codes_t=True), dh=new(M, N), dgate=new(M, N), dup=new(M, N),
                 y=new(M, K), dx=new(M, K), dwg=new(K, N), dwu=new(K, N), dwd=new(N, K))


def _own_mlp(fp4, s):
    c = s["ctx"]
    fp4.fp4_mx_linear_fwd(c, s["x"], s["wg"], saved_x=s["sx"], saved_w=s["sg"], out=s["gate"])
    fp4.fp4_mx_linear_fwd(c, s["x"], s["wu"], saved_x=s["sx"], saved_w=s["su"], reuse_x=True, out=s["up"])
    fp4.fp4_mx_swiglu_fwd(c, s["gate"], s["up"], checkpoint=s["ckpt"], quantized=s["hq"], want_h=False)
    fp4.fp4_mx_quantize(c, s["wd"], out=s["sd"])
    fp4.fp4_mx_gemm(c, s["hq"], s["sd"], b_t=True, out=s["y"])
    fp4.fp4_mx_quantize(c, s["dy"], out=s["dyq"])
    fp4.fp4_mx_gemm(c, s["dyq"], s["sd"], out=s["dh"])
    fp4.fp4_mx_swiglu_bwd(c, s["dh"], s["ckpt"], dgate=s["dgate"], dup=s["dup"], quantized=s["hqt"])
    fp4.fp4_mx_gemm(c, s["hqt"], s["dyq"], a_t=True, b_t=True, out=s["dwd"])
    fp4.fp4_mx_linear_bwd(c, s["dgate"], s["sx"], s["sg"], dX=s["dx"], dW=s["dwg"])
    fp4.fp4_mx_linear_bwd(c, s["dup"], s["sx"], s["su"], dX=s["dx"], dW=s["dwu"], accumulate_dx=True)
    return {k: s[k] for k in ("y", "dx", "dwg", "dwu", "dwd")}


def _own(s):
    import paper_2501_17116_b200 as fp4
    c, kind = s["ctx"], s["case"]["kind"]
    if kind == "quantize":
        fp4.fp4_mx_quantize(c, s["x"], out=s["q"])
        return fp4.fp4_mx_dequantize(c, s["q"], out=s["out"]), fp4.fp4_mx_dequantize(c, s["q"], transposed=True, out=s["out_t"])
    if kind == "gemm":
        return fp4.fp4_mx_gemm(c, s["qa"], s["qb"], out=s["out"])
    if kind == "serve":
        return fp4.fp4_mx_linear_fwd(c, s["x"], None, saved_x=s["sx"], saved_w=s["sw"], reuse_w=True, out=s["out"])[0]
    if kind == "step":
        fp4.fp4_mx_linear_fwd(c, s["x"], s["w"], saved_x=s["sx"], saved_w=s["sw"], out=s["y"])
        fp4.fp4_mx_linear_bwd(c, s["dy"], s["sx"], s["sw"], dX=s["dx"], dW=s["dw"])
        return {"y": s["y"], "dx": s["dx"], "dw": s["dw"]}
    if kind == "act":
        return fp4.fp4_mx_swiglu_fwd(c, s["gate"], s["up"], out=s["h"])[0]
    if kind == "swiglu":
        fp4.fp4_mx_swiglu_fwd(c, s["gate"], s["up"], out=s["h"], checkpoint=s["ckpt"])
        fp4.fp4_mx_swiglu_bwd(c, s["dh"], s["ckpt"], dgate=s["dgate"], dup=s["dup"])
        return {"h": s["h"], "dgate": s["dgate"], "dup": s["dup"]}
    return _own_mlp(fp4, s)


# ------------------------------------------------------------------------------- the cases ----
def prepare(case, seed):
    s = {"case": case, **_inputs(case, seed)}
    if own:
        _own_buffers(s)
    elif case["kind"] == "gemm":                     # operands that were quantised earlier, as the values they stand for
        s["a"], s["b"] = _fake(s["a"], case["fmt"]), _fake(s["b"], case["fmt"])
    elif case["kind"] == "serve":
        s["w"] = _fake_t(s["w"], case["fmt"])
    return s


def run(s):
    return _own(s) if own else _plain(s)


def work(case):
    """Inputs read once, outputs written once; what is kept for the backward pass is written once and read once."""
    kind, M, K, N = case["kind"], case["M"], case["K"], case.get("N", 0)
    b = 4 if case["dtype"] == "fp32" else 2
    code = 0.5 + (1 / 16 if case.get("fmt") == "nvfp4" else 1 / 32)            # bytes of a value in 4 bits, its scale included
    kept = 1 + 1 / 32                                                         # and in 8
    if kind == "quantize":                           # both directions, written and read, and both results in BF16
        return {"bytes": M * K * (b + 4 * code + 4), "flops": 6.0 * M * K}
    if kind == "gemm":
        return {"bytes": code * (M * K + K * N) + b * M * N, "flops": 2.0 * M * K * N}
    if kind == "serve":
        return {"bytes": b * M * K + code * K * N + b * M * N, "flops": 2.0 * M * K * N}
    if kind == "step":                               # the operands of the backward pass stay until then
        return {"bytes": 2.0 * b * (M * K + K * N + M * N) + 2 * code * (M * K + K * N), "flops": 6.0 * M * K * N}
    if kind == "act":
        return {"bytes": 3.0 * b * M * K, "flops": 8.0 * M * K}
    if kind == "swiglu":
        return {"bytes": M * K * (6.0 * b + 4 * kept), "flops": 24.0 * M * K}
    weights, tokens = 3 * K * N, M * K
    return {"bytes": b * (2 * weights + 4 * tokens) + 2 * code * (tokens + weights) + M * N * 4 * kept, "flops": 18.0 * M * K * N}


# ------------------------------------------------------------------------------- in 64 bits ---
def _nearest_e2m1(v):
    """Nearest of 0, 1/2, 1, 3/2, 2, 3, 4, 6 by comparison with the midpoints; a tie goes to the even place in that list."""
    a = v.abs()
    place = torch.zeros_like(a, dtype=torch.long)
    for i, mid in enumerate((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)):
        place += (a >= mid) if i % 2 else (a > mid)
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=v.device)
    return torch.sign(v) * grid[place]


def _nearest_e4m3(v):
    a = v.abs()
    e = torch.floor(torch.log2(a.clamp(min=2.0 ** -6)))
    step = torch.exp2(e - 3)
    return torch.sign(v) * (torch.round(a / step) * step).clamp(max=448.0)


def _exact_values(x, fmt):
    x = x.double()
    rows, cols = x.shape
    size = 16 if fmt == "nvfp4" else 32
    wide = torch.zeros((rows, -(-cols // size) * size), dtype=torch.float64, device=x.device)
    wide[:, :cols] = x
    b = wide.view(rows, -1, size)
    top = b.abs().max(2, keepdim=True)[0]
    if fmt == "nvfp4":
        g = 2.0 ** max(math.ceil(math.log2(max(float(x.abs().max()) / 2688.0, 2.0 ** -100))), -100)
        scale = _nearest_e4m3(top / 6.0 / g)
        v = _nearest_e2m1(torch.where(scale > 0, b / g / scale, 0.0)) * scale * g
    else:
        most = 6.0 if fmt == "mxfp4" else 448.0
        e = torch.ceil(torch.log2((top / most).clamp(min=2.0 ** -127))).clamp(min=-127)
        e = torch.where(top > most * torch.exp2(e), e + 1, e)
        e = torch.where((top <= most * torch.exp2(e - 1)) & (e > -127), e - 1, e)
        scale = torch.exp2(e)
        v = (_nearest_e2m1 if fmt == "mxfp4" else _nearest_e4m3)(b / scale) * scale
    return v.view(rows, -1)[:, :cols]


def _exact_h(g, u):
    return g * torch.sigmoid(g) * u


def _exact_grad(g, u, dh):
    s = torch.sigmoid(g)
    return dh * u * s * (1 + g * torch.sigmoid(-g)), dh * g * s


def exact(case, seed):
    s = _inputs(case, seed)
    kind, fmt, dt = case["kind"], case.get("fmt"), DTYPES[case["dtype"]]
    q = lambda x: _exact_values(x, fmt)                                # noqa: E731
    qt = lambda x: _exact_values(x.t(), fmt)                           # noqa: E731
    if kind == "quantize":
        return q(s["x"]), qt(s["x"])
    if kind == "gemm":
        return q(s["a"]) @ q(s["b"]).t()
    if kind == "serve":
        return q(s["x"]) @ qt(s["w"]).t()
    if kind == "step":
        return {"y": q(s["x"]) @ qt(s["w"]).t(), "dx": q(s["dy"]) @ q(s["w"]).t(), "dw": qt(s["x"]) @ qt(s["dy"]).t()}
    if kind == "act":
        return _exact_h(s["gate"].double(), s["up"].double())
    if kind == "swiglu":
        dgate, dup = _exact_grad(_exact_values(s["gate"], "mxfp8"), _exact_values(s["up"], "mxfp8"), s["dh"].double())
        return {"h": _exact_h(s["gate"].double(), s["up"].double()), "dgate": dgate, "dup": dup}
    # what stands between two operators of the MLP is held in its type: rounded there, as it is defined
    gate, up = (q(s["x"]) @ qt(s["wg"]).t()).to(dt), (q(s["x"]) @ qt(s["wu"]).t()).to(dt)
    h = _exact_h(gate.double(), up.double()).to(dt)
    g, u = _exact_values(gate, "mxfp8"), _exact_values(up, "mxfp8")
    dgate, dup = _exact_grad(g, u, (q(s["dy"]) @ q(s["wd"]).t()).to(dt).double())
    dgate, dup = dgate.to(dt), dup.to(dt)
    return {"y": q(h) @ qt(s["wd"]).t(), "dx": q(dgate) @ q(s["wg"]).t() + q(dup) @ q(s["wu"]).t(),
            "dwg": qt(s["x"]) @ qt(dgate).t(), "dwu": qt(s["x"]) @ qt(dup).t(), "dwd": qt(_exact_h(g, u).to(dt)) @ qt(s["dy"]).t()}
