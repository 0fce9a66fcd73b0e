"""The operators around the heads, as cases to measure: the residual sum and
RMS norm in front of the layer (output in the layer's type or in 8 bits with
scales), its gradient, the quantisation of weights and activations to 8 bits,
and the 8-bit product with a scale per block of 128.

A case is one call of one operator ("op"):

  norm      h = x + residual (rounded to the type), y = h / sqrt(mean h^2 + eps) * w
            as y in the type, or ("out": "e4m3") in 8 bits with a scale per 128 columns
  norm_bwd  its gradient: dx (with the gradient that reaches h besides), dw
  quantize  8 bits with a scale per 1 x 128 ("block": 1) or 128 x 128 ("block": 128),
            of x or ("transpose") of its transpose
  gemm      C[m][n] = sum_k A[m][k] B[n][k], both in 8 bits, A scaled per 1 x 128,
            B per 128 x 128 ("block": 128) or per 1 x 128 ("block": 1)

A block's scale is max(largest magnitude / 448, 2^-126), the 8-bit type is
e4m3 (torch.float8_e4m3fn, largest value 448).
"""
import math

import torch

own = False

EPS = 1e-6
E4M3_MAX = 448.0
SCALE_MIN = 2.0 ** -126
F8 = torch.float8_e4m3fn


def _norm(T, d, dtype="bf16", out="e4m3", residual=True, name=None):
    c = dict(op="norm", T=T, d=d, dtype=dtype, out=out, residual=residual)
    return dict(c, name=name) if name else c


def _norm_bwd(T, d, dtype="bf16", residual=True, name=None):
    c = dict(op="norm_bwd", T=T, d=d, dtype=dtype, residual=residual)
    return dict(c, name=name) if name else c


def _quantize(rows, cols, dtype="bf16", block=1, transpose=False, name=None):
    c = dict(op="quantize", rows=rows, cols=cols, dtype=dtype, block=block, transpose=transpose)
    return dict(c, name=name) if name else c


def _gemm(M, N, K, dtype="bf16", block=128, name=None):
    c = dict(op="gemm", M=M, N=N, K=K, dtype=dtype, block=block)
    return dict(c, name=name) if name else c


def listed():
    return [
        # serving: four decoded tokens of a 1024-wide model enter the layer
        _norm(4, 1024, name="norm_decode_t4"),
        # prefill of the 16 x 128-head layer: 16384 tokens of 2048 columns
        _norm(16384, 2048, name="norm_prefill_t16384"),
        # fp32 users, ragged: no residual, a width that no tile divides, output not quantised
        _norm(3001, 1000, "f32", "type", False, name="norm_f32_ragged"),
        # training that 16-head layer: the norm's gradient over 16384 tokens
        _norm_bwd(16384, 2048, name="norm_bwd_t16384"),
        # the gradient of a short ragged batch in front of a narrow layer, no residual
        _norm_bwd(777, 640, "bf16", False, name="norm_bwd_ragged"),
        # a projection's weights, once per optimiser step
        _quantize(2048, 2048, "f32", 128, name="quantize_weights"),
        # activations of a training step, transposed for the weight gradient; a batch that no block divides
        _quantize(16301, 2048, "bf16", 1, True, name="quantize_transposed_ragged"),
        # serving: one decoded token through a wide projection, read once
        _gemm(1, 8192, 8192, name="gemm_decode_m1"),
        # the default benchmark's projection: 4096 tokens, 1024 -> 8 heads x 128
        _gemm(4096, 1024, 1024, name="gemm_t4096_1024"),
        # the headline layer's: 16384 tokens, 2048 -> 16 heads x 128
        _gemm(16384, 2048, 2048, name="gemm_t16384_2048"),
        # the weight gradient of that projection: contracts over a ragged batch, both operands scaled per row
        _gemm(2048, 2048, 16304, "f32", 1, name="gemm_weight_gradient"),
        # a large square product
        _gemm(8192, 8192, 8192, name="gemm_8192"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    largest = _cost(listed()[-1])
    while True:
        op = rng.choice(["norm", "norm", "norm_bwd", "quantize", "quantize", "gemm", "gemm", "gemm"])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        if op in ("norm", "norm_bwd"):
            d = rng.choice([1, 8, 16]) * _log_int(rng, 16, 512)
            if op == "norm_bwd":
                c = _norm_bwd(_log_int(rng, 1, 32768), d, dtype, rng.random() < 0.6)
            else:
                out = "e4m3" if d % 16 == 0 and rng.random() < 0.7 else "type"
                c = _norm(_log_int(rng, 1, 65536), d, dtype, out, rng.random() < 0.6)
        elif op == "quantize":
            c = _quantize(_log_int(rng, 1, 32768), 16 * _log_int(rng, 4, 512), dtype,
                          rng.choice([1, 1, 128]), rng.random() < 0.4)
        else:
            c = _gemm(_log_int(rng, 1, 32768), _log_int(rng, 64, 8192), 16 * _log_int(rng, 4, 1024),
                      dtype, rng.choice([128, 128, 1]))
        if _cost(c) <= largest:
            return c


def work(case):
    c = case
    if c["op"] == "gemm":
        M, N, K = c["M"], c["N"], c["K"]
        g = -(-K // 128)
        scales = M * g + (N if c["block"] == 1 else -(-N // 128)) * g
        return {"bytes": M * K + N * K + 4 * scales + M * N * _size(c), "flops": 2 * M * N * K}
    if c["op"] == "quantize":
        n = c["rows"] * c["cols"]
        return {"bytes": n * (_size(c) + 1) + 4 * n / (128 * c["block"]), "flops": 3 * n}
    n, e = c["T"] * c["d"], _size(c)
    if c["op"] == "norm_bwd":
        return {"bytes": n * e * (4 if c["residual"] else 3) + 8 * c["d"], "flops": 9 * n}
    out = n + 4 * n / 128 if c["out"] == "e4m3" else n * e
    return {"bytes": n * e * (3 if c["residual"] else 1) + out + 4 * c["d"], "flops": 6 * n}


def _cost(c):
    # seconds at about half of what the card's memory and its fp32 products
    # give: the plain forms compute products in 32 bits
    w = work(c)
    return w["bytes"] / 2e12 + (w["flops"] / 5e13 if c["op"] == "gemm" else 0)


def _size(c):
    return 4 if c["dtype"] == "f32" else 2


def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt = _dtype(c)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    def buf(shape, dtype):
        return torch.empty(shape, dtype=dtype, device="cuda")

    s = {"case": c}
    if c["op"] in ("norm", "norm_bwd"):
        T, d = c["T"], c["d"]
        # activations whose rows differ in size, as a residual stream's do
        s["x"] = (normal(T, d) * torch.exp(normal(T, 1))).to(dt)
        s["w"] = 1.0 + 0.2 * normal(d)
        if c["op"] == "norm":
            s["residual"] = normal(T, d).to(dt) if c["residual"] else None
            s["sum"] = buf((T, d), dt) if c["residual"] else None
            if c["out"] == "e4m3":
                s["q"], s["scales"] = buf((T, d), F8), buf((T, -(-d // 128)), torch.float32)
            else:
                s["y"] = buf((T, d), dt)
        else:
            s["dy"] = normal(T, d).to(dt)
            s["dsum"] = normal(T, d).to(dt) if c["residual"] else None
            s["dx"], s["dw"] = buf((T, d), dt), buf((d,), torch.float32)
            s["ws"] = {}
    elif c["op"] == "quantize":
        R, C = c["rows"], c["cols"]
        s["x"] = (normal(R, C) * torch.exp(normal(R, 1))).to(dt)
        a, k = (C, -(-R // 16) * 16) if c["transpose"] else (R, C)
        s["q"] = buf((a, k), F8)
        s["scales"] = buf((-(-a // c["block"]), -(-k // 128)), torch.float32)
    else:
        M, N, K = c["M"], c["N"], c["K"]
        s["A"], s["sa"] = _quantized(normal(M, K) * torch.exp(0.5 * normal(M, 1)), 1)
        s["B"], s["sb"] = _quantized(normal(N, K) * K ** -0.5, c["block"])
        s["C"] = buf((M, N), dt)
    return s


def _blocks(x, block):
    """x [a, k] padded with zeros to whole blocks, as [a / block, block, k / 128, 128]."""
    a, k = x.shape
    x = torch.nn.functional.pad(x, (0, -k % 128, 0, -a % block))
    return x.view(x.shape[0] // block, block, x.shape[1] // 128, 128)


def _quantized(x, block):
    """e4m3 of x (fp32) and the scales of its blocks."""
    a, k = x.shape
    b = _blocks(x, block)
    scales = (b.abs().amax(dim=(1, 3)) / E4M3_MAX).clamp(min=SCALE_MIN)
    q = (b / scales[:, None, :, None]).clamp(-E4M3_MAX, E4M3_MAX).to(F8)
    q = q.view(torch.uint8).reshape(b.shape[0] * block, -1)[:a, :k].contiguous().view(F8)
    return q, scales


def _values(q, scales, block):
    """What 8 bits and their scales stand for, in 32 bits."""
    a, k = q.shape
    s = scales.repeat_interleave(block, 0)[:a].repeat_interleave(128, 1)[:, :k]
    return q.float() * s


def run(state):
    s = state
    c = s["case"]
    if own:
        return _run_own(s, c)
    if c["op"] == "norm":
        h = s["x"].float()
        res = {}
        if c["residual"]:
            res["sum"] = (h + s["residual"].float()).to(s["x"].dtype)
            h = res["sum"].float()
        y = h * torch.rsqrt((h * h).mean(dim=1, keepdim=True) + EPS) * s["w"]
        if c["out"] == "e4m3":
            res["q"], res["scales"] = _quantized(y, 1)
        else:
            res["y"] = y.to(s["x"].dtype)
        return res
    if c["op"] == "norm_bwd":
        h, dy = s["x"].float(), s["dy"].float()
        rs = torch.rsqrt((h * h).mean(dim=1, keepdim=True) + EPS)
        n = h * rs
        g = dy * s["w"]
        dx = rs * (g - n * (g * n).mean(dim=1, keepdim=True))
        if c["residual"]:
            dx = dx + s["dsum"].float()
        return {"dx": dx.to(s["x"].dtype), "dw": (dy * n).sum(dim=0)}
    if c["op"] == "quantize":
        x = s["x"].float()
        if c["transpose"]:
            x = torch.nn.functional.pad(x, (0, 0, 0, -x.shape[0] % 16)).t()
        q, scales = _quantized(x, c["block"])
        return {"q": q, "scales": scales}
    A = _values(s["A"], s["sa"], 1)
    B = _values(s["B"], s["sb"], c["block"])
    return {"C": (A @ B.t()).to(_dtype(c))}


def _run_own(s, c):
    import paper_2602_04870_amd as mh

    if c["op"] == "norm":
        if c["out"] == "e4m3":
            r = mh.mhlmoe_rmsnorm(s["x"], s["w"], EPS, residual=s["residual"], sum=s["sum"], q=s["q"],
                                  scales=s["scales"], quantized=True)
            res = {"q": r["q"], "scales": r["scales"]}
        else:
            r = mh.mhlmoe_rmsnorm(s["x"], s["w"], EPS, residual=s["residual"], sum=s["sum"], y=s["y"])
            res = {"y": r["y"]}
        return dict(res, sum=r["sum"]) if c["residual"] else res
    if c["op"] == "norm_bwd":
        # the workspace is made by the first call and kept, as a training loop keeps it
        if "buffer" not in s["ws"]:
            n = mh.mhlmoe_rmsnorm_backward_workspace(c["T"], c["d"])
            s["ws"]["buffer"] = torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")
        dx, dw = mh.mhlmoe_rmsnorm_backward(s["x"], s["w"], EPS, s["dy"], dsum=s["dsum"], dx=s["dx"],
                                            dweight=s["dw"], workspace=s["ws"]["buffer"])
        return {"dx": dx, "dw": dw}
    if c["op"] == "quantize":
        q, scales = mh.mhlmoe_quantize(s["x"], block_rows=c["block"], transpose=c["transpose"],
                                       q=s["q"], scales=s["scales"])
        return {"q": q, "scales": scales}
    return {"C": mh.mhlmoe_gemm_scaled(s["A"], s["sa"], s["B"], s["sb"], b_block_rows=c["block"],
                                       dtype=_dtype(c), C=s["C"])}


def exact(case, seed):
    """The same outputs from the definitions, in 64 bits."""
    c = case
    s = prepare(case, seed)
    f64 = torch.float64
    if c["op"] == "gemm":
        M, N, K = c["M"], c["N"], c["K"]
        C = torch.empty((M, N), dtype=f64, device="cuda")
        col = torch.arange(K, device="cuda") // 128
        row = torch.arange(N, device="cuda") // c["block"]
        B = s["B"].to(f64)
        B *= s["sb"].to(f64)[row][:, col]
        for m in range(0, M, 4096):
            A = s["A"][m:m + 4096].to(f64) * s["sa"][m:m + 4096].to(f64)[:, col]
            C[m:m + 4096] = torch.mm(A, B.t())
        return {"C": C}
    if c["op"] == "quantize":
        x = s["x"].to(f64)
        if c["transpose"]:
            x = x.t().contiguous()
        q, scales = _exact_e4m3(x, c["block"], s["q"].shape[1])
        return {"q": q, "scales": scales}
    x, w = s["x"].to(f64), s["w"].to(f64)
    if c["op"] == "norm":
        res = {}
        if c["residual"]:
            total = x + s["residual"].to(f64)
            res["sum"] = total
            x = total.to(s["x"].dtype).to(f64)  # the norm is that of the stored sum
        norm = torch.linalg.vector_norm(x, dim=1, keepdim=True)
        y = x * w / torch.sqrt(norm ** 2 / c["d"] + EPS)
        if c["out"] == "e4m3":
            res["q"], res["scales"] = _exact_e4m3(y, 1, c["d"])
        else:
            res["y"] = y
        return res
    dy = s["dy"].to(f64)
    r = torch.sqrt(x.square().sum(dim=1) / c["d"] + EPS)
    wdy = dy * w
    dot = (wdy * x).sum(dim=1) / (c["d"] * r ** 3)
    dx = wdy / r[:, None] - x * dot[:, None]
    if c["residual"]:
        dx += s["dsum"].to(f64)
    return {"dx": dx, "dw": torch.mv((dy * x).t(), 1.0 / r)}


def _exact_e4m3(x, block, width):
    """Each block by itself: its scale, and its values over the scale rounded
    to e4m3 by the type's own grid (3 bits behind the leading one, 2^-9 below
    2^-6, ties to even)."""
    a, k = x.shape
    nb, kb = -(-a // block), -(-width // 128)
    big = torch.zeros((nb * block, kb * 128), dtype=x.dtype, device=x.device)
    big[:a, :k] = x
    scales = big.abs().reshape(nb, block, kb, 128).transpose(1, 2).flatten(2).max(dim=2).values / E4M3_MAX
    scales = torch.clamp(scales, min=SCALE_MIN)
    v = big / scales.repeat_interleave(block, 0).repeat_interleave(128, 1)
    exponent = torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6)))
    step = torch.exp2(exponent - 3)
    v = torch.round(v / step) * step
    return v[:a, :width].to(torch.float32).to(F8), scales
