"""The operators around the quantized linears, as workloads: their plain forms and the values they must give.

Three operators of ``paper_2609_21849_amd``:

  norm    ``rms_norm``: the residual's addition, the root-mean-square norm and the quantization of its result,
            h = bf16(x + residual),  y_j = h_j / sqrt(mean(h^2) + eps) * weight_j,  y as bf16, FP8 or MXFP8.
  linear  ``linear_fused``: y = act(A W^T + bias) + residual, A and W quantized.
  gated   ``linear_gated``: y = act(A Wg^T) * (A Wu^T), both projections in one product.

Shapes are those of the denoising transformer (hidden 3072, FFN 9216, 4608 tokens for a 1024 x 1024 image) and of
its text encoder (hidden 1024, FFN 3072), and ragged sizes between and below them. Quantized outputs are
``float8`` tensors of the codes' values beside their scales. fp32 outputs are asked for where the matrix
instruction's sums keep fp32 accuracy (16-bit products and MXFP4).
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-6
F8 = torch.float8_e4m3fn
FORMATS = {"fp8": 1, "nvfp4": 2, "mxfp4": 3, "mxfp8": 4, "w4a16": 2}  # w4a16: NVFP4 weights, bf16 activations
ACTS = {"none": 0, "silu": 1, "gelu_tanh": 2, "gelu_erf": 3}
WEIGHT_BITS = {"fp8": 8.0, "nvfp4": 4.5, "w4a16": 4.5, "mxfp4": 4.25, "mxfp8": 8.25}


# ---------------------------------------------------------------- cases
def _norm(out, rows, cols, residual=True):
    return {"op": "norm", "out": out, "rows": rows, "cols": cols, "residual": residual}


def _linear(fmt, m, n, k, act="none", bias=False, residual=False, out="bf16"):
    return {"op": "linear", "fmt": fmt, "m": m, "n": n, "k": k, "act": act, "bias": bias, "residual": residual, "out": out}


def _gated(fmt, m, n, k, act="silu", out="bf16"):
    return {"op": "gated", "fmt": fmt, "m": m, "n": n, "k": k, "act": act, "out": out}


def listed():
    return [
        # one token of the text encoder in front of an FP8 linear, the scale taken from the token
        {"name": "norm_fp8_dynamic_1x1024", **_norm("fp8_dynamic", 1, 1024)},
        # the text encoder's first norm over a prompt of ragged length: nothing to add, bf16 to weight-only linears
        {"name": "norm_bf16_300x1024", **_norm("bf16", 300, 1024, residual=False)},
        # text tokens of the transformer in front of an MXFP8 linear
        {"name": "norm_mxfp8_500x3072", **_norm("mxfp8", 500, 3072)},
        # the transformer at a 1024 x 1024 image, calibrated FP8
        {"name": "norm_fp8_4608x3072", **_norm("fp8", 4608, 3072)},
        # the same with the scale of the whole tensor taken at run time
        {"name": "norm_fp8_dynamic_4608x3072", **_norm("fp8_dynamic", 4608, 3072)},
        # one token of the text encoder through a weight-only projection back to the hidden size, added to its stream
        {"name": "linear_w4a16_1x1024x3072", **_linear("w4a16", 1, 1024, 3072, residual=True)},
        # text tokens through MLP-up with bias and GELU, 4-bit block format
        {"name": "linear_mxfp4_500x9216x3072", **_linear("mxfp4", 500, 9216, 3072, act="gelu_tanh", bias=True)},
        # a ragged, smaller image through MLP-up with bias and GELU, its output the FP8 operand of MLP-down
        {"name": "linear_nvfp4_2800x9216x3072", **_linear("nvfp4", 2800, 9216, 3072, act="gelu_tanh", bias=True, out="fp8")},
        # MLP-down of a 1024 x 1024 image, added to the residual stream
        {"name": "linear_fp8_4608x3072x9216", **_linear("fp8", 4608, 3072, 9216, residual=True)},
        # one token through the text encoder's gated projections, weight-only
        {"name": "gated_w4a16_1x3072x1024", **_gated("w4a16", 1, 3072, 1024)},
        # a ragged batch of text tokens through the transformer's gated projections, MXFP8
        {"name": "gated_mxfp8_500x9216x3072", **_gated("mxfp8", 500, 9216, 3072)},
        # the gated projections of a 1024 x 1024 image, calibrated FP8 in and out: the largest
        {"name": "gated_fp8_4608x9216x3072", **_gated("fp8", 4608, 9216, 3072, out="fp8")},
    ]


def _log(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, int(round(v / step)) * step))


def draw(rng):
    op = rng.choice(["norm", "linear", "gated"])
    if op == "norm":
        out = rng.choice(["bf16", "fp8", "fp8_dynamic", "mxfp8"])
        while True:
            rows, cols = _log(rng, 1, 16384), _log(rng, 32, 16384, 32 if out == "mxfp8" else rng.choice([1, 8, 64]))
            if rows * cols <= 4608 * 9216:
                return _norm(out, rows, cols, residual=rng.random() < 0.75)
    fmt = rng.choice(sorted(FORMATS))
    exact_sums = fmt in ("nvfp4", "w4a16", "mxfp4")
    out = rng.choice(["bf16", "bf16", "fp8", "f32" if exact_sums else "bf16"])
    while True:
        m, n = _log(rng, 1, 4608), _log(rng, 64, 9216, 16)
        k = _log(rng, 256, 9216, 256 if fmt[:2] == "mx" else 128)
        if m * n * k <= 4608 * 9216 * 3072:
            break
    if op == "gated":
        return _gated(fmt, m, n, k, act=rng.choice(["silu", "gelu_tanh", "gelu_erf"]), out=out)
    return _linear(fmt, m, n, k, act=rng.choice(sorted(ACTS)), bias=rng.random() < 0.5, residual=rng.random() < 0.5, out=out)


# ---------------------------------------------------------------- inputs
def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 1000003 + 29)
    return gen


def _normal(gen, *shape, sigma=1.0):
    return (sigma * torch.randn(shape, generator=gen, device="cuda")).bfloat16()


def _to_e2m1(v):
    """Codes 0 to 15 of the nearest of 0, .5, 1, 1.5, 2, 3, 4, 6 and their negatives, ties to the even code."""
    a = v.abs()
    c = (a > 0.25).int() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)
    return (c + 8 * (v < 0)).to(torch.uint8)


def _quantize(x, fmt):
    """What a user has in hand: codes, block scales and tensor scale of a bf16 tensor in the library's formats."""
    v = x.float()
    if fmt in ("mxfp4", "mxfp8"):
        b = v.reshape(v.shape[0], -1, 32)
        e = torch.frexp(b.abs().amax(2, keepdim=True))[1] - 1 - (2 if fmt == "mxfp4" else 8)
        e = e.clamp(-127, 127)
        b = torch.ldexp(b, -e).reshape(v.shape)
        codes = b.clamp(-448, 448).to(F8).view(torch.uint8) if fmt == "mxfp8" else _to_e2m1(b)
        scales, tensor_scale = (e + 127).to(torch.uint8).squeeze(2), None
    elif fmt == "fp8":
        tensor_scale = (v.abs().max() / 448.0).reshape(1)
        codes, scales = (v / tensor_scale).clamp(-448, 448).to(F8).view(torch.uint8), None
    else:
        tensor_scale = (v.abs().max() / 2688.0).reshape(1)
        b = v.reshape(v.shape[0], -1, 16)
        scales = (b.abs().amax(2, keepdim=True) / (6.0 * tensor_scale)).clamp(max=448).to(F8)
        s = scales.float() * tensor_scale
        codes = _to_e2m1((b / torch.where(s > 0, s, 1.0)).reshape(v.shape))
        scales = scales.view(torch.uint8).squeeze(2)
    if fmt in ("mxfp4", "nvfp4"):
        codes = codes[:, 0::2] | (codes[:, 1::2] << 4)
    return {"codes": codes.contiguous(), "scales": None if scales is None else scales.contiguous(), "tensor_scale": tensor_scale}


def _e2m1_values(codes, dtype):
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0],
                        dtype=dtype, device=codes.device)
    return grid[torch.stack((codes & 15, codes >> 4), 2).reshape(codes.shape[0], -1).int()]


def _decode(q, fmt):
    """fp32 values of codes times scales."""
    v = _e2m1_values(q["codes"], torch.float32) if fmt in ("mxfp4", "nvfp4") else q["codes"].view(F8).float()
    if fmt == "nvfp4":
        v = v * q["scales"].view(F8).float().repeat_interleave(16, 1)
    elif fmt != "fp8":
        v = v * torch.ldexp(torch.ones(1, device=v.device), q["scales"].int() - 127).repeat_interleave(32, 1)
    return v if q["tensor_scale"] is None else v * q["tensor_scale"]


def _formats(case):
    """(activation format, weight format); a weight-only linear's activation stays bf16."""
    return (None, "nvfp4") if case["fmt"] == "w4a16" else (case["fmt"], case["fmt"])


def _out_scale(case):
    """A calibrated decode scale of an FP8 output: its largest value to be, by the products' spread."""
    sigma = 0.02 * math.sqrt(case["k"])
    amax = 5.0 * sigma if case["op"] == "linear" else 8.0 * sigma * sigma
    return torch.tensor([max(amax, 1.0) / 448.0], dtype=torch.float32, device="cuda")


def _inputs(case, seed):
    gen = _generator(seed)
    if case["op"] == "norm":
        rows, cols = case["rows"], case["cols"]
        s = {"x": _normal(gen, rows, cols), "weight": (1.0 + 0.1 * torch.randn(cols, generator=gen, device="cuda")).bfloat16()}
        if case["residual"]:
            s["residual"] = _normal(gen, rows, cols, sigma=3.0)
            # a few channels of the stream carry outliers, the same ones in every row
            s["residual"][:, torch.randperm(cols, generator=gen, device="cuda")[:max(1, cols // 1000)]] *= 10.0
        s["static_scale"] = torch.tensor([8.0 / 448.0], dtype=torch.float32, device="cuda") if case["out"] == "fp8" else None
        return s
    m, n, k = case["m"], case["n"], case["k"]
    a_fmt, w_fmt = _formats(case)
    x = _normal(gen, m, k)
    s = {"a": _quantize(x, a_fmt) if a_fmt else x}
    # gated: rows 2 i and 2 i + 1 are the gate and up rows of output i
    s["w"] = _quantize(_normal(gen, 2 * n if case["op"] == "gated" else n, k, sigma=0.02), w_fmt)
    s["bias"] = _normal(gen, n, sigma=0.5) if case.get("bias") else None
    s["residual"] = _normal(gen, m, n, sigma=3.0) if case.get("residual") else None
    s["y_scale"] = _out_scale(case) if case["out"] == "fp8" else None
    return s


def prepare(case, seed):
    """Inputs, and the weight as its program keeps it: packed for the library, or decoded to fp32."""
    s = {"case": case, **_inputs(case, seed)}
    if case["op"] == "norm":
        return s
    a_fmt, w_fmt = _formats(case)
    w = s.pop("w")
    rows = w["codes"].shape[0]
    if own:
        import paper_2609_21849_amd as q
        s["w"] = q.pack(q.QTensor(FORMATS[w_fmt], w["codes"], w["scales"], w["tensor_scale"], rows, case["k"]))
        if a_fmt:
            a = s["a"]
            s["a"] = q.QTensor(FORMATS[a_fmt], a["codes"], a["scales"], a["tensor_scale"], case["m"], case["k"])
    else:
        s["w"] = _decode(w, w_fmt)
    return s


# ---------------------------------------------------------------- one pass
def _fp8(y, scale):
    return (y / scale).clamp(-448.0, 448.0).to(F8)


def _act(z, act):
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    if act == "gelu_erf":
        return 0.5 * z * torch.erfc(z * -math.sqrt(0.5))
    return z


def _plain_norm(s):
    case, h = s["case"], s["x"]
    out = {}
    if case["residual"]:
        h = out["h"] = (h.float() + s["residual"].float()).bfloat16()
    v = h.float()
    y = v * torch.rsqrt((v * v).mean(1, keepdim=True) + EPS) * s["weight"].float()
    if case["out"] == "bf16":
        out["y"] = y.bfloat16()
    elif case["out"] == "mxfp8":
        b = y.reshape(y.shape[0], -1, 32)
        e = (torch.frexp(b.abs().amax(2, keepdim=True))[1] - 9).clamp(-127, 127)
        out["codes"] = torch.ldexp(b, -e).clamp(-448.0, 448.0).to(F8).reshape(y.shape)
        out["scales"] = (e + 127).to(torch.uint8).squeeze(2).view(torch.float8_e8m0fnu)
    else:
        scale = s["static_scale"] if case["out"] == "fp8" else (y.abs().max() / 448.0).reshape(1)
        out["codes"] = _fp8(y, scale)
        if case["out"] == "fp8_dynamic":
            out["scale"] = scale
    return out


def _plain_linear(s):
    case = s["case"]
    a = s["a"].float() if case["fmt"] == "w4a16" else _decode(s["a"], case["fmt"])
    z = a @ s["w"].t()
    if case["op"] == "gated":
        y = _act(z[:, 0::2], case["act"]) * z[:, 1::2]
    else:
        y = _act(z if s["bias"] is None else z + s["bias"].float(), case["act"])
        if s["residual"] is not None:
            y = y + s["residual"].float()
    if case["out"] == "fp8":
        return {"codes": _fp8(y, s["y_scale"])}
    return {"y": y if case["out"] == "f32" else y.bfloat16()}


def _own_norm(s):
    import paper_2609_21849_amd as q
    case = s["case"]
    fmt = {"bf16": q.QG_FMT_BF16, "mxfp8": q.QG_FMT_MXFP8}.get(case["out"], q.QG_FMT_FP8_E4M3)
    out = {}
    if case["residual"]:
        y, out["h"] = q.rms_norm(s["x"], s["weight"], EPS, residual=s["residual"], fmt=fmt, static_scale=s["static_scale"])
    else:
        y = q.rms_norm(s["x"], s["weight"], EPS, fmt=fmt, static_scale=s["static_scale"])
    if case["out"] == "bf16":
        out["y"] = y
        return out
    out["codes"] = y.codes.view(F8)
    if case["out"] == "mxfp8":
        out["scales"] = y.block_scales.view(torch.float8_e8m0fnu)
    elif case["out"] == "fp8_dynamic":
        out["scale"] = y.tensor_scale
    return out


def _own_linear(s):
    import paper_2609_21849_amd as q
    case = s["case"]
    fmt = FORMATS[_formats(case)[1]]
    out = {"bf16": q.QG_OUT_BF16, "f32": q.QG_OUT_F32, "fp8": q.QG_OUT_FP8}[case["out"]]
    if case["op"] == "gated":
        y = q.linear_gated(s["a"], s["w"], fmt, case["n"], act=ACTS[case["act"]], out_dtype=out, y_scale=s["y_scale"])
    else:
        y = q.linear_fused(s["a"], s["w"], fmt, case["n"], bias=s["bias"], act=ACTS[case["act"]], residual=s["residual"],
                           out_dtype=out, y_scale=s["y_scale"])
    return {"codes": y.codes.view(F8)} if case["out"] == "fp8" else {"y": y}


def run(state):
    if state["case"]["op"] == "norm":
        return _own_norm(state) if own else _plain_norm(state)
    return _own_linear(state) if own else _plain_linear(state)


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    if case["op"] == "norm":
        rows, cols = case["rows"], case["cols"]
        each = 2 + (4 if case["residual"] else 0)  # x; residual and its sum
        each += {"bf16": 2, "mxfp8": 1 + 1 / 32}.get(case["out"], 1)
        return {"bytes": rows * cols * each + 2 * cols, "flops": 6.0 * rows * cols}
    m, n, k = case["m"], case["n"], case["k"]
    rows = 2 * n if case["op"] == "gated" else n
    a_bits = 16.0 if case["fmt"] == "w4a16" else WEIGHT_BITS[case["fmt"]]
    out = m * n * {"bf16": 2, "f32": 4, "fp8": 1}[case["out"]]
    extra = (2 * n if case.get("bias") else 0) + (2 * m * n if case.get("residual") else 0)
    return {"bytes": m * k * a_bits / 8 + rows * k * WEIGHT_BITS[case["fmt"]] / 8 + out + extra, "flops": 2.0 * m * rows * k}


# ---------------------------------------------------------------- the same in 64 bits
def _values64(q, fmt):
    c = q["codes"]
    if fmt in ("fp8", "mxfp8"):
        v = c.view(F8).double()
    else:
        mag = torch.tensor([0, 1, 2, 3, 4, 6, 8, 12], dtype=torch.float64, device=c.device) / 2
        pairs = torch.stack((c % 16, c // 16), -1).flatten(1).long()
        v = torch.where(pairs >= 8, -mag[pairs % 8], mag[pairs % 8])
    if fmt == "fp8":
        return v * q["tensor_scale"].double()
    block = 16 if fmt == "nvfp4" else 32
    s = q["scales"].view(F8).double() if fmt == "nvfp4" else torch.exp2(q["scales"].double() - 127)
    v = (v.reshape(v.shape[0], -1, block) * s.unsqueeze(2)).reshape(v.shape)
    return v * q["tensor_scale"].double() if fmt == "nvfp4" else v


def _act64(z, act):
    if act == "silu":
        return z * torch.special.expit(z)
    if act == "gelu_tanh":
        return z * torch.special.expit(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))
    if act == "gelu_erf":
        return z * torch.special.ndtr(z)
    return z


def _exact_norm(case, s):
    h = s["x"].double()
    out = {}
    if case["residual"]:
        out["h"] = h + s["residual"].double()
        h = out["h"].bfloat16().double()  # the operator is defined on the stored sum
    y = h * s["weight"].double() / (h.square().sum(1, keepdim=True) / case["cols"] + EPS).sqrt()
    if case["out"] == "bf16":
        out["y"] = y
    elif case["out"] == "mxfp8":  # code values before their rounding
        b = y.unflatten(1, (-1, 32))
        e = torch.floor(torch.log2(b.abs().amax(2, keepdim=True))) - 8
        out["codes"], out["scales"] = (b * torch.exp2(-e)).flatten(1).clamp(-448, 448), torch.exp2(e).squeeze(2)
    else:
        scale = s["static_scale"].double() if case["out"] == "fp8" else y.abs().max().reshape(1) / 448
        out["codes"] = (y / scale).clamp(-448, 448)
        if case["out"] == "fp8_dynamic":
            out["scale"] = scale
    return out


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "norm":
        return _exact_norm(case, s)
    a_fmt, w_fmt = _formats(case)
    z = (_values64(s["a"], a_fmt) if a_fmt else s["a"].double()) @ _values64(s["w"], w_fmt).t()
    if case["op"] == "gated":
        y = _act64(z[:, ::2], case["act"]) * z[:, 1::2]
    else:
        y = _act64(z + (0 if s["bias"] is None else s["bias"].double()), case["act"])
        y = y + (0 if s["residual"] is None else s["residual"].double())
    return {"codes": (y / s["y_scale"].double()).clamp(-448, 448)} if case["out"] == "fp8" else {"y": y}
