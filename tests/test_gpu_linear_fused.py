"""linear_fused and linear_gated against their formulas in 64 bits: every operand
pair and kernel, activation, output type, bias and residual of both types; few
and many tokens, ragged tiles, pitched and unaligned outputs and residuals,
in place; what lies outside the output stays."""
import numpy as np
import pytest
import torch

import oracle
import paper_2609_21849_amd as q
import synth
from fused_util import ACTS, FMTS, check_finished, finished, pick_rows, take
from gpu_util import DEV, log, to_dev_bf16

pytestmark = pytest.mark.gpu

BF16, F32, FP8, NVFP4 = q.QG_OUT_BF16, q.QG_OUT_F32, q.QG_OUT_FP8, q.QG_OUT_NVFP4
KINDS = ["fp8", "nvfp4", "mxfp4", "mxfp8", "w4a16"]


def _operands(kind, m, rows, k, seed=1):
    fmt = FMTS[kind]
    x = synth.normal_bf16(m, k, 1.0, seed, 0)
    w = synth.normal_bf16(rows, k, 0.05, seed, 1)
    packed = q.pack(q.quantize(to_dev_bf16(w), fmt))
    xd = to_dev_bf16(x)
    return (xd if kind == "w4a16" else q.quantize(xd, fmt)), packed, fmt, x, w


def _vec(rng, n, dtype=torch.float32, sigma=0.5):
    return torch.from_numpy((sigma * rng.standard_normal(n)).astype(np.float32)).to(dtype).to(DEV)


def _scale(y64, out):
    """A decode scale with the largest outputs a little past its range."""
    return np.float32(0.9 * max(np.abs(y64).max(), 1e-6) / (448.0 if out == FP8 else 2688.0))


def _call(a, packed, fmt, n, gated, out, y64, **kw):
    s = _scale(y64, out) if out in (FP8, NVFP4) else None
    if s is not None:
        kw["y_scale"] = torch.full((1,), float(s), device=DEV)
    y = (q.linear_gated if gated else q.linear_fused)(a, packed, fmt, n, out_dtype=out, **kw)
    torch.cuda.synchronize()
    return y, s


def _outs(kind):
    return (BF16, F32, FP8) if kind == "w4a16" else (BF16, F32, FP8, NVFP4)


# few tokens (every split-K tiling of 256 CUs), 64 x 128 and large tiles of each height, 288 x 192 tiles, the kernels of a
# wide weight pool; last tiles ragged in both directions
FEW = [(1, 1024, 512), (5, 96, 1024), (33, 2048, 512), (100, 1040, 768), (200, 2912, 768), (300, 992, 1536),
       (500, 3040, 2304), (1030, 528, 4352)]
LARGE = {"fp8": [(700, 1056, 1152), (2380, 1584, 1536), (1900, 4128, 256), (2200, 4128, 256), (4600, 3040, 128), (4000, 4128, 128)],
         "nvfp4": [(150, 21568, 256), (1900, 4128, 256), (2300, 4128, 256), (4000, 4128, 128)],
         "mxfp4": [(1900, 4128, 256), (2300, 4128, 256), (4000, 4128, 256), (700, 4096, 512)],
         "mxfp8": [(1900, 4128, 256), (2300, 4128, 256), (4000, 4128, 256), (406, 6016, 6400)],
         "w4a16": [(1, 65568, 256), (3, 65568, 256), (13, 65568, 384), (1900, 4128, 256), (2300, 4128, 256), (4000, 4128, 128),
                   (700, 2112, 896), (17, 9216, 3328)]}


@pytest.mark.parametrize("kind,m,n,k", [(kind, *s) for kind in KINDS for s in FEW + LARGE[kind]])
def test_shapes(kind, m, n, k):
    log("linear_fused %s %d x %d x %d" % (kind, m, n, k))
    rng = np.random.default_rng(m + n + k)
    a, packed, fmt, _, _ = _operands(kind, m, n, k)
    rows = pick_rows(m, rng)
    z = take(q.linear(a, packed, fmt, n, out_dtype=F32), rows)
    for i, out in enumerate(_outs(kind)):
        bias, act = _vec(rng, n, torch.bfloat16 if i % 2 else torch.float32), ACTS[(i + 1 + m) % 4]
        res = _vec(rng, m * n, torch.float32 if i % 2 else torch.bfloat16, 2.0).view(m, n)
        # (FP8 outputs of a wide pool take another kernel than its fp32 sums: the product's contract)
        other = kind == "w4a16" and n > 60000 and out == FP8
        y64, err = finished(z, bias, act, take(res, rows), z_err=1e-3 * _abs_sum(a, packed, fmt, n) if other else None)
        y, s = _call(a, packed, fmt, n, False, out, y64, bias=bias, act=act, residual=res)
        check_finished(take(y, rows), y64, err, s)


@pytest.mark.parametrize("kind,m,n,k", [(kind, *s) for kind in KINDS for s in FEW + LARGE[kind]])
def test_gated_shapes(kind, m, n, k):
    log("linear_gated %s %d x %d x %d" % (kind, m, n // 2, k))
    rng = np.random.default_rng(m + n + k)
    n = n // 32 * 16
    a, packed, fmt, _, _ = _operands(kind, m, 2 * n, k)
    rows = pick_rows(m, rng)
    z = take(q.linear(a, packed, fmt, 2 * n, out_dtype=F32), rows)
    for i, out in enumerate(_outs(kind)):
        bias = None if i == 2 else _vec(rng, 2 * n, torch.bfloat16 if i % 2 else torch.float32)
        act = ACTS[(i + 1 + m) % 4]
        other = kind == "w4a16" and n > 30000 and out == FP8
        y64, err = finished(z, bias, act, gated=True, z_err=1e-3 * _abs_sum(a, packed, fmt, 2 * n) if other else None)
        y, s = _call(a, packed, fmt, n, True, out, y64, bias=bias, act=act)
        check_finished(take(y, rows), y64, err, s)


def _abs_sum(a, packed, fmt, rows):
    """sum_k |a w| of a weight-only product."""
    w = q.dequantize(q.unpack(packed, fmt, rows, a.shape[1])).double().abs()
    return (a.double().abs() @ w.t()).cpu().numpy()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("gated", [False, True])
def test_against_the_exact_product(kind, gated):
    """The whole operator from the oracle's exact product, within the product's contract."""
    m, n, k = 70, 192, 512
    a, packed, fmt, x, w = _operands(kind, m, n, k, seed=3)
    ref = oracle.linear_reference(kind, x, w)
    rng = np.random.default_rng(3)
    bias = _vec(rng, n)
    res = None if gated else _vec(rng, m * n, torch.bfloat16).view(m, n)
    for act in ACTS:
        y64, err = finished(ref["y"], bias, act, res, gated, z_err=1e-3 * ref["b"])
        for out in _outs(kind):
            kw = {} if gated else {"residual": res}
            y, s = _call(a, packed, fmt, n // 2 if gated else n, gated, out, y64, bias=bias, act=act, **kw)
            check_finished(y, y64, err, s)


@pytest.mark.parametrize("kind,m,n,k", [("fp8", 40, 1040, 512), ("fp8", 700, 1056, 1152), ("fp8", 1900, 4128, 256),
                                        ("fp8", 4600, 3040, 128), ("nvfp4", 40, 1040, 512), ("nvfp4", 1900, 4128, 256),
                                        ("mxfp4", 1900, 4128, 256), ("mxfp8", 1900, 4128, 256), ("w4a16", 1, 65568, 256),
                                        ("w4a16", 9, 65568, 256), ("w4a16", 40, 1040, 512), ("w4a16", 1900, 4128, 256)])
def test_pitches_alignments_and_in_place(kind, m, n, k):
    log("epilogue memory %s %d x %d x %d" % (kind, m, n, k))
    rng = np.random.default_rng(n)
    a, packed, fmt, _, _ = _operands(kind, m, n, k)
    for dt, out in ((torch.bfloat16, BF16), (torch.float32, F32)):
        bias = _vec(rng, n + 1, dt)
        res = _vec(rng, m * n, dt, 2.0).view(m, n)
        want = q.linear_fused(a, packed, fmt, n, bias=bias[1:].clone(), act=q.QG_ACT_SILU, residual=res, out_dtype=out)
        for pitch, shift in ((n + 8, 0), (n + 4, 4), (n + 3, 1)):
            rbuf = torch.full((m, pitch + 8), 3.0, dtype=dt, device=DEV)
            rbuf[:, shift:shift + n] = res
            y = torch.full((m + 1, pitch + 8), 77.0, dtype=dt, device=DEV)
            view = y[:m, shift:shift + n]
            got = q.linear_fused(a, packed, fmt, n, bias=bias[1:], act=q.QG_ACT_SILU, residual=rbuf[:, shift:shift + n],
                                 out_dtype=out, y=view)
            assert got is view and torch.equal(view, want)
            assert bool((y[m] == 77).all()) and bool((y[:, :shift] == 77).all()) and bool((y[:m, shift + n:] == 77).all())
            view.copy_(res)  # the residual stream updated in place
            q.linear_fused(a, packed, fmt, n, bias=bias[1:], act=q.QG_ACT_SILU, residual=view, out_dtype=out, y=view)
            assert torch.equal(view, want)
            assert bool((y[m] == 77).all()) and bool((y[:, :shift] == 77).all()) and bool((y[:m, shift + n:] == 77).all())
        half = n // 2
        if n % 32 == 0:
            gated = q.linear_gated(a, packed, fmt, half, out_dtype=out)
            for pitch, shift in ((half + 8, 0), (half + 5, 1)):
                y = torch.full((m + 1, pitch + 8), 77.0, dtype=dt, device=DEV)
                q.linear_gated(a, packed, fmt, half, out_dtype=out, y=y[:m, shift:shift + half])
                assert torch.equal(y[:m, shift:shift + half], gated)
                assert bool((y[m] == 77).all()) and bool((y[:, :shift] == 77).all()) and bool((y[:m, shift + half:] == 77).all())


@pytest.mark.parametrize("kind,m,n,k", [("fp8", 40, 1056, 512), ("fp8", 700, 1056, 1152), ("fp8", 1900, 4128, 256),
                                        ("fp8", 4600, 3040, 128), ("nvfp4", 1900, 4128, 256), ("mxfp4", 40, 1056, 512),
                                        ("mxfp8", 1900, 4128, 256)])
@pytest.mark.parametrize("gated", [False, True])
def test_pitched_codes(kind, m, n, k, gated):
    """FP8 and NVFP4 codes into rows of a wider buffer, of any alignment the ABI takes."""
    a, packed, fmt, _, _ = _operands(kind, m, n, k)
    cols = n // 2 if gated else n
    e = q.Epilogue(act=q.QG_ACT_SILU, gated=int(gated))
    args = (a.fmt, a.codes, a.block_scales, a.tensor_scale, k, fmt, packed, packed.numel(), m, cols, k, e)
    s = torch.full((1,), 0.01, device=DEV)
    run = q.linear_gated if gated else q.linear_fused
    want = run(a, packed, fmt, cols, act=q.QG_ACT_SILU, out_dtype=FP8, y_scale=s)
    for pitch in (cols + 16, cols + 4, cols + 1):
        buf = torch.full((m + 1, pitch), 77, dtype=torch.uint8, device=DEV)
        q.qg_gemm_fused(*args, buf, None, pitch, FP8, s)
        torch.cuda.synchronize()
        assert torch.equal(buf[:m, :cols], want.codes)
        assert bool((buf[m] == 77).all()) and bool((buf[:, cols:] == 77).all())
    want = run(a, packed, fmt, cols, act=q.QG_ACT_SILU, out_dtype=NVFP4, y_scale=s)
    for pitch in (cols + 16, -(-cols // 128) * 128 + 128):
        cb = torch.full((m + 1, pitch // 2), 77, dtype=torch.uint8, device=DEV)
        sb = torch.full((m + 1, pitch // 16), 77, dtype=torch.uint8, device=DEV)
        q.qg_gemm_fused(*args, cb, sb, pitch, NVFP4, s)
        torch.cuda.synchronize()
        assert torch.equal(cb[:m, :cols // 2], want.codes) and torch.equal(sb[:m, :cols // 16], want.block_scales)
        assert bool((cb[m] == 77).all()) and bool((cb[:, cols // 2:] == 77).all())
        assert bool((sb[m] == 77).all()) and bool((sb[:, cols // 16:] == 77).all())


@pytest.mark.parametrize("act", ACTS)
def test_activations_of_far_arguments(act):
    """Sums from 2^-60 to 2^60 of both signs: no NaN where the formula has none."""
    m, n, k = 32, 64, 128
    fmt = q.QG_FMT_FP8_E4M3
    a, packed, _, _, _ = _operands("fp8", m, n, k)
    a.codes.zero_()
    v = torch.cat([s * torch.logspace(-60, 60, n // 2, base=2.0) for s in (1.0, -1.0)]).to(DEV)
    y = q.linear_fused(a, packed, fmt, n, bias=v, act=act, out_dtype=F32)
    y64, err = finished(torch.zeros((m, n)), v, act)
    check_finished(y, y64, err)
    for fill in (float("inf"), 3.0e38, -3.0e38):
        y = q.linear_fused(a, packed, fmt, n, bias=torch.full((n,), fill, device=DEV), act=act, out_dtype=F32)
        assert not bool(y.isnan().any())


@pytest.mark.parametrize("gated", [False, True])
def test_no_reduction(gated):
    """k = 0: act(bias) and the residual remain."""
    m, n = 37, 48
    rows = 2 * n if gated else n
    rng = np.random.default_rng(2)
    bias = _vec(rng, rows)
    res = None if gated else _vec(rng, m * n).view(m, n)
    fmt = q.QG_FMT_FP8_E4M3
    packed = torch.zeros(256, dtype=torch.uint8, device=DEV)
    e = q.Epilogue(act=q.QG_ACT_GELU_TANH, gated=int(gated), bias=bias.data_ptr(), bias_dtype=F32, ldr=n, residual_dtype=F32,
                   residual=0 if gated else res.data_ptr())
    y64, err = finished(torch.zeros((m, rows)), bias, q.QG_ACT_GELU_TANH, res, gated)
    one = torch.ones(1, device=DEV)
    for out, dt in ((BF16, torch.bfloat16), (F32, torch.float32)):
        y = torch.full((m + 1, n + 3), 77.0, dtype=dt, device=DEV)
        q.qg_gemm_fused(fmt, one, None, one, 0, fmt, packed, 256, m, n, 0, e, y, None, n + 3, out)
        torch.cuda.synchronize()
        check_finished(y[:m, :n], y64, err)
        assert bool((y[m] == 77).all()) and bool((y[:, n:] == 77).all())
    s = torch.full((1,), 0.005, device=DEV)
    codes, bs = torch.empty((m, n // 2), dtype=torch.uint8, device=DEV), torch.empty((m, n // 16), dtype=torch.uint8, device=DEV)
    q.qg_gemm_fused(fmt, one, None, one, 0, fmt, packed, 256, m, n, 0, e, codes, bs, n, NVFP4, s)
    torch.cuda.synchronize()
    check_finished(q.QTensor(q.QG_FMT_NVFP4, codes, bs, s, m, n), y64, err, np.float32(0.005))
    codes = torch.empty((m, n), dtype=torch.uint8, device=DEV)
    q.qg_gemm_fused(fmt, one, None, one, 0, fmt, packed, 256, m, n, 0, e, codes, None, n, FP8, s)
    torch.cuda.synchronize()
    check_finished(q.QTensor(fmt, codes, None, s, m, n), y64, err, np.float32(0.005))


def test_nothing_to_do():
    a, packed, fmt, _, _ = _operands("fp8", 4, 32, 256)
    empty = q.QTensor(fmt, a.codes[:0], None, a.tensor_scale, 0, 256)
    assert q.linear_fused(empty, packed, fmt, 32, act=q.QG_ACT_SILU).shape == (0, 32)
    assert q.linear_gated(empty, packed, fmt, 16).shape == (0, 16)


def test_refusals():
    a, packed, fmt, _, _ = _operands("fp8", 4, 32, 256)
    s = torch.ones(1, device=DEV)
    vec = torch.zeros(32, device=DEV)
    bad = [dict(bias=vec[:16]), dict(bias=vec.half()), dict(bias=vec.cpu()), dict(residual=torch.zeros((4, 16), device=DEV)),
           dict(residual=torch.zeros((32, 4), device=DEV).t()), dict(y_scale=s), dict(out_dtype=q.QG_OUT_FP8), dict(out_dtype=7),
           dict(out_dtype=q.QG_OUT_FP8, y_scale=s.double()), dict(out_dtype=q.QG_OUT_F32, y=torch.empty((4, 32), device=DEV).bfloat16()),
           dict(out_dtype=q.QG_OUT_FP8, y_scale=s, y=torch.empty((4, 32), dtype=torch.uint8, device=DEV))]
    for kw in bad:
        with pytest.raises(ValueError):
            q.linear_fused(a, packed, fmt, 32, **kw)
    with pytest.raises(ValueError, match="shape"):
        q.linear_gated(a, packed, fmt, 16, bias=vec[:16])
    for call in (lambda: q.linear_fused(a, packed, fmt, 32, act=4), lambda: q.linear_fused(a, packed, fmt, 24),
                 lambda: q.linear_gated(a, packed, fmt, 32), lambda: q.linear_fused(a, packed, q.QG_FMT_NVFP4, 32)):
        with pytest.raises(q.QGError):
            call()
    x, w = torch.zeros((4, 256), dtype=torch.bfloat16, device=DEV), torch.ones(256, device=DEV)
    for kw in (dict(weight=w[:128]), dict(weight=w.half()), dict(residual=x[:, :128]), dict(residual=x.float()), dict(sum_out=x),
               dict(residual=x, sum_out=x[:2]), dict(fmt=FMTS["fp8"], static_scale=s.double()), dict(x=x.float()), dict(x=x[0])):
        with pytest.raises(ValueError):
            q.rms_norm(**{"x": x, "weight": w, **kw})
    for kw in (dict(eps=-1.0), dict(eps=float("nan")), dict(fmt=9), dict(fmt=FMTS["mxfp8"], static_scale=s),
               dict(x=x[:, :100], weight=w[:100], fmt=FMTS["mxfp4"])):
        with pytest.raises(q.QGError):
            q.rms_norm(**{"x": x, "weight": w, **kw})


class _Off:
    """A native module that never takes a call."""
    quantize = linear = linear_fp8 = linear_fused = rms_norm = staticmethod(lambda *a: None)


def test_native_and_python_calls_agree(monkeypatch):
    rng = np.random.default_rng(4)
    n, k = 64, 256
    side = torch.cuda.Stream()
    s = torch.full((1,), 0.01, device=DEV)

    def flat(v):
        if isinstance(v, q.QTensor):
            return [v.fmt, v.rows, v.cols, v.codes, v.block_scales, v.tensor_scale]
        return [u for t in v for u in flat(t)] if isinstance(v, tuple) else [v]

    def both(fn):
        native = flat(fn())
        with monkeypatch.context() as mp:
            mp.setattr(q, "_host", _Off)
            python = flat(fn())
        torch.cuda.synchronize()
        assert len(native) == len(python)
        for u, v in zip(native, python):
            assert (torch.equal(u, v) and u.dtype == v.dtype and u.stride() == v.stride()) if torch.is_tensor(u) else u == v

    for kind in KINDS:
        for m in (1, 9):
            a, packed, fmt, _, _ = _operands(kind, m, n, k)
            bias, res = _vec(rng, n), _vec(rng, m * n, torch.bfloat16).view(m, n)
            for out in _outs(kind):
                ys = s if out in (FP8, NVFP4) else None
                side.wait_stream(torch.cuda.current_stream())
                for stream in (None, side, side.cuda_stream):
                    both(lambda: q.linear_fused(a, packed, fmt, n, bias=bias, act=2, residual=res, out_dtype=out, y_scale=ys,
                                                stream=stream))
                    both(lambda: q.linear_gated(a, packed, fmt, n // 2, bias=bias, out_dtype=out, y_scale=ys, stream=stream))
    x, w = _vec(rng, 9 * k, torch.bfloat16).view(9, k), _vec(rng, k)
    for fmt in range(5):
        for static in (None, s) if fmt in (1, 2) else (None,):
            for rows in (1, 9):
                both(lambda: q.rms_norm(x[:rows], w, fmt=fmt, static_scale=static))
                both(lambda: q.rms_norm(x[:rows], w, 1e-5, residual=x[:rows], fmt=fmt, static_scale=static))
