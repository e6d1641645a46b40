"""C-ABI checks of qg_gemm_fused, qg_rms_norm and qg_rms_norm_static, and the
Python helpers' refusals: no GPU (every call fails validation, or has nothing to do)."""
import ctypes
import math

import pytest
import torch

import paper_2609_21849_amd as q

OK, INVALID, UNSUP, SHAPE, SMALL = 0, 1, 2, 3, 4
FP8, NVFP4, BF16, MXFP4, MXFP8 = q.QG_FMT_FP8_E4M3, q.QG_FMT_NVFP4, q.QG_FMT_BF16, q.QG_FMT_MXFP4, q.QG_FMT_MXFP8
P = 0x10000  # a fake, 64 KiB-aligned "device pointer" that validation never dereferences


def test_epilogue_layout():
    E = q.Epilogue
    assert ctypes.sizeof(E) == 40
    assert [getattr(E, n).offset for n in ("act", "gated", "bias", "residual", "ldr", "bias_dtype", "residual_dtype")] == \
        [0, 4, 8, 16, 24, 32, 36]


def _fused(a_fmt=FP8, w_fmt=FP8, abs_=None, ats=P, lda=256, wbytes=1 << 24, m=32, n=64, k=256, y=P, ybs=None, ldy=None,
           out=q.QG_OUT_BF16, ys=None, epi=True, **e):
    e.setdefault("ldr", n)
    return q.qg_gemm_fused(a_fmt, P, abs_, ats, lda, w_fmt, P, wbytes, m, n, k, q.Epilogue(**e) if epi else None, y, ybs,
                           n if ldy is None else ldy, out, ys, stream=0, check=False)


def test_fused_validation():
    assert _fused(epi=False) == INVALID
    assert _fused(act=4) == INVALID and _fused(act=-1) == INVALID
    assert _fused(gated=2) == INVALID
    assert _fused(out=4) == INVALID and _fused(out=-1) == INVALID
    assert _fused(ys=P) == INVALID                                    # a scale without a quantized output
    assert _fused(out=q.QG_OUT_FP8) == INVALID                        # and the other way round
    assert _fused(out=q.QG_OUT_FP8, ys=P + 2) == INVALID
    assert _fused(n=40) == SHAPE
    assert _fused(k=192, lda=256) == SHAPE
    assert _fused(ldy=48) == INVALID
    assert _fused(y=None) == INVALID and _fused(y=P + 1) == INVALID
    assert _fused(out=q.QG_OUT_F32, y=P + 2) == INVALID
    assert _fused(ybs=P) == INVALID                                   # block scales without an NVFP4 output
    assert _fused(a_fmt=FP8, w_fmt=NVFP4) == UNSUP
    assert _fused(ats=None) == INVALID                                # the product's own checks
    assert _fused(lda=128) == INVALID
    assert _fused(wbytes=100) == SMALL
    assert _fused(m=-1) == INVALID and _fused(n=-16) == INVALID and _fused(k=-128) == INVALID


def test_fused_bias_and_residual_validation():
    assert _fused(bias=P + 1) == INVALID
    assert _fused(bias=P + 2, bias_dtype=q.QG_OUT_F32) == INVALID
    assert _fused(bias=P, bias_dtype=2) == INVALID
    assert _fused(residual=P + 1) == INVALID
    assert _fused(residual=P + 2, residual_dtype=q.QG_OUT_F32) == INVALID
    assert _fused(residual=P, residual_dtype=3) == INVALID
    assert _fused(residual=P, ldr=48) == INVALID
    assert _fused(residual=P, gated=1) == INVALID


def test_fused_gated_and_quantized_validation():
    one = q.qg_packed_bytes(FP8, 64, 256)
    assert _fused(wbytes=one, act=9) == INVALID
    assert _fused(gated=1, wbytes=one) == SMALL                       # 2 n weight rows
    assert _fused(gated=1, n=2 ** 30) == INVALID                      # more rows than an int
    nv = dict(out=q.QG_OUT_NVFP4, ys=P)
    assert _fused(**nv) == INVALID                                    # block scales out
    assert _fused(**nv, ybs=P, y=P + 2) == INVALID
    assert _fused(**nv, ybs=P, ldy=72) == INVALID
    assert _fused(**nv, ybs=P, a_fmt=BF16, w_fmt=NVFP4, ats=None) == UNSUP
    assert _fused(m=0) == OK and _fused(n=0) == OK                    # nothing to do
    assert _fused(m=0, gated=1) == OK


def _norm(fmt=FP8, x=P, ldx=64, res=None, ldr=64, w=P, wdt=q.QG_OUT_BF16, eps=1e-6, rows=4, cols=64, sum_=None, lds=64, y=P,
          ldy=64, bs=None, ts=P, static=False):
    f = q.qg_rms_norm_static if static else q.qg_rms_norm
    return f(fmt, x, ldx, res, ldr, w, wdt, eps, rows, cols, sum_, lds, y, ldy, bs, ts, stream=0, check=False)


def test_norm_validation():
    assert _norm(fmt=9) == INVALID
    for fmt in (BF16, MXFP4, MXFP8):
        assert _norm(fmt=fmt, ts=None, bs=P, static=True) == UNSUP
        assert _norm(fmt=fmt, ts=P, bs=None if fmt == BF16 else P) == INVALID   # no tensor scale
    assert _norm(ts=None) == INVALID and _norm(ts=P + 2) == INVALID
    assert _norm(wdt=2) == INVALID
    for eps in (-1e-6, math.inf, math.nan):
        assert _norm(eps=eps) == INVALID
    assert _norm(rows=-1) == INVALID and _norm(cols=-1) == INVALID and _norm(rows=2 ** 31) == INVALID
    assert _norm(fmt=NVFP4, cols=40, bs=P) == SHAPE
    assert _norm(fmt=MXFP8, cols=48, bs=P, ts=None) == SHAPE
    assert _norm(bs=P) == INVALID                                     # FP8 has no block scales
    assert _norm(fmt=NVFP4) == INVALID                                # NVFP4 has
    assert _norm(sum_=P) == INVALID                                   # a sum without a residual
    assert _norm(ldx=32) == INVALID
    assert _norm(res=P, ldr=32) == INVALID
    assert _norm(res=P, sum_=P, lds=32) == INVALID
    assert _norm(fmt=BF16, ts=None, ldy=32) == INVALID
    assert _norm(x=None) == INVALID and _norm(x=P + 1) == INVALID
    assert _norm(res=P + 1) == INVALID and _norm(res=P, sum_=P + 1) == INVALID
    assert _norm(w=None) == INVALID and _norm(w=P + 1) == INVALID and _norm(w=P + 2, wdt=q.QG_OUT_F32) == INVALID
    assert _norm(y=None) == INVALID
    assert _norm(fmt=BF16, ts=None, y=P + 1) == INVALID
    assert _norm(fmt=NVFP4, bs=P, y=P + 4) == INVALID
    assert _norm(fmt=MXFP4, bs=P, ts=None, y=P + 2) == INVALID
    assert _norm(rows=0, static=True) == OK and _norm(fmt=BF16, rows=0, ts=None) == OK   # nothing to do


def test_helpers_refuse_host_tensors():
    x, w = torch.zeros((4, 128), dtype=torch.bfloat16), torch.ones(128, dtype=torch.bfloat16)
    packed = torch.zeros(4096, dtype=torch.uint8)
    for call in (lambda s: q.rms_norm(x, w, stream=s), lambda s: q.linear_fused(x, packed, NVFP4, 16, stream=s),
                 lambda s: q.linear_gated(x, packed, NVFP4, 16, stream=s)):
        for stream in (None, object()):
            with pytest.raises(ValueError, match="CUDA"):
                call(stream)


def test_helpers_without_the_native_extension(monkeypatch):
    import sys
    monkeypatch.setitem(sys.modules, "paper_2609_21849_amd._qgemm_torch", None)
    monkeypatch.delattr(q, "_qgemm_torch", raising=False)
    monkeypatch.setattr(q, "_host", None)
    x = torch.zeros((4, 128), dtype=torch.bfloat16)
    with pytest.warns(RuntimeWarning, match="_qgemm_torch"), pytest.raises(ValueError, match="CUDA"):
        q.rms_norm(x, x[0])
    with pytest.raises(ValueError, match="CUDA"):
        q.linear_fused(x, torch.zeros(4096, dtype=torch.uint8), NVFP4, 16)


def test_interleaved_rows():
    a, b = torch.arange(6).view(3, 2), 10 + torch.arange(6).view(3, 2)
    assert q.interleave_gated(a, b).tolist() == [[0, 1], [10, 11], [2, 3], [12, 13], [4, 5], [14, 15]]
    assert q.interleave_gated(a[:, 0], b[:, 0]).tolist() == [0, 10, 2, 12, 4, 14]
    for bad in (b[:2], b.float()):
        with pytest.raises(ValueError, match="gate and up"):
            q.interleave_gated(a, bad)
