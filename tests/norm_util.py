"""What qg_rms_norm may return, from its formula in 64 bits.

y = fl(fl(h r) w) in fp32. With u = 2^-24 and L at least the longest chain of
fp32 additions behind the sum of squares (16 elements of each of a thread's
units, at most four of them up to 16384 columns and ceil(cols / 16384) past
that, six lane swaps, the waves), all terms positive: the sum is within (L + 1) u of
the exact one relatively, the mean one division, eps one addition, so the root
of it within half of (L + 3) u plus one rounding; the reciprocal and the two
products round once each: |y - y64| <= ((L + 3) / 2 + 4) u |y64|. A quantized
output rounds fl(y r) once more (its scale steps are fp32 as well), and rounding
is monotone, so every code lies between the codes of the two ends."""
import numpy as np
import torch

import oracle
import paper_2609_21849_amd as q
from gpu_util import bf16_rne, check_nvfp4_codes, host, order_key

U = 2.0 ** -24


def rel_error(cols: int) -> float:
    units = -(-cols // 16)
    per_thread = max(4, -(-units // 1024))
    return ((16 * per_thread + 6 + 16 + 3) / 2 + 4) * U


def reference(x, weight, eps, residual=None):
    """(h as a float64 array, y in 64 bits)."""
    h = x.float() if residual is None else (x.float() + residual.float()).bfloat16().float()
    h = host(h).astype(np.float64)
    w = host(weight.float()).astype(np.float64)
    ms = np.mean(h * h, axis=1, keepdims=True) + float(np.float32(eps))
    r = np.where(ms > 0, 1.0 / np.sqrt(np.where(ms > 0, ms, 1.0)), 0.0)
    return h, h * r * w


def _f32_ends(v, rel):
    a, b = v * (1 - rel), v * (1 + rel)
    lo, hi = np.minimum(a, b).astype(np.float32), np.maximum(a, b).astype(np.float32)
    return np.nextafter(lo, np.float32(-np.inf)), np.nextafter(hi, np.float32(np.inf))


def check_scale(got: float, y64, divisor: float, rel: float):
    want = np.max(np.abs(y64)) / divisor
    assert abs(got - want) <= want * (rel + 2 * U), (got, want)


def check_e4m3(codes, y64, r, rel):
    lo, hi = _f32_ends(y64 * r, rel + 2 * U)
    k = order_key(codes)
    klo, khi = order_key(oracle.e4m3_encode_array(lo)), order_key(oracle.e4m3_encode_array(hi))
    bad = int(np.count_nonzero((k < klo) | (k > khi)))
    assert bad == 0, "%d of %d codes" % (bad, k.size)


def _unpack4(codes):
    return np.stack((codes & 15, codes >> 4), axis=2).reshape(codes.shape[0], -1)


def check_mx(codes, scales, y64, fp4, rel):
    rows, cols = y64.shape
    am = np.abs(y64).reshape(rows, -1, 32).max(axis=2)
    emax = 2 if fp4 else 8

    def code(v):
        e = np.where(v > 0, np.frexp(np.where(v > 0, v, 1.0))[1] - 1 - emax + 127, 0)
        return np.clip(e, 0, 254)
    lo, hi = code(am * (1 - rel)), code(am * (1 + rel))
    assert not np.count_nonzero((scales < lo) | (scales > hi))
    f = np.exp2(127.0 - np.repeat(scales.astype(np.float64), 32, axis=1))
    if not fp4:
        return check_e4m3(codes, y64 * f, 1.0, rel)
    a, b = _f32_ends(y64 * f, rel + 2 * U)
    key = lambda c: np.where(c & 8, -(c.astype(np.int32) & 7), c.astype(np.int32) & 7)  # noqa: E731
    k, klo, khi = key(_unpack4(codes)), key(oracle.e2m1_encode_array(a)), key(oracle.e2m1_encode_array(b))
    assert not np.count_nonzero((k < klo) | (k > khi))


def check_norm(y, y64, fmt, static=False):
    """y: what rms_norm returned in format fmt for the 64-bit values y64."""
    rel = rel_error(y64.shape[1])
    if fmt == q.QG_FMT_BF16:
        got = host(y.float()).astype(np.float64)
        lo, hi = bf16_rne(y64 - rel * np.abs(y64)), bf16_rne(y64 + rel * np.abs(y64))
        bad = int(np.count_nonzero((got < lo) | (got > hi)))
        assert bad == 0, "%d of %d values" % (bad, got.size)
        return
    codes = host(y.codes)
    if fmt in (q.QG_FMT_MXFP4, q.QG_FMT_MXFP8):
        check_mx(codes, host(y.block_scales), y64, fmt == q.QG_FMT_MXFP4, rel)
        return
    s = np.float32(host(y.tensor_scale)[0])
    if not static:
        check_scale(float(s), y64, 448.0 if fmt == q.QG_FMT_FP8_E4M3 else 2688.0, rel)
    if fmt == q.QG_FMT_FP8_E4M3:
        r = float(np.float32(1.0) / s) if s > 0 else 0.0
        check_e4m3(codes, y64, r, rel)
    else:
        check_nvfp4_codes(codes, host(y.block_scales), {"y": y64, "b": np.abs(y64)}, s, tol=rel + 2 * U)


def bf16_tensor(rng, rows, cols, sigma=1.0):
    return torch.from_numpy((sigma * rng.standard_normal((rows, cols))).astype(np.float32)).bfloat16().cuda()
