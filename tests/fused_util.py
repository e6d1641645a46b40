"""What a linear with an epilogue may return, from its formula in 64 bits.

The sums z are taken from the plain linear's fp32 output (the same kernels up
to their end, and tested against the oracle on their own); everything behind
them is computed here in 64 bits. With u = 2^-24 and z exact:
  z + bias: the kernel scales the sum and adds in one or two roundings, the
    fp32 output rounded it once: 2 u |z| + u |z + bias|;
  activation: its documented relative error, and at most 1.13 times the error
    of its argument (the largest slope of SiLU and GELU);
  the gate's product: both factors' errors, one rounding;
  residual: one rounding of the sum.
The result is rounded once more, which is monotone: an output lies between the
roundings of the two ends."""
import numpy as np
import torch
from scipy.special import erfc, expit

import oracle
import paper_2609_21849_amd as q
from gpu_util import bf16_rne, check_nvfp4_codes, host, order_key

U = 2.0 ** -24
FMTS = {"fp8": q.QG_FMT_FP8_E4M3, "nvfp4": q.QG_FMT_NVFP4, "mxfp4": q.QG_FMT_MXFP4, "mxfp8": q.QG_FMT_MXFP8,
        "w4a16": q.QG_FMT_NVFP4}
ACTS = (q.QG_ACT_NONE, q.QG_ACT_SILU, q.QG_ACT_GELU_TANH, q.QG_ACT_GELU_ERF)


def pick_rows(m, rng):
    """Up to about 160 rows of m: the first and last 32 (ragged tiles) and others at random."""
    if m <= 160:
        return np.arange(m)
    return np.unique(np.concatenate([np.arange(32), np.arange(m - 32, m), rng.integers(0, m, 96)]))


def take(t, rows):
    """Rows of a tensor or QTensor (None stays)."""
    if t is None:
        return None
    if isinstance(t, q.QTensor):
        return q.QTensor(t.fmt, take(t.codes, rows), take(t.block_scales, rows), t.tensor_scale, len(rows), t.cols)
    return t[torch.from_numpy(np.asarray(rows)).to(t.device)]


def activation(z, act):
    """(value, error bound) in 64 bits."""
    if act == q.QG_ACT_SILU:
        y = z * expit(z)
        return y, np.abs(y) * (6 + 4 * np.abs(z)) * 2 * U + 2.0 ** -100
    if act == q.QG_ACT_GELU_TANH:
        t = 2 * np.sqrt(2 / np.pi) * (z + 0.044715 * z ** 3)
        y = z * expit(t)
        return y, np.abs(y) * (6 + 4 * np.abs(t)) * 2 * U + 2.0 ** -100
    if act == q.QG_ACT_GELU_ERF:
        y = 0.5 * z * erfc(-z / np.sqrt(2))
        return y, np.abs(y) * (20 + 2 * z * z) * 2 * U + 2.0 ** -100
    return z, np.zeros_like(z)


def finished(z, bias=None, act=q.QG_ACT_NONE, residual=None, gated=False, z_err=None):
    """(y, error bound) for sums z [m, n] ([m, 2 n] when gated), each within z_err."""
    f64 = lambda t: host(t.float()).astype(np.float64)  # noqa: E731
    z = f64(z) if isinstance(z, torch.Tensor) else z
    e = (0 if z_err is None else z_err) + 2 * U * np.abs(z)
    if bias is not None:
        z = z + f64(bias)
        e = e + U * np.abs(z)
    g, eg = (z[:, 0::2], e[:, 0::2]) if gated else (z, e)
    y, err = activation(g, act)
    err = err + (1.13 if act else 1.0) * eg
    if gated:
        up, eu = z[:, 1::2], e[:, 1::2]
        err = err * (np.abs(up) + eu) + np.abs(y) * eu
        y = y * up
        err = err + U * np.abs(y)
    if residual is not None:
        y = y + f64(residual)
        err = err + U * (np.abs(y) + err)
    return y, err


def check_finished(y, y64, err, s=None):
    """y: a bf16 or fp32 tensor, or a QTensor of decode scale s."""
    if isinstance(y, q.QTensor) and y.fmt == q.QG_FMT_NVFP4:
        tiny = np.finfo(np.float32).tiny
        return check_nvfp4_codes(host(y.codes), host(y.block_scales), {"y": y64, "b": err + tiny}, s, tol=1.0)
    if isinstance(y, q.QTensor):
        r = float(np.float32(1) / np.float32(s))
        lo, hi = [((y64 + d * err) * r * (1 + d * np.sign(y64) * U)).astype(np.float32) for d in (-1, 1)]
        lo, hi = np.nextafter(lo, np.float32(-np.inf)), np.nextafter(hi, np.float32(np.inf))
        k = order_key(host(y.codes))
        klo, khi = order_key(oracle.e4m3_encode_array(lo)), order_key(oracle.e4m3_encode_array(hi))
        bad = int(np.count_nonzero((k < klo) | (k > khi)))
        assert bad == 0, "%d of %d codes" % (bad, k.size)
        return
    got = host(y.float()).astype(np.float64)
    if y.dtype == torch.bfloat16:
        lo, hi = bf16_rne(y64 - err), bf16_rne(y64 + err)
    else:
        lo, hi = y64 - err - U * (np.abs(y64) + err), y64 + err + U * (np.abs(y64) + err)
    bad = (got < lo) | (got > hi)
    assert not bad.any(), "%d of %d values, first at %s: %r not in [%r, %r]" % (
        np.count_nonzero(bad), bad.size, np.argwhere(bad)[0], got[bad][0], lo[bad][0], hi[bad][0])
