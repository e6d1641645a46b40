"""Sums and outputs past 2^32 bytes: the last rows of a very large call against the
formula and against the same rows in a smaller call."""
import numpy as np
import pytest
import torch

import paper_2609_21849_amd as q
from fused_util import check_finished, finished, take
from gpu_util import DEV, log

pytestmark = pytest.mark.gpu


def test_norm_of_more_than_2_32_elements():
    rows, cols = (1 << 20) + 37, 4096
    log("rms_norm %d x %d" % (rows, cols))
    gen = torch.Generator(device=DEV)
    gen.manual_seed(1)
    x = torch.empty((rows, cols), dtype=torch.bfloat16, device=DEV)
    for part in x.split(1 << 17):
        part.copy_(torch.randn(part.shape, generator=gen, device=DEV))
    w = torch.rand(cols, generator=gen, device=DEV)
    s = torch.full((1,), 0.02, device=DEV)
    y, h = q.rms_norm(x, w, 1e-6, residual=x, fmt=q.QG_FMT_FP8_E4M3, static_scale=s)
    for rows_of in (slice(0, 300), slice(rows // 2, rows // 2 + 300), slice(rows - 300, rows)):
        part = x[rows_of].clone()
        want, want_h = q.rms_norm(part, w, 1e-6, residual=part, fmt=q.QG_FMT_FP8_E4M3, static_scale=s)
        assert torch.equal(y.codes[rows_of], want.codes) and torch.equal(h[rows_of], want_h)
    del y, h
    d = q.rms_norm(x, w, 1e-6, fmt=q.QG_FMT_FP8_E4M3)
    part = q.rms_norm(x[-300:].clone(), w, 1e-6, fmt=q.QG_FMT_FP8_E4M3, static_scale=d.tensor_scale)
    assert torch.equal(d.codes[-300:], part.codes)


@pytest.mark.parametrize("gated", [False, True])
def test_outputs_past_4_gib(gated):
    m, n, k, fmt = 140000, 16384, 128, q.QG_FMT_FP8_E4M3
    log("linear_%s %d x %d x %d" % ("gated" if gated else "fused", m, n, k))
    gen = torch.Generator(device=DEV)
    gen.manual_seed(2)
    a = q.quantize(torch.randn((m, k), generator=gen, device=DEV).bfloat16(), fmt)
    weight = (0.1 * torch.randn((2 * n if gated else n, k), generator=gen, device=DEV)).bfloat16()
    packed = q.pack(q.quantize(weight, fmt))
    rows = np.concatenate([np.arange(8), np.arange(m // 2, m // 2 + 8), np.arange(m - 40, m)])
    sub = take(a, rows)
    z = q.linear(q.QTensor(fmt, sub.codes.contiguous(), None, a.tensor_scale, len(rows), k), packed, fmt,
                 weight.shape[0], out_dtype=q.QG_OUT_F32)
    # (another tiling than the large call's: one 128-wide chunk either way, so the same sums)
    if gated:
        y64, err = finished(z, act=q.QG_ACT_SILU, gated=True)
        y = q.linear_gated(a, packed, fmt, n)
        assert y.numel() * 2 > 1 << 32
        check_finished(take(y, rows), y64, err)
        return
    res = torch.randn((len(rows), n), generator=gen, device=DEV).bfloat16()
    y = torch.zeros((m, n), dtype=torch.bfloat16, device=DEV)
    y[torch.from_numpy(rows).to(DEV)] = res
    y64, err = finished(z, act=q.QG_ACT_GELU_ERF, residual=res)
    q.linear_fused(a, packed, fmt, n, act=q.QG_ACT_GELU_ERF, residual=y, y=y)  # in place
    check_finished(take(y, rows), y64, err)
