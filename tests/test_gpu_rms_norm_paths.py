"""rms_norm by the launches that a call takes: the tensor scale of many workgroups'
rows, sums in place of ragged rows, calls without a stored sum, captured calls."""
import numpy as np
import pytest
import torch

import paper_2609_21849_amd as q
from gpu_util import DEV, host, log
from norm_util import bf16_tensor, check_norm, check_scale, reference, rel_error

pytestmark = pytest.mark.gpu

BF16, FP8, NVFP4 = q.QG_FMT_BF16, q.QG_FMT_FP8_E4M3, q.QG_FMT_NVFP4
EPS = 1e-6


@pytest.mark.parametrize("fmt,rows,cols", [(FP8, 4608, 3072), (FP8, 2500, 2001), (FP8, 2100, 5000), (FP8, 70000, 40),
                                           (NVFP4, 4608, 3072), (NVFP4, 2500, 2000), (FP8, 2100, 20000), (FP8, 2051, 49200)])
def test_scale_of_more_rows_than_workgroups(fmt, rows, cols):
    """The first launch's workgroups take several rows each: the largest |y| in a first, a middle or the last one."""
    log("rms_norm scale %d x %d fmt=%d" % (rows, cols, fmt))
    gen = torch.Generator(device=DEV)
    gen.manual_seed(rows + cols)
    x = torch.randn((rows, cols), generator=gen, device=DEV).bfloat16()
    w = 1.0 + 0.1 * torch.rand(cols, generator=gen, device=DEV)
    for at in (0, 1, rows // 2, 2048, rows - 1):
        a = x.clone()
        a[at] = 0.0
        a[at, (at * 7) % cols] = 1.0  # y = sqrt(cols) w, past every other row's largest
        y = q.rms_norm(a, w, EPS, fmt=fmt)
        _, y64 = reference(a[at:at + 1], w, EPS)
        assert np.abs(y64).max() > 0.99 * (cols / (1 + cols * EPS)) ** 0.5
        check_scale(float(y.tensor_scale), y64, 448.0 if fmt == FP8 else 2688.0, rel_error(cols))
        part = q.rms_norm(a[at:at + 1], w, EPS, fmt=fmt, static_scale=y.tensor_scale)
        assert torch.equal(y.codes[at:at + 1], part.codes)
    want = q.rms_norm(a, w, EPS, fmt=fmt, static_scale=y.tensor_scale)
    assert torch.equal(y.codes, want.codes)


@pytest.mark.parametrize("cols", [7, 17, 1001, 3077, 5003, 20001, 65537])
@pytest.mark.parametrize("fmt", [BF16, FP8])
def test_sum_in_place_of_ragged_rows(cols, fmt):
    """A row's short last unit is loaded from elements that the thread beside it replaces. One, two and three launches."""
    log("rms_norm in place cols=%d fmt=%d" % (cols, fmt))
    rng = np.random.default_rng(cols)
    for rows in (1, 40, 600) if cols < 20000 else (1, 9):
        x, r = bf16_tensor(rng, rows, cols), bf16_tensor(rng, rows, cols, 2.0)
        w = torch.from_numpy((1.0 + 0.2 * rng.standard_normal(cols)).astype(np.float32)).cuda()
        _, y64 = reference(x, w, EPS, r)
        h = (x.float() + r.float()).bfloat16()
        for into_residual in (False, True):
            a, b = x.clone(), r.clone()
            y, got = q.rms_norm(a, w, EPS, residual=b, fmt=fmt, sum_out=b if into_residual else a)
            assert torch.equal(got, h) and torch.equal(a if into_residual else b, x if into_residual else r)
            check_norm(y, y64, fmt)


# one launch; two, the maxima in every workgroup's codes; three; three over rows past the registers
PATHS = [(4, 1024), (200, 2048), (500, 3072), (3, 70000), (300, 1001), (5, 49201)]


@pytest.mark.parametrize("rows,cols", PATHS)
def test_without_a_stored_sum(rows, cols):
    rng = np.random.default_rng(cols)
    x, r = bf16_tensor(rng, rows, cols), bf16_tensor(rng, rows, cols, 2.0)
    w = torch.from_numpy((1.0 + 0.2 * rng.standard_normal(cols)).astype(np.float32)).cuda()
    want, _ = q.rms_norm(x, w, EPS, residual=r, fmt=FP8)
    codes = torch.full((rows + 1, cols), 77, dtype=torch.uint8, device=DEV)
    ts = torch.empty(1, device=DEV)
    q.qg_rms_norm(FP8, x, cols, r, cols, w, q.QG_OUT_F32, EPS, rows, cols, None, 0, codes, cols, None, ts)
    torch.cuda.synchronize()
    assert torch.equal(codes[:rows], want.codes) and torch.equal(ts, want.tensor_scale)
    assert bool((codes[rows] == 77).all())
    _, y64 = reference(x, w, EPS, r)
    check_norm(want, y64, FP8)


@pytest.mark.parametrize("rows,cols", PATHS)
@pytest.mark.parametrize("fmt", [FP8, NVFP4])
def test_captured(rows, cols, fmt):
    if fmt == NVFP4:
        cols = cols // 16 * 16
    rng = np.random.default_rng(cols)
    x, r = bf16_tensor(rng, rows, cols), bf16_tensor(rng, rows, cols, 2.0)
    w = torch.from_numpy((1.0 + 0.2 * rng.standard_normal(cols)).astype(np.float32)).cuda()
    q.rms_norm(x, w, EPS, residual=r, fmt=fmt)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y, h = q.rms_norm(x, w, EPS, residual=r, fmt=fmt)
    for i in range(3):
        x.copy_(bf16_tensor(rng, rows, cols, 1.0 + i))
        g.replay()
        want, want_h = q.rms_norm(x, w, EPS, residual=r, fmt=fmt)
        torch.cuda.synchronize()
        assert torch.equal(y.codes, want.codes) and torch.equal(y.tensor_scale, want.tensor_scale) and torch.equal(h, want_h)
        if fmt == NVFP4:
            assert torch.equal(y.block_scales, want.block_scales)
        assert host(y.codes).any()
