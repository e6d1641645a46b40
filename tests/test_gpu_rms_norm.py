"""rms_norm (residual addition, root-mean-square norm, quantization) against its
formula in 64 bits: every format, lengths of one to many tokens, odd row
lengths, strides, alignments, rows where the squares leave fp32, empty rows."""
import numpy as np
import pytest
import torch

import paper_2609_21849_amd as q
from gpu_util import DEV, host, log
from norm_util import bf16_tensor, check_norm, reference

pytestmark = pytest.mark.gpu

BF16, FP8, NVFP4, MXFP4, MXFP8 = (q.QG_FMT_BF16, q.QG_FMT_FP8_E4M3, q.QG_FMT_NVFP4, q.QG_FMT_MXFP4, q.QG_FMT_MXFP8)
EPS = 1e-6
STATIC = {FP8: 8.0 / 448, NVFP4: 8.0 / 2688}


def _weight(rng, cols, dtype=torch.bfloat16):
    return torch.from_numpy((1.0 + 0.2 * rng.standard_normal(cols)).astype(np.float32)).to(dtype).cuda()


def _run(x, w, residual, fmt, static, eps=EPS, **kw):
    scale = torch.full((1,), STATIC[fmt], device=DEV) if static else None
    out = q.rms_norm(x, w, eps, residual=residual, fmt=fmt, static_scale=scale, **kw)
    torch.cuda.synchronize()
    return out if residual is not None else (out, None)


def _check(x, w, residual, fmt, static=False, eps=EPS, **kw):
    want_h = None if residual is None else (x.float() + residual.float()).bfloat16()
    _, y64 = reference(x, w, eps, residual)
    y, h = _run(x, w, residual, fmt, static, eps, **kw)
    if want_h is not None:
        assert torch.equal(h, want_h)
    check_norm(y, y64, fmt, static)
    return y, h


# one wave a row (1 to 4 units a lane), a workgroup a row (256 and 1024 threads), rows past the registers; one token,
# a few (one launch with the tensor's scale), many; row ends inside a unit
SHAPES = [(1, 32), (1, 1024), (16, 1024), (17, 1024), (3, 2080), (300, 1024), (9, 3072), (5, 4096), (1, 4128), (4, 5120),
          (37, 9216), (1, 16384), (2, 16416), (3, 65536), (2, 65568), (1, 131104),
          # several rows a wave (one launch, maxima in every workgroup's codes, three launches); a thread's units by the
          # number of rows; the longest rows in registers
          (100, 128), (1000, 128), (9000, 96), (70, 224), (300, 512), (129, 480), (2100, 480), (257, 6144), (256, 6144),
          (300, 1600), (60, 20000), (3, 49152), (2, 49184)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("fmt,static", [(BF16, False), (FP8, False), (FP8, True), (NVFP4, False), (NVFP4, True),
                                        (MXFP4, False), (MXFP8, False)])
def test_shapes(rows, cols, fmt, static):
    log("rms_norm %d x %d fmt=%d static=%d" % (rows, cols, fmt, static))
    rng = np.random.default_rng(rows * 7919 + cols)
    x, r, w = bf16_tensor(rng, rows, cols), bf16_tensor(rng, rows, cols, 2.0), _weight(rng, cols)
    _check(x, w, r, fmt, static)
    _check(x, w, None, fmt, static)


@pytest.mark.parametrize("cols", [1, 2, 7, 15, 16, 17, 31, 1000, 1001, 1023, 3077, 4097, 5003, 16385, 65537])
@pytest.mark.parametrize("rows", [1, 2, 19])
@pytest.mark.parametrize("fmt,static", [(BF16, False), (FP8, False), (FP8, True)])
def test_odd_lengths(rows, cols, fmt, static):
    rng = np.random.default_rng(rows * 101 + cols)
    x, r, w = bf16_tensor(rng, rows, cols), bf16_tensor(rng, rows, cols, 2.0), _weight(rng, cols, torch.float32)
    _check(x, w, r, fmt, static)


@pytest.mark.parametrize("cols", [48, 528, 4112, 16400])
@pytest.mark.parametrize("rows", [1, 18])
def test_nvfp4_rows_of_an_odd_number_of_blocks(rows, cols):
    rng = np.random.default_rng(cols)
    for static in (False, True):
        _check(bf16_tensor(rng, rows, cols), _weight(rng, cols), None, NVFP4, static)


@pytest.mark.parametrize("shift", [0, 1, 3, 8])
@pytest.mark.parametrize("pitch", [1040, 1043])
@pytest.mark.parametrize("fmt", [BF16, FP8, NVFP4, MXFP4, MXFP8])
def test_slices_of_wider_rows(fmt, pitch, shift):
    """Rows of any pitch and alignment; nothing outside the sum's rows is written."""
    rng = np.random.default_rng(pitch + shift)
    rows, cols = 21, 1024

    def wide():
        return bf16_tensor(rng, rows, pitch)[:, shift:shift + cols]
    x, r, w = wide(), wide(), _weight(rng, cols + 1)[1:]
    buf = torch.full((rows + 1, pitch), 77.0, dtype=torch.bfloat16, device=DEV)
    _check(x, w, r, fmt, sum_out=buf[:rows, shift:shift + cols])
    assert bool((buf[rows] == 77).all()) and bool((buf[:, :shift] == 77).all()) and bool((buf[:, shift + cols:] == 77).all())


@pytest.mark.parametrize("rows,cols", [(1, 1024), (300, 1024), (7, 6000), (3, 70000)])
@pytest.mark.parametrize("fmt", [BF16, FP8])
def test_sum_in_place(rows, cols, fmt):
    rng = np.random.default_rng(cols)
    x, r, w = bf16_tensor(rng, rows, cols), bf16_tensor(rng, rows, cols, 2.0), _weight(rng, cols)
    want, want_h = _run(x, w, r, fmt, False)
    for into_residual in (False, True):
        a, b = x.clone(), r.clone()
        y, h = _run(a, w, b, fmt, False, sum_out=b if into_residual else a)
        assert h is (b if into_residual else a) and torch.equal(h, want_h)
        assert torch.equal(a, x) == into_residual and torch.equal(b, r) != into_residual
        assert torch.equal(y.codes, want.codes) if fmt == FP8 else torch.equal(y, want)


@pytest.mark.parametrize("cols", [64, 1024, 5000, 70000])
def test_rows_of_extreme_values(cols):
    """Squares past fp32's range and below it, zero rows (also at eps = 0), single nonzero elements."""
    rng = np.random.default_rng(cols)
    x = bf16_tensor(rng, 8, cols).float()
    x[0] *= 1e37            # squares overflow
    x[1] = 3.0e38           # the largest, all equal
    x[2] *= 1e-30           # squares underflow: eps decides
    x[3] = 0.0
    x[4] = 0.0
    x[4, cols - 1] = -2.0 ** 100
    x[5] = 0.0
    x[5, 0] = 2.0 ** -120
    x[6] *= 1e18            # the sum overflows, no single square
    x = x.bfloat16()
    w = _weight(rng, cols)
    for fmt in (BF16, FP8):
        y, _ = _check(x, w, None, fmt)
        assert not host((y if fmt == BF16 else y.codes)[3]).any() if fmt == FP8 else not y[3].any()
    y = q.rms_norm(torch.zeros_like(x), w, 0.0)
    assert not y.any()
    s = q.rms_norm(torch.zeros_like(x), w, EPS, fmt=FP8)
    assert not s.codes.any() and float(s.tensor_scale) == 0.0


def test_non_finite_rows_stay_in_their_row():
    rng = np.random.default_rng(1)
    for rows, cols in ((5, 512), (3, 5000)):
        x, w = bf16_tensor(rng, rows, cols), _weight(rng, cols)
        x[1, 7], x[2, 9] = float("inf"), float("nan")
        y = q.rms_norm(x, w, EPS)
        _, y64 = reference(x[:1], w, EPS)
        check_norm(y[:1], y64, BF16)
        assert bool(y[1].isnan().any()) and bool(y[2].isnan().any())
        s = q.rms_norm(x, w, EPS, fmt=FP8)
        assert bool(s.tensor_scale.isnan())
        m = q.rms_norm(x[:, :512].contiguous(), w[:512].contiguous(), EPS, fmt=MXFP8)
        assert bool((m.block_scales[0] != 255).all()) and bool((m.block_scales[1] == 255).any())


def test_empty():
    w = torch.ones(64, device=DEV, dtype=torch.bfloat16)
    y = q.rms_norm(torch.empty((0, 64), dtype=torch.bfloat16, device=DEV), w, EPS, fmt=FP8)
    assert y.codes.shape == (0, 64) and float(y.tensor_scale) == 0.0
    y, h = q.rms_norm(torch.empty((3, 0), dtype=torch.bfloat16, device=DEV), w[:0], EPS,
                      residual=torch.empty((3, 0), dtype=torch.bfloat16, device=DEV))
    assert y.shape == (3, 0) and h.shape == (3, 0)


def test_without_a_stored_sum():
    """sum = NULL: the same y, the scale of the tensor included (x and the residual are read twice)."""
    rng = np.random.default_rng(5)
    rows, cols = 40, 2048
    x, r, w = bf16_tensor(rng, rows, cols), bf16_tensor(rng, rows, cols), _weight(rng, cols)
    want, _ = _run(x, w, r, FP8, False)
    codes = torch.empty((rows, cols), dtype=torch.uint8, device=DEV)
    ts = torch.empty(1, device=DEV)
    q.qg_rms_norm(FP8, x, cols, r, cols, w, q.QG_OUT_BF16, EPS, rows, cols, None, 0, codes, cols, None, ts)
    torch.cuda.synchronize()
    assert torch.equal(codes, want.codes) and torch.equal(ts, want.tensor_scale)


def test_codes_at_odd_addresses():
    """FP8 and MXFP8 codes of any alignment, and a bf16 y of its own pitch."""
    rng = np.random.default_rng(6)
    rows, cols = 30, 992
    x, w = bf16_tensor(rng, rows, cols), _weight(rng, cols)
    for fmt in (FP8, MXFP8):
        want, _ = _run(x, w, None, fmt, False)
        for shift in (0, 1, 5):
            buf = torch.full((rows * cols + 16,), 77, dtype=torch.uint8, device=DEV)
            bs = torch.empty((rows, cols // 32), dtype=torch.uint8, device=DEV) if fmt == MXFP8 else None
            ts = torch.empty(1, device=DEV) if fmt == FP8 else None
            q.qg_rms_norm(fmt, x, cols, None, 0, w, q.QG_OUT_BF16, EPS, rows, cols, None, 0, buf[shift:], cols, bs, ts)
            torch.cuda.synchronize()
            assert torch.equal(buf[shift:shift + rows * cols].view(rows, cols), want.codes)
            assert bool((buf[:shift] == 77).all()) and bool((buf[shift + rows * cols:] == 77).all())
    buf = torch.full((rows + 1, cols + 5), 77.0, dtype=torch.bfloat16, device=DEV)
    q.qg_rms_norm(BF16, x, cols, None, 0, w, q.QG_OUT_BF16, EPS, rows, cols, None, 0, buf, cols + 5, None, None)
    torch.cuda.synchronize()
    assert torch.equal(buf[:rows, :cols], q.rms_norm(x, w, EPS))
    assert bool((buf[rows] == 77).all()) and bool((buf[:, cols:] == 77).all())


def test_dynamic_scale_of_tiny_tensors():
    """Codes too small a buffer for the maxima of the first launch."""
    rng = np.random.default_rng(8)
    for rows, cols in ((17, 1), (40, 1), (100, 3), (33, 2)):
        _check(bf16_tensor(rng, rows, cols), _weight(rng, cols), None, FP8)


def test_graph_replays():
    """A captured call (one launch, and three with the tensor's scale) replayed on new inputs, eager work between."""
    rng = np.random.default_rng(9)
    w = _weight(rng, 2048)
    for rows in (4, 200):
        x, r = bf16_tensor(rng, rows, 2048), bf16_tensor(rng, rows, 2048)
        q.rms_norm(x, w, EPS, residual=r, fmt=FP8)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            y, h = q.rms_norm(x, w, EPS, residual=r, fmt=FP8)
        for _ in range(3):
            x.copy_(bf16_tensor(rng, rows, 2048))
            g.replay()
            want, want_h = q.rms_norm(x, w, EPS, residual=r, fmt=FP8)
            torch.cuda.synchronize()
            assert torch.equal(y.codes, want.codes) and torch.equal(y.tensor_scale, want.tensor_scale) and torch.equal(h, want_h)


def test_side_stream():
    rng = np.random.default_rng(10)
    x, w = bf16_tensor(rng, 500, 3072), _weight(rng, 3072)
    want, _ = _run(x, w, None, FP8, False)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for stream in (side, side.cuda_stream):
        y = q.rms_norm(x, w, EPS, fmt=FP8, stream=stream)
        side.synchronize()
        assert torch.equal(y.codes, want.codes) and torch.equal(y.tensor_scale, want.tensor_scale)
    with torch.cuda.stream(side):
        y = q.rms_norm(x, w, EPS, fmt=FP8)
    side.synchronize()
    assert torch.equal(y.codes, want.codes)
