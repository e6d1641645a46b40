"""rms_norm where the squares leave fp32's range, upwards and downwards, against its
formula in 64 bits, and that a row's norm does not depend on the rows beside it."""
import numpy as np
import pytest
import torch

import paper_2609_21849_amd as q
from gpu_util import log
from norm_util import bf16_tensor, check_norm, reference

pytestmark = pytest.mark.gpu

# lanes of a wave, a workgroup of 128, 256 (few and many rows) and 1024, a row walked twice; row ends inside a unit
COLS = [48, 333, 2048, 4096, 5000, 12001, 20000, 49200]


def _check(x, cols, eps, rng):
    w = torch.from_numpy((1.0 + 0.2 * rng.standard_normal(cols)).astype(np.float32)).cuda()
    for residual in (False, True):
        for rows in (len(x), 300):
            t = x.repeat(-(-rows // len(x)), 1)[:rows]
            res = torch.zeros_like(t) if residual else None
            _, y64 = reference(t, w, eps, res)
            y = q.rms_norm(t, w, eps, residual=res)
            check_norm(y if res is None else y[0], y64, q.QG_FMT_BF16)


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("eps", [1e34, 1e37, 3e38])
def test_large_eps_beside_an_overflowing_sum(cols, eps):
    log("rms_norm cols=%d eps=%g" % (cols, eps))
    rng = np.random.default_rng(cols)
    x = bf16_tensor(rng, 5, cols).float() * torch.tensor([[2.0 ** 58], [2.0 ** 61], [2.0 ** 63], [2.0 ** 70], [2.0 ** 120]], device="cuda")
    _check(x.bfloat16(), cols, eps, rng)


@pytest.mark.parametrize("cols", COLS)
def test_small_elements_of_an_overflowing_row(cols):
    """One element past 2^64 and the rest far below it: those keep their digits."""
    log("rms_norm cols=%d" % cols)
    rng = np.random.default_rng(cols)
    x = bf16_tensor(rng, 4, cols).float() * torch.tensor([[2.0 ** -20], [2.0 ** -35], [2.0 ** -40], [2.0 ** -45]], device="cuda")
    x[:, cols // 3] = 2.0 ** 70
    _check(x.bfloat16(), cols, 1e-6, rng)


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("eps", [0.0, 1e-45, 1e-40, 1e-37, 1e-35])
def test_squares_below_the_smallest_number(cols, eps):
    """Rows whose squares are subnormal or zero, where eps does not hide them."""
    log("rms_norm cols=%d eps=%g" % (cols, eps))
    rng = np.random.default_rng(cols)
    x = bf16_tensor(rng, 7, cols).float() * torch.tensor([[1e-12], [1e-17], [1e-20], [1e-22], [1e-30], [1e-38], [0.0]], device="cuda")
    x[6, cols // 2] = 2.0 ** -133  # the smallest bf16
    _check(x.bfloat16(), cols, eps, rng)


@pytest.mark.parametrize("cols", COLS)
def test_squares_below_the_smallest_number_quantized(cols):
    rng = np.random.default_rng(cols)
    cols = cols // 32 * 32
    x, w = (1e-30 * bf16_tensor(rng, 20, cols).float()).bfloat16(), torch.ones(cols, device="cuda")
    _, y64 = reference(x, w, 0.0)
    for fmt in (q.QG_FMT_FP8_E4M3, q.QG_FMT_NVFP4, q.QG_FMT_MXFP4, q.QG_FMT_MXFP8):
        check_norm(q.rms_norm(x, w, 0.0, fmt=fmt), y64, fmt)


@pytest.mark.parametrize("cols", [40, 1024, 3001, 4096, 4112, 5003, 6144, 9216, 12305, 16384, 20000])
def test_a_row_among_any_number_of_rows(cols):
    """The sum's order is fixed by cols: the same bits in calls of 1024, 257, 256 and one row."""
    log("rms_norm rows of cols=%d" % cols)
    rng = np.random.default_rng(cols)
    x = bf16_tensor(rng, 1024, cols)
    w = torch.from_numpy((1.0 + 0.2 * rng.standard_normal(cols)).astype(np.float32)).cuda()
    y = q.rms_norm(x, w)
    for part in (256, 257):
        for i in range(0, 1024, part):
            assert torch.equal(q.rms_norm(x[i:i + part], w), y[i:i + part])
    for i in (0, 511, 1023):
        assert torch.equal(q.rms_norm(x[i:i + 1], w), y[i:i + 1])
