"""Formats and activations past 32 bits are refused: the buffers are allocated by the
number given, and what ctypes would hand to the library is another one."""
import pytest
import torch

import paper_2609_21849_amd as q
from gpu_util import DEV

pytestmark = pytest.mark.gpu

INVALID = 1


@pytest.mark.parametrize("fmt", [2 ** 32 + f for f in range(5)] + [-1, 5, -2 ** 32 + 1])
@pytest.mark.parametrize("static", [False, True])
def test_norm_formats(fmt, static):
    x, w = torch.zeros((4, 128), dtype=torch.bfloat16, device=DEV), torch.ones(128, device=DEV)
    s = torch.ones(1, device=DEV) if static else None
    with pytest.raises(q.QGError) as e:
        q.rms_norm(x, w, fmt=fmt, static_scale=s)
    assert e.value.status == INVALID


@pytest.mark.parametrize("act", [2 ** 32, 2 ** 32 + 1, -2 ** 32, -1, 4])
def test_activations(act):
    fmt = q.QG_FMT_FP8_E4M3
    a = q.quantize(torch.ones((4, 256), dtype=torch.bfloat16, device=DEV), fmt)
    packed = q.pack(q.quantize(torch.ones((32, 256), dtype=torch.bfloat16, device=DEV), fmt))
    for call in (lambda: q.linear_fused(a, packed, fmt, 32, act=act), lambda: q.linear_gated(a, packed, fmt, 16, act=act)):
        with pytest.raises(q.QGError) as e:
            call()
        assert e.value.status == INVALID
