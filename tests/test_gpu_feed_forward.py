"""The feed-forward half of a transformer block as three launches of the library:
rms_norm of the residual sum into the linear's format, linear_gated, linear_fused
onto the residual stream. Each step against its formula in 64 bits, from what the
step before it returned; eagerly, and captured and replayed on new inputs."""
import numpy as np
import pytest
import torch

import paper_2609_21849_amd as q
from fused_util import FMTS, check_finished, finished
from gpu_util import DEV, log
from norm_util import bf16_tensor, check_norm, reference

pytestmark = pytest.mark.gpu

EPS = 1e-6
SCALES = {"fp8": (6.0 / 448, 8.0 / 448), "nvfp4": (6.0 / 2688, 8.0 / 2688)}


class Block:
    def __init__(self, kind, hidden, ffn, seed=7):
        rng = np.random.default_rng(seed)
        self.kind, self.fmt, self.hidden, self.ffn = kind, FMTS[kind], hidden, ffn
        self.norm = (1 + 0.1 * bf16_tensor(rng, 1, hidden)[0].float()).bfloat16()
        self.up = q.pack_gated(bf16_tensor(rng, ffn, hidden, 0.05), bf16_tensor(rng, ffn, hidden, 0.05), self.fmt)
        self.down = q.pack(q.quantize(bf16_tensor(rng, hidden, ffn, 0.05), self.fmt))
        self.scales = [torch.full((1,), s, device=DEV) for s in SCALES.get(kind, ())]

    def normed(self, x, r):
        fmt = q.QG_FMT_BF16 if self.kind == "w4a16" else self.fmt
        return q.rms_norm(x, self.norm, EPS, residual=r, fmt=fmt, static_scale=self.scales[0] if self.scales else None)

    def gated(self, a):
        if not self.scales:
            return q.linear_gated(a, self.up, self.fmt, self.ffn)
        return q.linear_gated(a, self.up, self.fmt, self.ffn, y_scale=self.scales[1],
                              out_dtype=q.QG_OUT_FP8 if self.kind == "fp8" else q.QG_OUT_NVFP4)

    def __call__(self, x, r):
        a, h = self.normed(x, r)
        g = self.gated(a)
        if self.kind in ("mxfp4", "mxfp8"):
            g = q.quantize(g, self.fmt)
        y = q.linear_fused(g, self.down, self.fmt, self.hidden, residual=h)
        return a, h, g, y


@pytest.mark.parametrize("kind", list(FMTS))
@pytest.mark.parametrize("m,hidden,ffn", [(1, 256, 768), (77, 512, 1024), (700, 1024, 2304)])
def test_each_step(kind, m, hidden, ffn):
    log("feed forward %s m=%d" % (kind, m))
    rng = np.random.default_rng(m)
    block = Block(kind, hidden, ffn)
    x, r = bf16_tensor(rng, m, hidden), bf16_tensor(rng, m, hidden, 2.0)
    a, h, g, y = block(x, r)
    torch.cuda.synchronize()
    assert torch.equal(h, (x.float() + r.float()).bfloat16())
    _, n64 = reference(x, block.norm, EPS, r)
    check_norm(a, n64, q.QG_FMT_BF16 if kind == "w4a16" else block.fmt, static=bool(block.scales))
    z = q.linear(a, block.up, block.fmt, 2 * ffn, out_dtype=q.QG_OUT_F32)
    y64, err = finished(z, act=q.QG_ACT_SILU, gated=True)
    if kind in ("mxfp4", "mxfp8"):
        check_finished(block.gated(a), y64, err)
    else:
        check_finished(g, y64, err, float(block.scales[1]) if block.scales else None)
    z = q.linear(g, block.down, block.fmt, hidden, out_dtype=q.QG_OUT_F32)
    y64, err = finished(z, residual=h)
    check_finished(y, y64, err)


@pytest.mark.parametrize("kind", ["fp8", "nvfp4", "mxfp8", "w4a16"])
def test_captured(kind):
    rng = np.random.default_rng(11)
    m, hidden, ffn = 130, 512, 1024
    block = Block(kind, hidden, ffn)
    x, r = bf16_tensor(rng, m, hidden), bf16_tensor(rng, m, hidden, 2.0)
    block(x, r)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = block(x, r)[3]
    for _ in range(3):
        x.copy_(bf16_tensor(rng, m, hidden))
        graph.replay()
        want = block(x, r)[3]
        torch.cuda.synchronize()
        assert torch.equal(y, want)


def test_two_streams_at_once():
    """The same weights read by two calls that run side by side."""
    rng = np.random.default_rng(12)
    block = Block("fp8", 1024, 2304)
    inputs = [(bf16_tensor(rng, m, 1024), bf16_tensor(rng, m, 1024)) for m in (300, 9)]
    want = [block(*v)[3] for v in inputs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in inputs]
    got = []
    for s, v in zip(streams, inputs):
        with torch.cuda.stream(s):
            got.append(block(*v)[3])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
