"""Scales of either sign and any size: logits are sums of exact products, scaled in fp32, in bf16 too."""
import math

import numpy as np
import pytest
import torch

from paper_2603_06738_amd import binding as rb
from test_gpu_rpb import DEV, Case, close, np64, storage

pytestmark = pytest.mark.gpu
H = 2.0 ** -24          # half a step of fp32


# (scale, sizes of q and k that bring the logits to the order of 1)
SCALES = [(0.18, 1, 1), (-0.4, 1, 1), (-1e-9, 1, 1e9), (2.0 ** -39, 2.0 ** 20, 2.0 ** 19), (3e-20, 1, 3e19), (-2.0 ** -140, 2.0 ** 20, 2.0 ** 120), (1e12, 1e-6, 1e-6),
          (-3e30, 1e-15, 1e-15), (0.0, 1, 1)]


@pytest.mark.parametrize("dtype,M,d", [("bf16", 7, 30), ("bf16", 9, 32), ("bf16", 16, 30), ("bf16", 16, 15), ("bf16", 24, 48), ("f32", 5, 30), ("f32", 16, 30)])
@pytest.mark.parametrize("scale,qsize,ksize", SCALES)
def test_logits_are_exact(dtype, M, d, scale, qsize, ksize):
    """Every token sees the one below it alone, so LSE is the logit: d + 8 fp32 roundings of a sum of d products and a bias, 4 more for the
    way to base 2 and back, 2^-20 for exp2 and the logarithm.  fp32 rounds scale * q beside that, once."""
    c = Case(dtype, 1, M, M, 1, d, M, 0, seed=M + d, scale=scale)
    rng = np.random.default_rng(M)
    c.q, c.k = (storage(rng.standard_normal(c.q.shape) * s, dtype).to(DEV) for s in (qsize, ksize))
    c.bias.fill_(-math.inf)
    c.bias[:, (2 * M - 1) ** 2 // 2 - (2 * M - 1)] = 0.37
    rb.rib_rpb_attn_fwd(c.p, c.q, c.k, c.v, c.bias, c.out, c.lse)
    scale, bias = float(np.float32(scale)), float(np.float32(0.37))
    q, k = np64(c.q)[0, :-1], np64(c.k)[0, 1:]
    want, mag = np.full((M, M), -np.inf), np.zeros((M, M))
    want[:-1] = scale * (q * k).sum(-1) + bias
    mag[:-1] = abs(scale) * (abs(q) * abs(k)).sum(-1) + bias
    close("lse", c.lse[0, 0].reshape(M, M), want, (d + 13) * H * mag + 2.0 ** -20)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [1.0, 2.0 ** -39, -2.0 ** -39])
def test_biases_next_to_the_border_do_not_exclude(dtype, scale):
    """A bias of -9e29 for every pair: it is above -1e30, so no row is empty.  Logits of that size are all alike in fp32: O is the mean."""
    for M in (7, 16):
        c = Case(dtype, 1, M, M, 2, 30, M, 1, seed=M, scale=scale)
        c.bias.fill_(-9e29)
        rb.rib_rpb_attn_fwd(c.p, c.q, c.k, c.v, c.bias, c.out, c.lse)
        u = 2.0 ** -8 if dtype == "bf16" else H
        v = np64(c.v)
        mean = v.mean((1, 2), keepdims=True)
        close("out", c.out, np.broadcast_to(mean, v.shape), np.broadcast_to(u * abs(mean) + (M * M + 8) * H * abs(v).mean((1, 2), keepdims=True), v.shape))
        close("lse", c.lse, np.full(c.lse.shape, float(np.float32(-9e29))), np.full(c.lse.shape, 8 * H * 9e29))
