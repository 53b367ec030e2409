"""What a row's softmax is held in: LSE and the sums it comes from, in 32 bits through forward and backward."""
import math

import numpy as np
import pytest
import torch

from paper_2603_06738_amd import binding as rb
from test_gpu_rpb import DEV, Case, close, np64, repeated, storage

pytestmark = pytest.mark.gpu
H = 2.0 ** -24          # half a step of fp32
U = 2.0 ** -8           # and of bf16

# windows of up to 64 tokens, small grids whose waves share 64 stationary tokens, large grids; with strips and without; each source of rows
KERNELS = [(8, 30, 1), (8, 32, 1), (8, 15, 1), (7, 30, 1), (16, 30, 1), (16, 32, 1), (16, 15, 1), (16, 40, 1), (16, 64, 1), (16, 30, 180), (16, 15, 180), (16, 64, 180),
           (9, 30, 1), (9, 30, 180), (20, 32, 100), (32, 30, 1)]


def uniform(dtype, M, d, copies, value, seed):
    """A case whose logits are all `value`: q is zero, every bias `value`."""
    c = Case(dtype, 1, M, M, 1, d, M, 0, seed=seed, scale=1.0)
    c.q = torch.zeros_like(c.k)
    c.qkv = torch.cat((c.q, c.k, c.v), -1).contiguous()
    c.dout = storage(np.random.default_rng(seed).uniform(0.5, 1.5, c.dout.shape), dtype).to(DEV)
    c.bias.fill_(value)
    return repeated(c, copies) if copies > 1 else c


# (the negative ones: exp of them is zero without a maximum, the positive ones overflow; at the ones beyond 16000 a pair of bf16 parts is 0.04 to 0.09
# off for windows of 64, 256 and 1024 tokens)
@pytest.mark.parametrize("M,d,copies", KERNELS)
@pytest.mark.parametrize("value", [1000.0, -5000.0, 16475.75, 16490.25, 16473.0, -16420.25])
def test_gradients_of_rows_far_from_zero(M, d, copies, value):
    """Uniform rows: P = 1 / N whatever the logits' common value.  In fp32 the value rounds a handful of times at its size: bias in the
    product's unit (2), base 2 (2), LSE (top, its sum with the logarithm, base e and the store: 5), LSE in base 2 (2), the exponent (1);
    14 H |value| of P holds all of them.  P is then rounded to bf16 (U), as is dv (U).  dbias is a sum of dS, which is not rounded."""
    c = uniform("bf16", M, d, copies, value, M + d)
    N = M * M
    rb.rib_rpb_attn_fwd(c.p, c.q, c.k, c.v, c.bias, c.out, c.lse)
    rb.rib_rpb_attn_bwd(c.p, c.q, c.k, c.v, c.bias, c.out, c.dout, c.lse, c.dq, c.dk, c.dv, c.dbias, c.ws)
    t = 14 * H * (abs(value) + 10)
    do, v, k, out = (np64(x)[0].reshape(N, d) for x in (c.dout, c.v, c.k, c.out))
    close("lse", c.lse, np.full(c.lse.shape, value + math.log(N)), np.full(c.lse.shape, t + N * H))
    close("out", c.out[0].reshape(N, d), np.broadcast_to(v.mean(0), (N, d)), np.broadcast_to(U * abs(v.mean(0)) + (2 * U + t + N * H) * abs(v - v.mean(0)).mean(0)
                                                                                            + N * H * abs(v).mean(0), (N, d)))
    want = do.mean(0)
    close("dv", c.dv[0].reshape(N, d), np.broadcast_to(want, (N, d)), np.broadcast_to((1.02 * (t + U) + N * H) * want + U * want, (N, d)))
    delta = (do * out).sum(1, keepdims=True)
    dS = (do @ v.T - delta) / N
    # -delta as two bf16 parts: 2^-16 of it; fp32 sums of d products
    off = (2.0 ** -16 * abs(delta) + H * (d + 4) * (abs(do) @ abs(v).T + abs(do * out).sum(1, keepdims=True))) / N
    eS = 1.02 * t * abs(dS) + 1.02 * off
    close("dq", c.dq[0].reshape(N, d), dS @ k, 1.02 * ((eS + U * abs(dS)) + N * H * abs(dS)) @ abs(k) + U * abs(dS @ k) + 1e-30)
    assert (c.dk == 0).all()
    want, tol = np.zeros((2 * M - 1) ** 2), np.zeros((2 * M - 1) ** 2)
    iy, ix = np.divmod(np.arange(N), M)
    rel = (iy[:, None] - iy[None, :] + M - 1) * (2 * M - 1) + ix[:, None] - ix[None, :] + M - 1
    np.add.at(want, rel.reshape(-1), dS.reshape(-1))
    np.add.at(tol, rel.reshape(-1), (eS + 2 * H * abs(dS)).reshape(-1))
    close("dbias", c.dbias[0], copies * want, copies * (1.02 * tol + (copies + 40) * H * abs(want)) + 1e-30)


@pytest.mark.parametrize("M,d,copies", [k for k in KERNELS if k[1] in (15, 30)] + [(8, 8, 1), (7, 8, 1), (16, 8, 1), (16, 8, 180), (9, 9, 1), (9, 8, 180), (24, 8, 1)])
def test_gradients_that_vanish(M, d, copies):
    """Every token sees itself alone: dP = delta, so dS is zero but for the fp32 sums of d products, whatever the size of delta (positive
    dO and v of 1 to 2: the sum of their magnitudes is delta).  A sum of d products rounds at most d times at its size, H each, in two orders; LSE
    and P are 1 to within 1.02."""
    c = Case("bf16", 1, M, M, 1, d, M, 0, seed=M)
    rng = np.random.default_rng(d)
    c.v, c.dout = (storage(rng.uniform(1, 2, c.v.shape), "bf16").to(DEV) for _ in range(2))
    c.qkv = torch.cat((c.q, c.k, c.v), -1).contiguous()
    c.bias.fill_(-math.inf)
    c.bias[:, (2 * M - 1) ** 2 // 2] = 0.0
    if copies > 1:
        c = repeated(c, copies)
    rb.rib_rpb_attn_fwd(c.p, c.q, c.k, c.v, c.bias, c.out, c.lse)
    c.out.copy_(c.v)                # (what softmax of one key gives)
    rb.rib_rpb_attn_bwd(c.p, c.q, c.k, c.v, c.bias, c.out, c.dout, c.lse, c.dq, c.dk, c.dv, c.dbias, c.ws)
    q, k, v, do = (np64(x)[0] for x in (c.q, c.k, c.v, c.dout))
    off = 1.02 * 2 * d * H * (do * v).sum(-1, keepdims=True)
    assert (abs(np64(c.dq)[0]) <= 1.02 * c.scale * off * abs(k)).all() and (abs(np64(c.dk)[0]) <= 1.02 * c.scale * off * abs(q)).all()
    centre = (2 * M - 1) ** 2 // 2
    assert abs(float(c.dbias[0, centre])) <= 1.02 * copies * off.sum()
    assert (c.dbias[0, :centre] == 0).all() and (c.dbias[0, centre + 1:] == 0).all()


@pytest.mark.parametrize("M,d,copies", KERNELS + [(12, 46, 1), (12, 46, 100), (24, 62, 1), (5, 7, 1), (6, 64, 1), (1, 30, 1), (32, 32, 48)])
def test_rows_of_one_key(M, d, copies):
    """Every token sees one other alone (the one below it, and the last row of tokens none): O is that token's v and dv is dO, exactly, since
    P is divided by itself as rounded, and is 1 in the backward; LSE is the logit, to fp32's rounding of a sum of d products and a bias
    (d + 8 roundings of H), 2^-20 for exp2 and the logarithm, and H of it a few times."""
    c = Case("bf16", 1, M, M, 1, d, M, 0, seed=M + d)
    c.bias.fill_(-math.inf)
    offset = (2 * M - 1) ** 2 // 2 - (2 * M - 1 if M > 1 else 0)
    c.bias[:, offset] = 0.37
    if copies > 1:
        c = repeated(c, copies)
    rb.rib_rpb_attn_fwd(c.p, c.q, c.k, c.v, c.bias, c.out, c.lse)
    rb.rib_rpb_attn_bwd(c.p, c.q, c.k, c.v, c.bias, c.out, c.dout, c.lse, c.dq, c.dk, c.dv, c.dbias, c.ws)
    down = 1 if M > 1 else 0
    first = M - down                # rows of tokens that have a key
    assert torch.equal(c.out[:, :first], c.v[:, down:]) and (c.out[:, first:] == 0).all()
    assert torch.equal(c.dv[:, down:], c.dout[:, :first]) and (c.dv[:, :down] == 0).all()
    q, k = np64(c.q)[0, :first], np64(c.k)[0, down:]
    bias = float(np.float32(0.37))
    want = np.full((M, M), -np.inf)
    want[:first] = c.scale * (q * k).sum(-1) + bias
    mag = np.zeros((M, M))
    mag[:first] = c.scale * (abs(q) * abs(k)).sum(-1) + bias
    close("lse", c.lse[0, 0].reshape(M, M), want, (d + 12) * H * mag + 2.0 ** -20)
