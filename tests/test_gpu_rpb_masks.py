"""Masks that cover a whole row without excluding it: finite, but far below every logit."""
import numpy as np
import pytest
import torch

from paper_2603_06738_amd import binding as rb
from test_gpu_rpb import Case, np64, repeated

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,M,d,copies", [("bf16", 7, 30, 1), ("bf16", 8, 64, 1), ("bf16", 16, 30, 1), ("bf16", 16, 15, 1), ("bf16", 16, 30, 180), ("bf16", 20, 32, 100), ("bf16", 24, 48, 60),
                                              ("f32", 5, 30, 1), ("f32", 12, 30, 1), ("f32", 16, 40, 1)])
@pytest.mark.parametrize("mask", [-1e9, -3e10, -9e29])
def test_a_row_masked_by_a_finite_value(dtype, M, d, copies, mask):
    """Attention to earlier tokens, the others at `mask`: the window's first token has nothing else.  Everything stays finite.  With a running
    maximum from the start (else the first token's row calls for it, and its neighbours' sums round in another order) the other tokens' rows are
    bit for bit those of a mask of minus infinity; the first adds to dk and dv no more than probabilities of 1 give: |dO| to dv, and to dk, with
    |dS| <= |dO.v| + |dO.out|, that times scale |q|."""
    c = Case(dtype, 1, M, M, 1, d, M, 0, buckets="past", seed=M + d)
    if copies > 1:
        c = repeated(c, copies)
    names = ("dq", "dk", "dv", "dbias")

    def gradients():
        rb.rib_rpb_attn_fwd(c.p, c.q, c.k, c.v, c.bias, c.out, c.lse)
        rb.rib_rpb_attn_bwd(c.p, c.q, c.k, c.v, c.bias, c.out, c.dout, c.lse, c.dq, c.dk, c.dv, c.dbias, c.ws)
        return c.out.clone(), c.lse.clone(), *(getattr(c, n).clone() for n in names)

    rb.rib_rpb_table_fwd(c.tp, c.table, c.index, c.bias)
    past = torch.isfinite(c.bias)
    c.bias = torch.where(past, c.bias, torch.full_like(c.bias, mask))
    assert all(torch.isfinite(x).all() for x in gradients())
    c.p.flags = rb.RIB_FLAG_FORCE_ROW_MAX
    out, lse, dq, dk, dv, dbias = gradients()
    assert all(torch.isfinite(x).all() for x in (out, lse, dq, dk, dv, dbias))
    c.bias = torch.where(past, c.bias, torch.full_like(c.bias, -np.inf))
    out0, lse0, dq0, dk0, dv0, dbias0 = gradients()
    N = M * M
    flat = [x[0].reshape(N, d) for x in (out0, out, dq0, dq)]
    assert torch.equal(flat[0][1:], flat[1][1:]) and torch.equal(flat[2][1:], flat[3][1:]) and torch.equal(lse0[..., 1:], lse[..., 1:])
    u = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    q, v, do = (np64(x)[0].reshape(N, d) for x in (c.q, c.v, c.dout))
    o = np64(out)[0].reshape(N, d)
    # (rounded once as an operand, once in fp32 sums of N terms; dk and dv are themselves rounded on both sides)
    room = 1 + 2 * u + N * 2.0 ** -23
    dS = abs(do[0] @ v.T) + abs(do[0] @ o[0])
    for a, b, most in ((dv0, dv, np.broadcast_to(abs(do[0]), (N, d))), (dk0, dk, c.scale * dS[:, None] * abs(q[0]))):
        a, b = (np64(x)[0].reshape(N, d) for x in (a, b))
        assert (abs(a - b) <= room * most + 3 * u * (abs(a) + abs(b)) + 1e-5).all()
    assert ((dbias - dbias0)[:, past[0]] == 0).all()
