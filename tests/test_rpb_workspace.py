"""Scratch of the learned bias's backward: what a call asks for with and without the bias's gradient."""
import pytest
import torch

from paper_2603_06738_amd import binding as rb

FAKE = 0x10000          # non-NULL dummy "device pointer", aligned to everything


@pytest.mark.parametrize("dtype,B,M,heads", [("f32", 1, 4, 3), ("bf16", 2, 7, 3), ("bf16", 1, 96, 6), ("f32", 1, 33, 1)])
def test_what_is_asked_for(dtype, B, M, heads):
    """One byte less is refused (and that is all that can be shown without a GPU: the call that has enough launches)."""
    p = rb.make_params(B, M, 2 * M, heads, 4, 0, M, 0, 0.5, 0.0, dtype)
    small = (8 * B * M * 2 * M * heads + 255) // 256 * 256
    total = rb.rib_rpb_attn_bwd_workspace_bytes(p)
    assert total > small
    for nbytes, dbias in ((small - 1, None), (0, None), (total - 1, FAKE), (small, FAKE)):
        assert rb.rib_rpb_attn_bwd_status(p, *[FAKE] * 10, dbias, FAKE, nbytes, stream=0) == 5
        assert rb.rib_rpb_attn_bwd_ckpt_status(p, *[FAKE] * 8, dbias, FAKE, nbytes, stream=0) == 5


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,M,d,copies", [("bf16", 7, 30, 1), ("bf16", 16, 30, 1), ("bf16", 16, 64, 180), ("bf16", 20, 15, 1), ("f32", 5, 30, 1), ("f32", 12, 40, 1)])
def test_without_the_gradient_of_the_bias(dtype, M, d, copies):
    """The small scratch, with a guard behind it: the other gradients as with all of it, from tensors and from a checkpoint."""
    from test_gpu_rpb import DEV, Case, packed, repeated
    c = Case(dtype, 1, M, M, 2, d, M, 1, seed=M)
    if copies > 1:
        c = repeated(c, copies)
    c.forward()
    need = (8 * c.q.shape[0] * M * M * 2 + 255) // 256 * 256
    ws = torch.full((need + 4096,), 0xa5, dtype=torch.uint8, device=DEV)
    ck = packed(c)
    for first, call in (((c.q, c.k, c.v), rb.rib_rpb_attn_bwd), ((ck,), rb.rib_rpb_attn_bwd_ckpt)):
        call(c.p, *first, c.bias, c.out, c.dout, c.lse, c.dq, c.dk, c.dv, c.dbias, c.ws)
        want = [x.clone() for x in (c.dq, c.dk, c.dv)]
        for x in (c.dq, c.dk, c.dv):
            x.fill_(float("nan"))
        call(c.p, *first, c.bias, c.out, c.dout, c.lse, c.dq, c.dk, c.dv, None, ws, need)
        assert all(torch.equal(a, b) for a, b in zip(want, (c.dq, c.dk, c.dv)))
        assert (ws[need:] == 0xa5).all()
