"""8-bit checkpoints of rows whose values lie at the upper end of their type: what they stand for is finite, and the backward takes it
from the codes as it takes it from tensors."""
import itertools

import numpy as np
import pytest
import torch

import rpb_reference as ref
from paper_2603_06738_amd import binding as rb
from test_gpu_rpb import DEV, Case, np64, packed, storage

pytestmark = pytest.mark.gpu


def expected(rows):
    """(codes, exponent bytes, values) of rows [..., d] of 64-bit floats, finite and not all zero: the smallest step that holds the largest
    as 127 or less, 2^121 at most; there codes stay within 127."""
    big = np.abs(rows).max(-1, keepdims=True)
    e = np.ones(big.shape, int)
    for _ in range(247):
        e = np.where((big > 127 * 2.0 ** (e - 127.0)) & (e < 248), e + 1, e)
    step = 2.0 ** (e - 127.0)
    codes = np.clip(np.rint(rows / step), -127, 127)
    return (codes + 128).astype(np.uint8), e[..., 0].astype(np.uint8), codes * step


# the last row a step of 2^120 holds, the next value above it, 2^127, the last one 2^121 holds, the largest
TOPS = {"bf16": (127 * 2.0 ** 120, 255 * 2.0 ** 119, 2.0 ** 127, 127 * 2.0 ** 121, 255 * 2.0 ** 120),
        "f32": (127 * 2.0 ** 120, 127 * 2.0 ** 120 * (1 + 2.0 ** -23), 2.0 ** 127, 127 * 2.0 ** 121, (2.0 ** 24 - 1) * 2.0 ** 104)}


@pytest.mark.parametrize("dtype,d", itertools.product(("bf16", "f32"), (1, 7, 30, 40, 64)))
def test_codes_of_the_largest_values(dtype, d):
    M, heads = 3, 2
    c = Case(dtype, 1, M, 2 * M, heads, d, M, 0, seed=d)
    for j, x in enumerate((c.q, c.k, c.v)):
        for i, top in enumerate(TOPS[dtype]):
            row = x[0, i % M, i, j % heads * d:][:d]
            row *= 2.0 ** 118                               # (normal values: far below the largest)
            row[(i + j) % d] = top if i % 2 == 0 else -top
        assert torch.isfinite(x).all()
    ck = packed(c).cpu().numpy()
    dp, rows = (d + 15) // 16 * 16, 2 * heads * M * M
    back = [torch.full_like(c.q, 3.0) for _ in range(3)]
    rb.rib_checkpoint_unpack(c.p, torch.from_numpy(ck).to(DEV), *back)
    again = torch.full((ck.size,), 0xff, dtype=torch.uint8, device=DEV)
    rb.rib_checkpoint_pack(c.p, *back, again)
    for i, x in enumerate((c.q, c.k, c.v)):
        grid = np64(x).reshape(M, 2, M, heads, d).transpose(1, 3, 0, 2, 4).reshape(rows, d)       # one image, no shift: [window][head][token]
        codes, exps, values = expected(grid)
        assert np.array_equal(ck[3 * rows * dp + i * rows:3 * rows * dp + (i + 1) * rows], exps)
        got = ck[i * rows * dp:(i + 1) * rows * dp].reshape(rows, dp)
        assert np.array_equal(got[:, :d], codes) and (got[:, d:] == 128).all()
        unpacked = np64(back[i]).reshape(M, 2, M, heads, d).transpose(1, 3, 0, 2, 4).reshape(rows, d)
        assert np.isfinite(unpacked).all() and np.array_equal(unpacked, values)
    assert np.array_equal(again.cpu().numpy(), ck)          # (packing what a checkpoint stands for changes nothing)


@pytest.mark.parametrize("dtype,M,d", [("bf16", 7, 30), ("bf16", 9, 30), ("bf16", 16, 30), ("bf16", 16, 32), ("bf16", 12, 15), ("bf16", 24, 40),
                                       ("f32", 5, 30), ("f32", 9, 30), ("f32", 16, 40)])
def test_backward_from_a_checkpoint_of_the_largest_values(dtype, M, d):
    """Keys of up to the largest finite value against queries of 2^-120, values likewise against a gradient of 2^-120: everything that
    comes out is an ordinary number, and bit for bit what the exact values as tensors give."""
    c = Case(dtype, 1, M, M, 1, d, M, 0, seed=M)
    rng = np.random.default_rng(d)
    top = TOPS[dtype][-1]

    def large():
        return storage(np.clip(rng.standard_normal((1, M, M, d)) * 2.0 ** 126, -top, top), dtype).to(DEV)

    for huge in "kv":
        c.q, c.k, c.v = (storage(rng.standard_normal((1, M, M, d)), dtype).to(DEV) for _ in range(3))
        c.dout = storage(rng.standard_normal((1, M, M, d)), dtype).to(DEV)
        setattr(c, huge, large())
        assert (getattr(c, huge).abs().amax(-1) > 127 * 2.0 ** 120).any()
        if huge == "k":
            c.q, c.dout = c.q * 2.0 ** -124, c.dout * 2.0 ** -10        # (dS sums up to 2^-10 * 30, times a key under 2^128: not above it)
        else:
            c.dout = c.dout * 2.0 ** -124
        c.forward()
        assert torch.isfinite(c.lse).all()
        c.out = storage(np.zeros((1, M, M, d)), dtype).to(DEV) if huge == "v" else c.out      # (dO.out stays an ordinary number either way)
        ck = packed(c)
        held = [expected(np64(x).reshape(M * M, d))[2].reshape(1, M, M, d) for x in (c.q, c.k, c.v)]
        exact = [storage(x, dtype).to(DEV) for x in held]
        assert all(np.array_equal(np64(t), x) for t, x in zip(exact, held))
        names = ("dq", "dk", "dv", "dbias")
        rb.rib_rpb_attn_bwd(c.p, *exact, c.bias, c.out, c.dout, c.lse, c.dq, c.dk, c.dv, c.dbias, c.ws)
        want = [getattr(c, n).clone() for n in names]
        for n in names:
            getattr(c, n).fill_(float("nan"))
        rb.rib_rpb_attn_bwd_ckpt(c.p, ck, c.bias, c.out, c.dout, c.lse, c.dq, c.dk, c.dv, c.dbias, c.ws)
        for n, x in zip(names, want):
            assert torch.isfinite(x).all() and torch.equal(getattr(c, n), x), (huge, n)


def test_reference_agrees_below_the_top():
    """The rule here is the format's: the same codes as the reference's where no row is above 127 * 2^121."""
    rng = np.random.default_rng(0)
    x = rng.standard_normal((1, 4, 4, 10)) * 2.0 ** rng.integers(-100, 124, (1, 4, 4, 1))
    codes, exps = ref.pack(x, 1, 4, 0)
    mine = expected(x.reshape(16, 10))
    assert np.array_equal(codes[0, :, :10], mine[0]) and np.array_equal(exps[0], mine[1])


@pytest.mark.parametrize("M,d", [(7, 30), (16, 30), (20, 32), (16, 64)])
def test_backward_from_a_checkpoint_beside_unaligned_tensors(M, d):
    """out, d_out and the gradients one value into their allocations: as from the unpacked tensors, which then run on the same kernels however they
    lie.  Where out, d_out and the gradients are aligned and the unpacked tensors are not, the bits may differ: only the roundings do (three of
    bf16's on the way of any term: P or dS, the sum's order, the output)."""
    c = Case("bf16", 1, M, 2 * M, 1, d, M, 1, seed=M)
    c.forward()
    ck = packed(c)
    held = [torch.empty_like(c.q) for _ in range(3)]
    rb.rib_checkpoint_unpack(c.p, ck, *held)
    names = ("out", "dout", "dq", "dk", "dv")

    def off(x):
        view = torch.full((x.numel() + 8,), 7.0, dtype=x.dtype, device=DEV)[1:1 + x.numel()].view(x.shape)
        return view.copy_(x)

    def run(call, *first, t):
        call(c.p, *first, c.bias, t["out"], t["dout"], c.lse, t["dq"], t["dk"], t["dv"], c.dbias, c.ws)
        return [t[n].clone() for n in ("dq", "dk", "dv")] + [c.dbias.clone()]

    aligned = {n: getattr(c, n) for n in names}
    moved = {n: off(x) for n, x in aligned.items()}
    want = run(rb.rib_rpb_attn_bwd_ckpt, ck, t=moved)
    for tensors in (held, [off(x) for x in held]):
        for a, b in zip(want, run(rb.rib_rpb_attn_bwd, *tensors, t=moved)):
            assert torch.equal(a, b)
    for a, b in zip(run(rb.rib_rpb_attn_bwd_ckpt, ck, t=aligned), run(rb.rib_rpb_attn_bwd, *[off(x) for x in held], t=aligned)):
        assert (a - b).float().norm() <= 3 * 2.0 ** -8 * a.float().norm()
