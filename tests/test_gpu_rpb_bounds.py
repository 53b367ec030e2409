"""Every element of every result of the learned bias's attention, and the 2-norm of its error, within what the kernels round (rpb_bounds.py)."""
import itertools

import numpy as np
import pytest
import torch

import rpb_bounds
from paper_2603_06738_amd import binding as rb
from test_gpu_rpb import Case, np64, packed, repeated
import rpb_reference as ref

pytestmark = pytest.mark.gpu


def check(c, one=None, copies=1, bwd_qkv=None):
    """`one`: the single image that `c` repeats."""
    one = one or c
    assert (c.out == c.out[:1]).all() and (c.dq == c.dq[:1]).all() and (c.dk == c.dk[:1]).all() and (c.dv == c.dv[:1]).all() or copies == 1
    n = 1 if copies > 1 else c.out.shape[0]
    windows = one.lse.shape[0]
    R = rpb_bounds.attention(*(np64(x) for x in (one.q, one.k, one.v)), ref.bias_of(np64(one.table), one.index_np), c.heads, c.M, c.s, c.p.scale_c,
                             c.dtype == "bf16", out=np64(c.out[:n]), dout=np64(one.dout), bwd_qkv=bwd_qkv)
    wrong = [rpb_bounds.outside("lse", np64(c.lse[:windows]), R)] + [rpb_bounds.outside(x, np64(getattr(c, x)[:n]), R) for x in ("out", "dq", "dk", "dv")]
    wrong.append(rpb_bounds.outside("dbias", np64(c.dbias), R, copies))
    assert not any(wrong), [x for x in wrong if x]


def run(*a, **kw):
    c = Case(*a, **kw)
    c.forward()
    c.backward()
    check(c)


@pytest.mark.parametrize("dtype,M", itertools.product(("bf16", "f32"), (1, 2, 3, 5, 7, 8, 9, 11, 12, 16, 17, 20, 24)))
def test_window_sides(dtype, M):
    nwy, nwx = (3, 2) if M <= 12 else (1, 2)
    run(dtype, 1, nwy * M, nwx * M, 2, 30, M, M // 2, seed=M)


@pytest.mark.parametrize("dtype,d", itertools.product(("bf16", "f32"), (1, 2, 7, 8, 10, 16, 31, 32, 33, 40, 46, 48, 50, 62, 63, 64)))
def test_head_dims(dtype, d):
    run(dtype, 1, 16, 24, 1 if d % 2 else 2, d, 8, 3, seed=d)
    run(dtype, 1, 16, 16, 1, d, 16, 5, seed=d, packed=True)


@pytest.mark.parametrize("dtype,M,kind", itertools.product(("bf16", "f32"), (7, 16, 18), ("coarse", "near", "past", "none")))
def test_bucket_maps(dtype, M, kind):
    run(dtype, 2, M, 2 * M, 2, 30, M, 1, buckets=kind, packed=True, seed=3)


@pytest.mark.parametrize("dtype,M,d,scale", [("bf16", 7, 30, -0.4), ("bf16", 16, 30, -0.4), ("bf16", 20, 32, 1e-9), ("bf16", 16, 15, 3.0), ("f32", 12, 30, -0.4), ("bf16", 16, 30, 0.0)])
def test_scales(dtype, M, d, scale):
    run(dtype, 1, M, 2 * M, 2, d, M, 1, buckets="past", seed=6, scale=scale)


@pytest.mark.parametrize("dtype,M,d", [("bf16", 32, 30), ("bf16", 40, 30), ("bf16", 37, 20), ("bf16", 32, 15), ("bf16", 48, 33), ("bf16", 64, 16), ("f32", 32, 30), ("f32", 33, 16), ("f32", 48, 40)])
def test_large_windows(dtype, M, d):
    run(dtype, 1, M, M, 1, d, M, M // 3, seed=M)


@pytest.mark.parametrize("dtype,M", [("bf16", 7), ("bf16", 8), ("bf16", 9), ("bf16", 16), ("bf16", 20), ("bf16", 24), ("f32", 5), ("f32", 12), ("f32", 16)])
@pytest.mark.parametrize("flags", [0, rb.RIB_FLAG_FORCE_ROW_MAX])
def test_large_logits(dtype, M, flags):
    """Logits in the hundreds: the walk with a running maximum, and the merge of two halves' maxima on small grids."""
    run(dtype, 1, M, M, 2, 24, M, 0, buckets="past" if M % 2 else "full", seed=5, spread=8.0, scale=1.0, table_std=40.0, flags=flags)


GRIDS = [(7, 2, 30, 100), (9, 2, 30, 100), (11, 2, 16, 100), (13, 1, 32, 180), (16, 2, 30, 100), (16, 1, 15, 180), (18, 1, 34, 100), (20, 1, 30, 100), (24, 1, 30, 60),
         (24, 1, 64, 60), (32, 1, 30, 48), (48, 1, 32, 20)]


@pytest.mark.parametrize("M,heads,d,copies", GRIDS)
@pytest.mark.parametrize("large", [False, True])
def test_large_grids(M, heads, d, copies, large):
    """One to four waves a workgroup, strips and none; with ordinary logits and with those that need the maximum."""
    kw = dict(spread=8.0, scale=1.0, table_std=40.0, buckets="past") if large else {}
    one = Case("bf16", 1, M, M, heads, d, M, 0 if large else M // 2, seed=M, **kw)
    c = repeated(one, copies)
    c.forward()
    c.backward()
    check(c, one, copies)


@pytest.mark.parametrize("dtype,d,M", [("bf16", 30, 7), ("bf16", 30, 16), ("bf16", 15, 12), ("bf16", 40, 24), ("bf16", 64, 16), ("f32", 30, 8), ("f32", 48, 9)])
def test_backward_from_a_checkpoint(dtype, d, M):
    c = Case(dtype, 1, M, 2 * M, 1, d, M, 2, buckets="near", seed=M)
    c.forward()
    ck = packed(c)
    held = [torch.empty_like(c.q) for _ in range(3)]
    rb.rib_checkpoint_unpack(c.p, ck, *held)
    rb.rib_rpb_attn_bwd_ckpt(c.p, ck, c.bias, c.out, c.dout, c.lse, c.dq, c.dk, c.dv, c.dbias, c.ws)
    check(c, bwd_qkv=[np64(x) for x in held])
