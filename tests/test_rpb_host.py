"""The learned relative position bias and the 8-bit checkpoints, host side: refusals, sizes, structures.  No GPU: every call
has to return before anything is launched."""
import ctypes

import numpy as np
import pytest

import rpb_reference as ref
from paper_2603_06738_amd import binding as rb

FAKE = 0x10000          # non-NULL dummy "device pointer", aligned to everything


def good(**kw):
    base = dict(B=2, H=8, W=8, heads=2, d=4, r=0, window=4, shift=1, scale_c=0.5, scale_p=0.0, dtype="f32")
    base.update(kw)
    return rb.make_params(**base)


def fwd(p, **kw):
    a = dict(q=FAKE, k=FAKE, v=FAKE, bias=FAKE, out=FAKE, lse=FAKE)
    a.update(kw)
    return rb.rib_rpb_attn_fwd_status(p, *a.values(), stream=0)


def bwd(p, ws=FAKE, nbytes=1 << 40, **kw):
    a = {n: FAKE for n in ("q", "k", "v", "bias", "out", "d_out", "lse", "dq", "dk", "dv", "dbias")}
    a.update(kw)
    return rb.rib_rpb_attn_bwd_status(p, *a.values(), ws, nbytes, stream=0)


def bwd_ckpt(p, ws=FAKE, nbytes=1 << 40, **kw):
    a = {n: FAKE for n in ("ckpt", "bias", "out", "d_out", "lse", "dq", "dk", "dv", "dbias")}
    a.update(kw)
    return rb.rib_rpb_attn_bwd_ckpt_status(p, *a.values(), ws, nbytes, stream=0)


def test_struct_layout():
    assert ctypes.sizeof(rb.RibRpbParams) == 16 and rb.RibRpbParams.dtype.offset == 12


BAD_SHAPES = [dict(B=0), dict(H=-8), dict(d=0), dict(window=0), dict(H=10), dict(W=6), dict(shift=4), dict(shift=-1), dict(token_stride=7),
              dict(scale_c=float("nan")), dict(scale_c=float("inf"))]


@pytest.mark.parametrize("kw", BAD_SHAPES)
def test_bad_shapes(kw):
    p = good(**kw)
    assert fwd(p) == 2 and bwd(p) == 2 and bwd_ckpt(p) == 2
    assert rb.rib_checkpoint_pack_status(p, FAKE, FAKE, FAKE, FAKE, stream=0) == 2
    assert rb.rib_checkpoint_unpack_status(p, FAKE, FAKE, FAKE, FAKE, stream=0) == 2
    assert rb.rib_rpb_attn_bwd_workspace_bytes(p) == 0 and rb.rib_checkpoint_bytes(p) == 0


def test_bad_types_and_what_is_not_built():
    for call in (fwd, bwd, bwd_ckpt):
        assert call(good(dtype=7)) == 3
        assert call(None) == 1
        for kw in (dict(d=65), dict(r=2), dict(flags=rb.RIB_FLAG_VECTOR_ONLY), dict(flags=rb.RIB_FLAG_WIDE), dict(H=257, W=257, window=257), dict(heads=65536, d=1)):
            assert call(good(**kw)) == 4, kw
    assert fwd(good(flags=64)) == 2
    assert rb.rib_rpb_attn_bwd_workspace_bytes(good(r=2)) == 0
    assert rb.rib_checkpoint_bytes(good(r=2)) > 0                   # (a checkpoint serves the implicit bias too)
    assert rb.rib_checkpoint_bytes(None) == 0 and rb.rib_rpb_attn_bwd_workspace_bytes(None) == 0


@pytest.mark.parametrize("name", ["q", "k", "v", "bias", "out"])
def test_forward_pointers(name):
    assert fwd(good(), **{name: None}) == 1
    assert fwd(good(), **{name: FAKE + 2}) == 2
    assert fwd(good(dtype="bf16"), **{name: FAKE + 1}) == 2
    assert fwd(good(), lse=FAKE + 2) == 2


@pytest.mark.parametrize("name", ["q", "k", "v", "bias", "out", "d_out", "lse", "dq", "dk", "dv"])
def test_backward_pointers(name):
    assert bwd(good(), **{name: None}) == 1
    assert bwd(good(), **{name: FAKE + 2}) == 2
    assert bwd(good(), dbias=FAKE + 2) == 2
    if name not in "qkv":
        assert bwd_ckpt(good(), **{name: None}) == 1
    assert bwd_ckpt(good(), ckpt=None) == 1 and bwd_ckpt(good(), ckpt=FAKE + 8) == 2


def test_workspace():
    p = good()
    n = rb.rib_rpb_attn_bwd_workspace_bytes(p)
    assert n > 0 and n % 256 == 0
    for call in (bwd, bwd_ckpt):
        assert call(p, ws=None) == 5 and call(p, ws=FAKE + 128) == 5 and call(p, nbytes=n - 1) == 5


def test_table_refusals():
    tp = rb.make_rpb_params(4, 2, 49, "f32")
    for kw in (dict(window=0), dict(window=257), dict(heads=0), dict(heads=65536), dict(buckets=0), dict(buckets=(1 << 24) + 1)):
        bad = rb.make_rpb_params(**{**dict(window=4, heads=2, buckets=49), **kw})
        assert rb.rib_rpb_table_fwd_status(bad, FAKE, FAKE, FAKE, stream=0) == 2
        assert rb.rib_rpb_table_bwd_status(bad, FAKE, FAKE, FAKE, stream=0) == 2
    assert rb.rib_rpb_table_fwd_status(rb.make_rpb_params(4, 2, 49, 9), FAKE, FAKE, FAKE, stream=0) == 3
    assert rb.rib_rpb_table_fwd_status(None, FAKE, FAKE, FAKE, stream=0) == 1
    for i in range(3):
        for value, status in ((None, 1), (FAKE + 2, 2)):
            a = [FAKE] * 3
            a[i] = value
            assert rb.rib_rpb_table_fwd_status(tp, *a, stream=0) == status
            assert rb.rib_rpb_table_bwd_status(tp, *a, stream=0) == status


@pytest.mark.parametrize("i", range(4))
def test_checkpoint_pointers(i):
    for call in (rb.rib_checkpoint_pack_status, rb.rib_checkpoint_unpack_status):
        a = [FAKE] * 4
        a[i] = None
        assert call(good(), *a, stream=0) == 1
        a[i] = FAKE + 2
        assert call(good(), *a, stream=0) == 2
    assert rb.rib_checkpoint_pack_status(None, FAKE, FAKE, FAKE, FAKE, stream=0) == 1


@pytest.mark.parametrize("d,dp", [(1, 16), (16, 16), (30, 32), (33, 48), (64, 64)])
def test_checkpoint_size(d, dp):
    assert rb.rib_checkpoint_bytes(good(d=d)) == 3 * (2 * 4 * 2) * 16 * (dp + 1)         # windows * heads, tokens, row and exponent


def test_calls_raise():
    with pytest.raises(rb.RibError):
        rb.rib_rpb_attn_fwd(good(r=2), FAKE, FAKE, FAKE, FAKE, FAKE, None, stream=0)
    with pytest.raises(rb.RibError):
        rb.rib_checkpoint_pack(good(H=10), FAKE, FAKE, FAKE, FAKE, stream=0)


# ---- the reference itself --------------------------------------------------------------------------------------------


@pytest.mark.parametrize("kind", ["full", "coarse", "past", "near"])
def test_reference_gradients_are_differences(kind):
    """Central differences of the reference's forward: every gradient, the table's too.  An error of h^2 = 1e-10 times third derivatives of
    order 10, and of 1e-16 / h from rounding: 1e-7 holds both."""
    rng = np.random.default_rng(0)
    B, H, W, heads, d, M, s, scale = 1, 4, 8, 2, 3, 4, 1, 0.7
    q, k, v, do = (rng.standard_normal((B, H, W, heads * d)) for _ in range(4))
    index, nb = ref.bucket_index(kind, M)
    table = rng.standard_normal((heads, nb))

    def forward(a):
        return ref.attention(a[0], a[1], a[2], ref.bias_of(a[3], index), heads, M, s, scale, 2.0 ** -24)

    args = [q, k, v, table]
    out = forward(args).out
    R = ref.attention(q, k, v, ref.bias_of(table, index), heads, M, s, scale, 2.0 ** -24, out=out, dout=do)
    for j, grad in enumerate((R.dq, R.dk, R.dv, ref.table_grad(R.dbias, index, nb))):
        for _ in range(6):
            at = tuple(rng.integers(n) for n in args[j].shape)
            total = []
            for h in (1e-5, -1e-5):
                a = list(args)
                a[j] = a[j].copy()
                a[j][at] += h
                total.append((forward(a).out * do).sum())
            assert abs((total[0] - total[1]) / 2e-5 - grad[at]) < 1e-7


def test_reference_equals_softmax_of_a_materialised_bias():
    """One window, one head, against numpy's own steps on explicit N x N arrays."""
    rng = np.random.default_rng(1)
    M, d = 3, 5
    q, k, v = (rng.standard_normal((1, M, M, d)) for _ in range(3))
    table = rng.standard_normal((1, (2 * M - 1) ** 2))
    index = np.arange((2 * M - 1) ** 2).astype(np.int32)
    bias = np.zeros((M * M, M * M))
    for i, j in np.ndindex(M * M, M * M):
        bias[i, j] = table[0, (i // M - j // M + M - 1) * (2 * M - 1) + i % M - j % M + M - 1]
    S = 0.3 * q.reshape(-1, d) @ k.reshape(-1, d).T + bias
    P = np.exp(S) / np.exp(S).sum(1, keepdims=True)
    R = ref.attention(q, k, v, ref.bias_of(table, index), 1, M, 0, 0.3, 2.0 ** -24)
    assert np.allclose(R.out.reshape(-1, d), P @ v.reshape(-1, d), atol=1e-12) and np.allclose(R.lse[0, 0], np.log(np.exp(S).sum(1)), atol=1e-12)


def test_reference_codes():
    """Half a step is the most that a value moves; packing what a checkpoint stands for changes nothing."""
    rng = np.random.default_rng(2)
    x = rng.standard_normal((1, 4, 4, 10)) * 10.0 ** rng.integers(-6, 6, (1, 4, 4, 1))
    x[0, 0, 0, :5] = 0
    codes, exps = ref.pack(x, 2, 2, 1)
    y = ref.unpack(codes, exps, x.shape, 2, 2, 1)
    big = np.abs(x).reshape(1, 4, 4, 2, 5).max(-1, keepdims=True).repeat(5, -1).reshape(x.shape)
    assert (np.abs(x - y) <= big / 127).all()           # (a step is at most 2 / 127 of the largest)
    again = ref.pack(y, 2, 2, 1)
    assert (again[0] == codes).all() and (again[1] == exps).all()
