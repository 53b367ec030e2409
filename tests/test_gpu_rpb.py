"""Window attention with a learned relative position bias on the GPU, every element of every result against the plain
64-bit form, within bounds that follow from the kernels' roundings (tests/rpb_reference.py)."""
import itertools

import numpy as np
import pytest
import torch

import rpb_reference as ref
from paper_2603_06738_amd import binding as rb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def storage(x, dtype):
    t = torch.from_numpy(np.ascontiguousarray(x)).float()
    return t.to(torch.bfloat16) if dtype == "bf16" else t


class Case:
    """Tensors of one call on the GPU, and their values in 64 bits."""

    def __init__(self, dtype, B, H, W, heads, d, M, s, buckets="full", packed=False, scale=None, seed=0, spread=1.0, table_std=0.5,
                 flags=0):
        rng = np.random.default_rng(seed)
        self.dtype, self.B, self.H, self.W, self.heads, self.d, self.M, self.s = dtype, B, H, W, heads, d, M, s
        self.scale = d ** -0.5 if scale is None else scale
        self.C, self.N = heads * d, M * M
        self.u = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
        self.td = torch.bfloat16 if dtype == "bf16" else torch.float32
        qkv = storage(rng.standard_normal((B, H, W, 3 * self.C)) * spread, dtype)
        self.qkv = qkv.to(DEV)
        parts = [self.qkv[..., i * self.C:(i + 1) * self.C] for i in range(3)]
        self.q, self.k, self.v = parts if packed else [x.contiguous() for x in parts]
        self.dout = storage(rng.standard_normal((B, H, W, self.C)), dtype).to(DEV)
        self.index_np, self.nb = ref.bucket_index(buckets, M)
        self.table = storage(rng.standard_normal((heads, self.nb)) * table_std, dtype).to(DEV)
        self.index = torch.from_numpy(self.index_np).to(DEV)
        self.p = rb.make_params(B, H, W, heads, d, 0, M, s, self.scale, 0.0, dtype, flags=flags, token_stride=3 * self.C if packed else 0)
        self.tp = rb.make_rpb_params(M, heads, self.nb, dtype)
        L, nw = (2 * M - 1) ** 2, B * (H // M) * (W // M)
        f32 = torch.float32
        self.bias, self.dbias = self.nan(heads, L, dtype=f32), self.nan(heads, L, dtype=f32)
        self.lse = self.nan(nw, heads, self.N, dtype=f32)
        self.out, self.dq, self.dk, self.dv = (self.nan(B, H, W, self.C) for _ in range(4))
        self.dtable = self.nan(heads, self.nb)
        self.ws = torch.full((max(rb.rib_rpb_attn_bwd_workspace_bytes(self.p), 256),), 0xff, dtype=torch.uint8, device=DEV)

    def nan(self, *shape, dtype=None):
        return torch.full(shape, float("nan"), dtype=dtype or self.td, device=DEV)

    def forward(self):
        rb.rib_rpb_table_fwd(self.tp, self.table, self.index, self.bias)
        rb.rib_rpb_attn_fwd(self.p, self.q, self.k, self.v, self.bias, self.out, self.lse)

    def backward(self):
        rb.rib_rpb_attn_bwd(self.p, self.q, self.k, self.v, self.bias, self.out, self.dout, self.lse, self.dq, self.dk, self.dv,
                            self.dbias, self.ws)
        rb.rib_rpb_table_bwd(self.tp, self.dbias, self.index, self.dtable)

    def reference(self, backward=True, bwd_qkv=None):
        g = [np64(x) for x in (self.q, self.k, self.v)]
        bias = ref.bias_of(np64(self.table), self.index_np)
        kw = dict(out=np64(self.out), dout=np64(self.dout), bwd_qkv=bwd_qkv) if backward else {}
        return ref.attention(*g, bias, self.heads, self.M, self.s, self.scale, self.u, **kw)


def np64(t):
    return t.detach().double().cpu().numpy()


def close(name, got, want, tol):
    got = np64(got)
    inf = np.isinf(want)
    assert np.array_equal(got[inf], want[inf]), name
    off = np.abs(np.where(inf, 0, got - np.where(inf, 0, want)))
    assert not np.isnan(off).any(), f"{name}: NaN"
    worst = np.unravel_index(np.argmax(off - tol), off.shape)
    assert (off <= tol).all(), f"{name} at {worst}: {got[worst]} for {want[worst]}, {off[worst]:.3g} off, {tol[worst]:.3g} allowed"


def check(c, R, backward=True):
    close("lse", c.lse, R.lse, R.lse_tol)
    close("out", c.out, R.out, R.out_tol)
    if not backward:
        return
    for n in ("dq", "dk", "dv", "dbias"):
        close(n, getattr(c, n), getattr(R, n), getattr(R, n + "_tol"))
    want = ref.table_grad(R.dbias, c.index_np, c.nb)
    # a bucket's sum is of whole multiples of a unit: the power of two above the head's largest over 2^(62 - bits of L), so of at most
    # 2^(bits - 61) of the largest; every term is half a unit off at most
    L = (2 * c.M - 1) ** 2
    unit = 2.0 ** (max(1, int(np.ceil(np.log2(L)))) - 61) * np.abs(np64(c.dbias)).max(1, keepdims=True)
    terms = np.bincount(c.index_np[(c.index_np >= 0) & (c.index_np < c.nb)], minlength=c.nb)
    close("dtable", c.dtable, want, ref.table_grad(R.dbias_tol, c.index_np, c.nb) + 0.5 * terms * unit + c.u * np.abs(want) + 1e-30)


def run(*a, **kw):
    c = Case(*a, **kw)
    c.forward()
    c.backward()
    check(c, c.reference())
    return c


# window sides over every tile edge: a single token, partial tiles, one wave, whole tiles, several workgroups
SIDES = [1, 2, 3, 5, 6, 7, 8, 9, 11, 12, 16, 17, 20, 24]


@pytest.mark.parametrize("dtype,M", itertools.product(("bf16", "f32"), SIDES))
def test_window_sides(dtype, M):
    nwy, nwx = (3, 2) if M <= 12 else (1, 2)
    run(dtype, 1, nwy * M, nwx * M, 2, 30, M, M // 2, seed=M)


@pytest.mark.parametrize("dtype,d", itertools.product(("bf16", "f32"), (1, 2, 3, 7, 8, 10, 15, 16, 31, 32, 33, 34, 46, 47, 48, 62, 63, 64)))
def test_head_dims(dtype, d):
    run(dtype, 1, 16, 24, 1 if d % 2 else 2, d, 8, 3, seed=d)
    run(dtype, 1, 18, 9, 1, d, 9, 0, seed=d, packed=True)
    if d in (7, 15, 30, 47, 64):
        run(dtype, 1, 16, 16, 1, d, 16, 5, seed=d)


@pytest.mark.parametrize("dtype,M,kind", itertools.product(("bf16", "f32"), (4, 7, 16, 18), ("coarse", "near", "past", "none", "one")))
def test_bucket_maps(dtype, M, kind):
    c = run(dtype, 2, M, 2 * M, 3, 30, M, 1, buckets=kind, packed=True, seed=3)
    if kind == "past":
        assert torch.isinf(c.lse[:, :, 0]).all()
    if kind == "none":
        assert (c.out == 0).all() and (c.dq == 0).all() and (c.dk == 0).all() and (c.dv == 0).all() and (c.dbias == 0).all()


@pytest.mark.parametrize("dtype,M,heads,d", [("bf16", 32, 2, 30), ("bf16", 40, 1, 30), ("bf16", 48, 1, 32), ("bf16", 64, 1, 16), ("bf16", 37, 1, 20),
                                             ("bf16", 32, 1, 15), ("bf16", 48, 1, 33), ("bf16", 96, 1, 8),
                                             ("f32", 32, 1, 30), ("f32", 33, 1, 16), ("f32", 48, 1, 40), ("f32", 64, 1, 16)])
def test_large_windows(dtype, M, heads, d):
    """Several workgroups a unit; bias rows and sums in chunks of the walk."""
    run(dtype, 1, M, M, heads, d, M, M // 3, seed=M)


def repeated(c, copies):
    """A case of one image, as `copies` of it: what large grids run on, for the price of one reference."""
    big = Case.__new__(Case)
    big.__dict__.update(c.__dict__)
    big.B = copies
    big.qkv = c.qkv.repeat(copies, 1, 1, 1)
    big.q, big.k, big.v = (big.qkv[..., i * c.C:(i + 1) * c.C].contiguous() for i in range(3))
    big.dout = c.dout.repeat(copies, 1, 1, 1)
    big.p = rb.make_params(copies, c.H, c.W, c.heads, c.d, 0, c.M, c.s, c.scale, 0.0, c.dtype)
    big.lse = big.nan(copies * (c.H // c.M) * (c.W // c.M), c.heads, c.N, dtype=torch.float32)
    big.out, big.dq, big.dk, big.dv = (big.nan(copies, c.H, c.W, c.C) for _ in range(4))
    big.dbias = torch.full_like(c.dbias, float("nan"))
    big.ws = torch.full((rb.rib_rpb_attn_bwd_workspace_bytes(big.p),), 0xff, dtype=torch.uint8, device=DEV)
    return big


# grids beyond the split of small ones: one, two, three and four waves a workgroup, strips of 8, 16 and 32 columns and none
@pytest.mark.parametrize("M,heads,d,copies", [(7, 2, 30, 100), (9, 2, 30, 100), (11, 2, 16, 100), (13, 1, 32, 180), (16, 2, 30, 100), (16, 1, 15, 180),
                                              (18, 1, 34, 100), (20, 1, 30, 100), (24, 1, 30, 60), (24, 1, 64, 60), (32, 1, 30, 48), (48, 1, 32, 20),
                                              (64, 1, 16, 12)])
def test_large_grids(M, heads, d, copies):
    one = Case("bf16", 1, M, M, heads, d, M, M // 2, seed=M)
    c = repeated(one, copies)
    c.forward()
    c.backward()
    one.out = c.out[:1].contiguous()
    R = one.reference()
    for n in ("out", "dq", "dk", "dv"):
        x = getattr(c, n)
        assert torch.equal(x, x[:1].expand_as(x)), n            # every image alike
        close(n, x[:1], getattr(R, n), getattr(R, n + "_tol"))
    close("lse", c.lse[:1], R.lse, R.lse_tol)
    close("dbias", c.dbias, copies * R.dbias, copies * R.dbias_tol + copies * 2.0 ** -24 * copies * np.abs(R.dbias))


@pytest.mark.parametrize("dtype,M,copies", [("bf16", 7, 1), ("bf16", 16, 1), ("bf16", 16, 200), ("bf16", 24, 60), ("f32", 9, 1)])
def test_runs_are_identical(dtype, M, copies):
    c = Case(dtype, 1, M, M, 2, 30, M, 1, buckets="coarse", seed=2)
    if copies > 1:
        c = repeated(c, copies)
    got = []
    for _ in range(3):
        c.ws.fill_(0xff)
        c.forward()
        c.backward()
        got.append([getattr(c, n).clone() for n in ("out", "lse", "dq", "dk", "dv", "dbias", "dtable")])
    for other in got[1:]:
        for a, b in zip(got[0], other):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype,M", [("bf16", 7), ("bf16", 16), ("bf16", 20), ("f32", 12)])
def test_forced_row_maximum(dtype, M):
    a = Case(dtype, 1, M, 2 * M, 2, 30, M, 1, buckets="past", seed=4, flags=rb.RIB_FLAG_FORCE_ROW_MAX)
    a.forward()
    a.backward()
    check(a, a.reference())


@pytest.mark.parametrize("dtype,M", [("bf16", 7), ("bf16", 16), ("bf16", 20), ("f32", 12)])
def test_large_logits_need_the_row_maximum(dtype, M):
    """Logits in the hundreds: exp2 of them overflows without a maximum; the bounds grow with them by themselves."""
    run(dtype, 1, M, M, 2, 24, M, 0, seed=5, spread=8.0, scale=1.0, table_std=40.0)


@pytest.mark.parametrize("dtype,scale", [("bf16", 0.0), ("bf16", -0.4), ("bf16", 1e-20), ("f32", 0.0), ("f32", -0.4)])
def test_scales_that_are_no_ordinary_number(dtype, scale):
    for M in (6, 16):
        run(dtype, 1, M, M, 2, 16, M, 1, buckets="past", seed=6, scale=scale)


def test_no_lse_and_no_dbias():
    for dtype, M in itertools.product(("bf16", "f32"), (7, 16, 18)):
        c = Case(dtype, 1, M, M, 2, 30, M, 1, seed=7)
        c.forward()
        c.backward()
        out = torch.full_like(c.out, float("nan"))
        rb.rib_rpb_attn_fwd(c.p, c.q, c.k, c.v, c.bias, out)
        assert torch.equal(out, c.out)
        dq, dk, dv = (torch.full_like(c.dq, float("nan")) for _ in range(3))
        rb.rib_rpb_attn_bwd(c.p, c.q, c.k, c.v, c.bias, c.out, c.dout, c.lse, dq, dk, dv, None, c.ws)
        assert torch.equal(dq, c.dq) and torch.equal(dk, c.dk) and torch.equal(dv, c.dv)


@pytest.mark.parametrize("low", [-np.inf, -3.3895313892515355e38, -1e30])
def test_lowest_values_exclude(low):
    """A table at a type's lowest value (bf16's here, which fp32 has too), at -1e30 or at minus infinity excludes; -100 does not."""
    for dtype in ("bf16", "f32"):
        c = Case(dtype, 1, 8, 16, 2, 16, 8, 3, seed=8)
        table = c.table.clone()
        table[:, ::2] = low
        table[:, 1] = -100.0
        c.table = table
        c.forward()
        c.backward()
        check(c, c.reference())
        row = torch.full_like(c.bias, float(np.float32(low)))
        rb.rib_rpb_attn_fwd(c.p, c.q, c.k, c.v, row, c.out, c.lse)      # every row empty, straight from the caller's own bias
        assert (c.out == 0).all() and torch.isneginf(c.lse).all()


def test_not_finite_stays_in_its_window():
    """An infinity in one window's keys: other windows and heads as they were."""
    for dtype, M in (("bf16", 7), ("bf16", 16), ("f32", 9)):
        c = Case(dtype, 1, M, 3 * M, 2, 16, M, 0, seed=9)
        c.forward()
        c.backward()
        before = [x.clone() for x in (c.out, c.dq, c.dk, c.dv)]
        c.k[0, 1, M + 1, 3] = float("inf")          # window 1, head 0
        c.forward()
        c.backward()
        for a, b in zip(before, (c.out, c.dq, c.dk, c.dv)):
            assert torch.equal(a[:, :, :M], b[:, :, :M]) and torch.equal(a[:, :, 2 * M:], b[:, :, 2 * M:])
            assert torch.equal(a[..., 16:], b[..., 16:])
        assert torch.isnan(c.out[0, :, M:2 * M, :16].float()).any()


def test_table_sums_of_values_that_are_not_finite():
    M, heads, nb = 5, 2, 7
    tp = rb.make_rpb_params(M, heads, nb)
    rng = np.random.default_rng(1)
    index = torch.from_numpy(rng.integers(-2, nb + 2, 81).astype(np.int32)).to(DEV)
    db = torch.from_numpy(rng.standard_normal((heads, 81)).astype(np.float32) * 10.0 ** rng.integers(-20, 20, (heads, 1))).float().to(DEV)
    got = torch.empty(heads, nb, device=DEV)
    rb.rib_rpb_table_bwd(tp, db, index, got)
    want = ref.table_grad(np64(db), index.cpu().numpy(), nb)
    # 2^-45 of the head's largest a term (81 terms), and fp32's rounding
    assert (np.abs(np64(got) - want) <= 81 * 2.0 ** -45 * np.abs(np64(db)).max(1, keepdims=True) + 2.0 ** -24 * np.abs(want)).all()
    where = [int((index == b).nonzero()[0]) for b in (0, 1, 2, 3)]
    other = int((index == 3).nonzero()[-1])
    db[0, where[0]], db[0, where[1]], db[0, where[2]], db[0, where[3]] = float("inf"), float("-inf"), float("nan"), float("inf")
    db[0, other] = float("-inf") if other != where[3] else float("nan")
    rb.rib_rpb_table_bwd(tp, db, index, got)
    g = np64(got)
    assert g[0, 0] == np.inf and g[0, 1] == -np.inf and np.isnan(g[0, 2]) and np.isnan(g[0, 3])
    assert np.isfinite(g[0, 4:]).all() and np.isfinite(g[1]).all()
    db.zero_()
    rb.rib_rpb_table_bwd(tp, db, index, got)
    assert (got == 0).all()


# ---- checkpoints -----------------------------------------------------------------------------------------------------


def packed(c):
    ck = torch.full((rb.rib_checkpoint_bytes(c.p),), 0xff, dtype=torch.uint8, device=DEV)
    rb.rib_checkpoint_pack(c.p, c.q, c.k, c.v, ck)
    return ck


@pytest.mark.parametrize("dtype,d,M,stride", [("bf16", 30, 6, False), ("bf16", 7, 5, True), ("bf16", 64, 8, True), ("bf16", 16, 1, False), ("f32", 30, 7, True),
                                              ("f32", 33, 4, False)])
def test_checkpoint_codes(dtype, d, M, stride):
    """Every code and exponent byte as the format says; rows of zeros, of tiny, huge and not finite values among them."""
    c = Case(dtype, 2, 2 * M, M, 3, d, M, M // 2, packed=stride, seed=d)
    for x, n in ((c.q, 0), (c.k, 1), (c.v, 2)):
        x[0, 0, 0, :d] = 0
        x[0, M, 0, :d] *= 2.0 ** -120
        x[1, 0, 0, :d] *= 2.0 ** 100
        x[1, 1 % (2 * M), 0, d:2 * d] = 127.0          # the largest that a step of one holds
        x[0, 2 % (2 * M), 0, n] = float("nan") if n else float("inf")
    ck = packed(c).cpu().numpy()
    dp = (d + 15) // 16 * 16
    rows = 2 * 2 * 3 * M * M
    for i, x in enumerate((c.q, c.k, c.v)):
        codes, exps = ref.pack(np64(x), 3, M, M // 2)
        assert np.array_equal(ck[3 * rows * dp + i * rows:3 * rows * dp + (i + 1) * rows], exps.reshape(-1))
        assert np.array_equal(ck[i * rows * dp:(i + 1) * rows * dp], codes.reshape(-1))
    back = [torch.full_like(x, 3.0) for x in (c.qkv, c.qkv, c.qkv)] if stride else [torch.full_like(c.q, 3.0) for _ in range(3)]
    views = [b[..., i * c.C:(i + 1) * c.C] for i, b in enumerate(back)] if stride else back
    rb.rib_checkpoint_unpack(c.p, torch.from_numpy(ck).to(DEV), *views)
    for i, x in enumerate((c.q, c.k, c.v)):
        want = ref.unpack(*ref.pack(np64(x), 3, M, M // 2), tuple(x.shape), 3, M, M // 2)
        assert np.array_equal(np64(views[i]), want, equal_nan=True)
        if stride:
            rest = [back[i][..., j * c.C:(j + 1) * c.C] for j in range(3) if j != i]
            assert all((r == 3).all() for r in rest)            # nothing between the tokens is touched


@pytest.mark.parametrize("dtype,d,M,copies", [("bf16", 30, 7, 1), ("bf16", 30, 16, 1), ("bf16", 30, 16, 200), ("bf16", 32, 9, 200), ("bf16", 15, 12, 1), ("bf16", 40, 24, 1),
                                              ("bf16", 64, 6, 1), ("bf16", 62, 16, 180), ("f32", 30, 8, 1), ("f32", 48, 9, 1)])
def test_backward_from_a_checkpoint(dtype, d, M, copies):
    """Bit for bit what the backward gives for the unpacked tensors, and within bounds of the plain form."""
    c = Case(dtype, 1, M, M, 1, d, M, 2 % M, buckets="near", seed=M)
    if copies > 1:
        c = repeated(c, copies)
    c.forward()
    ck = packed(c)
    q, k, v = c.q, c.k, c.v
    c.q, c.k, c.v = (torch.empty_like(q) for _ in range(3))
    rb.rib_checkpoint_unpack(c.p, ck, c.q, c.k, c.v)
    c.backward()
    plain = [getattr(c, n).clone() for n in ("dq", "dk", "dv", "dbias")]
    for n in ("dq", "dk", "dv", "dbias"):
        getattr(c, n).fill_(float("nan"))
    c.ws.fill_(0xff)
    rb.rib_rpb_attn_bwd_ckpt(c.p, ck, c.bias, c.out, c.dout, c.lse, c.dq, c.dk, c.dv, c.dbias, c.ws)
    for n, x in zip(("dq", "dk", "dv", "dbias"), plain):
        assert torch.equal(getattr(c, n), x), n
    if copies == 1:
        held = [np64(x) for x in (c.q, c.k, c.v)]
        c.q, c.k, c.v = q, k, v
        R = c.reference(bwd_qkv=held)
        for n in ("dq", "dk", "dv", "dbias"):
            close(n, getattr(c, n), getattr(R, n), getattr(R, n + "_tol"))


def test_checkpoint_of_a_step_with_the_implicit_bias():
    """The other attention's backward takes what a checkpoint stands for: gradients near those of the tensors themselves.  A value moves by
    at most 1 / 127 of its row's largest, so a logit of 30 products by under 30 * 2 * 3.5 * (3.5 / 127) * scale = 1.06, in earnest by a
    hundredth of that; the gradients' 2-norm is held to a tenth."""
    rng = np.random.default_rng(3)
    B, H, W, heads, d, r, M = 1, 32, 32, 2, 30, 16, 16
    t = [storage(rng.standard_normal((B, H, W, heads * d)), "bf16").to(DEV) for _ in range(4)]
    f = [storage(rng.standard_normal((heads, M * M, r)) * 0.5, "bf16").to(DEV) for _ in range(2)]
    p = rb.make_params(B, H, W, heads, d, r, M, 4, d ** -0.5, r ** -0.5, "bf16")
    out, lse = torch.empty_like(t[0]), torch.empty(4, heads, M * M, device=DEV)
    rb.rib_window_attn_fwd(p, *t[:3], *f, out, lse)
    ck = torch.empty(rb.rib_checkpoint_bytes(p), dtype=torch.uint8, device=DEV)
    rb.rib_checkpoint_pack(p, *t[:3], ck)
    held = [torch.empty_like(t[0]) for _ in range(3)]
    rb.rib_checkpoint_unpack(p, ck, *held)
    ws = rb.alloc_workspace(p)
    grads = []
    for qkv in (t[:3], held):
        g = [torch.empty_like(t[0]) for _ in range(3)] + [torch.empty(heads, M * M, r, device=DEV) for _ in range(2)]
        rb.rib_window_attn_bwd(p, *qkv, *f, out, t[3], lse, *g, ws)
        grads.append(g)
    for a, b in zip(*grads):
        assert (a - b).float().norm() <= 0.1 * a.float().norm()


# ---- streams, graphs, strides ----------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype,M", [("bf16", 7), ("bf16", 16), ("f32", 12)])
def test_captured_step(dtype, M):
    """A whole step recorded into a graph, replayed with other inputs and eager work between the replays; two graphs share the workspace."""
    c = Case(dtype, 1, 2 * M, M, 2, 30, M, 1, seed=11)
    ck = torch.empty(rb.rib_checkpoint_bytes(c.p), dtype=torch.uint8, device=DEV)
    names = ("out", "lse", "dq", "dk", "dv", "dbias", "dtable")

    def step(eight):
        c.forward()
        if not eight:
            return c.backward()
        rb.rib_checkpoint_pack(c.p, c.q, c.k, c.v, ck)
        rb.rib_rpb_attn_bwd_ckpt(c.p, ck, c.bias, c.out, c.dout, c.lse, c.dq, c.dk, c.dv, c.dbias, c.ws)
        rb.rib_rpb_table_bwd(c.tp, c.dbias, c.index, c.dtable)

    step(False), step(True)
    torch.cuda.synchronize()
    graphs = []
    for eight in (False, True):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(eight)
        graphs.append(g)
    gen = torch.Generator(device=DEV).manual_seed(1)
    for turn in range(4):
        for x in (c.q, c.k, c.v, c.dout):
            x.copy_(torch.randn(x.shape, generator=gen, device=DEV))
        for eight in (False, True):
            step(eight)
            torch.cuda.synchronize()
            want = [getattr(c, n).clone() for n in names]
            for n in names:
                getattr(c, n).fill_(float("nan"))
            graphs[eight].replay()
            torch.cuda.synchronize()
            for n, x in zip(names, want):
                assert torch.equal(getattr(c, n), x), (turn, eight, n)


def test_two_streams():
    """Two steps at once on streams of their own, each with its workspace, as each alone."""
    cases = [Case("bf16", 2, 32, 32, 2, 30, 16, 3, seed=12), Case("bf16", 2, 28, 14, 2, 32, 7, 0, seed=13)]
    want = []
    for c in cases:
        c.forward(), c.backward()
        want.append([getattr(c, n).clone() for n in ("out", "dq", "dk", "dv", "dtable")])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for c, s in zip(cases, streams):
            with torch.cuda.stream(s):
                c.forward(), c.backward()
    torch.cuda.synchronize()
    for c, w in zip(cases, want):
        for n, x in zip(("out", "dq", "dk", "dv", "dtable"), w):
            assert torch.equal(getattr(c, n), x)


@pytest.mark.parametrize("dtype,shift", [("bf16", 1), ("bf16", 2), ("f32", 1)])
def test_tensors_off_their_usual_boundaries(dtype, shift):
    """q, k, v, outputs and gradients that begin one or two values into an allocation, an odd token stride: same results."""
    a = Case(dtype, 1, 16, 16, 1, 30, 16, 3, seed=14)
    a.forward(), a.backward()
    b = Case(dtype, 1, 16, 16, 1, 30, 16, 3, seed=14)
    stride = 97 if shift == 1 else 98

    def off(x, dense):
        n = x.numel() if dense else 256 * stride
        flat = torch.full((n + 8,), 7.0, dtype=b.td, device=DEV)
        view = flat[shift:shift + x.numel()].view(x.shape) if dense else \
            flat.as_strided((1, 16, 16, 30), (256 * stride, 16 * stride, stride, 1), shift)
        view.copy_(x)
        return flat, view

    keep = []
    for n in ("q", "k", "v"):
        flat, view = off(getattr(b, n), False)
        keep.append(flat)
        setattr(b, n, view)
    guards = []
    for n in ("out", "dout", "dq", "dk", "dv"):
        flat, view = off(getattr(b, n), True)
        guards.append((flat, view.numel()))
        setattr(b, n, view)
    b.p = rb.make_params(1, 16, 16, 1, 30, 0, 16, 3, b.scale, 0.0, dtype, token_stride=stride)
    b.ws = torch.empty(rb.rib_rpb_attn_bwd_workspace_bytes(b.p), dtype=torch.uint8, device=DEV)
    b.forward(), b.backward()
    check(b, b.reference())
    for flat, n in guards:
        assert (flat[:shift] == 7).all() and (flat[shift + n:] == 7).all()      # nothing before or behind a tensor is touched


@pytest.mark.parametrize("M,heads,copies,buckets", [(9, 2, 100, "full"), (11, 2, 100, "past"), (16, 2, 100, "past"), (18, 1, 100, "full"), (20, 1, 100, "past"), (24, 1, 60, "past"),
                                                    (32, 1, 48, "full")])
def test_large_grids_with_the_row_maximum(M, heads, copies, buckets):
    """Logits in the hundreds on the kernels of large grids: the second walk, and rows without a key beside it."""
    one = Case("bf16", 1, M, M, heads, 24, M, 0, buckets=buckets, seed=M, spread=8.0, scale=1.0, table_std=40.0)
    c = repeated(one, copies)
    c.forward()
    c.backward()
    one.out = c.out[:1].contiguous()
    R = one.reference()
    close("lse", c.lse[:1], R.lse, R.lse_tol)
    for n in ("out", "dq", "dk", "dv"):
        x = getattr(c, n)
        assert torch.equal(x, x[:1].expand_as(x)), n
        close(n, x[:1], getattr(R, n), getattr(R, n + "_tol"))
