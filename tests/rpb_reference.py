"""Window attention with a learned relative position bias and the 8-bit checkpoint format, plainly, in 64 bits on the CPU,
with bounds on what a kernel's rounding may change.

Everything is written from global pixel coordinates, one (window, head) at a time; nothing is shared with the kernels.
Bounds are per element: every input of a sum moves by its own relative error, so a sum moves by at most the sum of
|term| times that error.  u is half a step of the operands' type: bf16 2^-8, fp32 2^-24.

    Q times scale is rounded once           a logit moves by at most eps_ij = u * scale * sum_c |q_ic k_jc|
    P = exp(S - LSE), LSE of those logits   a probability by at most 2 max_j eps_ij (S by one, LSE by one), relative, and by u: LSE's
                                            denominator adds up probabilities as rounded, log sum p (1 + t) with |t| <= u
    P and dS are rounded for the products   u more; Q's own rounding enters dK once more; outputs are rounded: u
    bf16 keeps -LSE and -delta as two parts 2^-16 of each
    fp32 sums of n terms                    n 2^-24
"""
import numpy as np


def bucket_index(kind, M, rng=None):
    """[(2M-1)^2] int32, number of buckets."""
    n = 2 * M - 1
    dy, dx = np.meshgrid(np.arange(n) - (M - 1), np.arange(n) - (M - 1), indexing="ij")
    index = np.arange(n * n).reshape(n, n)
    nb = n * n
    if kind == "coarse":
        index = (np.abs(dy) // 2) * (M // 2 + 1) + np.abs(dx) // 2
        nb = (M // 2 + 1) ** 2
    elif kind == "near":
        index = np.where(dy * dy + dx * dx <= (M / 2) ** 2, index, -1)
    elif kind == "past":
        index = np.where((dy > 0) | ((dy == 0) & (dx > 0)), index, -1)
    elif kind == "none":
        index = np.where(index % 2 == 0, -5, nb + 7)
    elif kind == "one":
        index, nb = np.zeros_like(index), 1
    elif kind != "full":
        raise ValueError(kind)
    return np.ascontiguousarray(index.reshape(-1).astype(np.int32)), nb


def bias_of(table, index):
    """[heads][L] from [heads][buckets]."""
    L, nb = len(index), table.shape[1]
    bias = np.full((table.shape[0], L), -np.inf)
    for o in range(L):
        if 0 <= index[o] < nb:
            bias[:, o] = table[:, index[o]]
    bias[bias <= -1e30] = -np.inf
    return bias


def table_grad(dbias, index, nb):
    grad = np.zeros((dbias.shape[0], nb))
    for o in range(len(index)):
        if 0 <= index[o] < nb:
            grad[:, index[o]] += dbias[:, o]
    return grad


def pixels(H, W, M, s, wy, wx):
    iy, ix = np.divmod(np.arange(M * M), M)
    return (wy * M + iy + s) % H, (wx * M + ix + s) % W


def offsets(M):
    iy, ix = np.divmod(np.arange(M * M), M)
    return (iy[:, None] - iy[None, :] + M - 1) * (2 * M - 1) + ix[:, None] - ix[None, :] + M - 1


class Result:
    pass


def attention(q, k, v, bias, heads, M, s, scale, u, out=None, dout=None, bwd_qkv=None):
    """q, k, v [B][H][W][C] float64 (storage values), bias [heads][L].  With `dout`: gradients too, delta from `out` (storage
    values; the kernel's own, as a caller has it), probabilities from `bwd_qkv` (default: q, k, v) and the forward's LSE.
    Returns values and bounds (names with _tol)."""
    B, H, W, C = q.shape
    d, N = C // heads, M * M
    wide = u < 2.0 ** -20
    rel = offsets(M)
    R = Result()
    nw = B * (H // M) * (W // M)
    R.lse, R.lse_tol = np.zeros((nw, heads, N)), np.zeros((nw, heads, N))
    names = ["out"] + (["dq", "dk", "dv"] if dout is not None else [])
    for n in names:
        setattr(R, n, np.zeros(q.shape)), setattr(R, n + "_tol", np.zeros(q.shape))
    L = (2 * M - 1) ** 2
    R.dbias, R.dbias_tol = np.zeros((heads, L)), np.zeros((heads, L))
    add = 2.0 ** -24 * (N + d + 16)
    split = 0.0 if wide else 2.0 ** -16

    def scores(qq, kk, b):
        s0 = scale * qq @ kk.T
        mag = abs(scale) * np.abs(qq) @ np.abs(kk).T
        # (fp32: the sum's own roundings and the bias's product with log2 e; exp2 has an error of its own)
        eps = u * mag + 2.0 ** -24 * ((d + 4) * mag + 3 * np.abs(np.where(np.isfinite(b), b, 0.0))) + 2.0 ** -22
        return s0 + b, eps

    w = 0
    for bi in range(B):
        for wy in range(H // M):
            for wx in range(W // M):
                ys, xs = pixels(H, W, M, s, wy, wx)
                for h in range(heads):
                    c = slice(h * d, (h + 1) * d)
                    qq, kk, vv = q[bi, ys, xs, c], k[bi, ys, xs, c], v[bi, ys, xs, c]
                    b = bias[h][rel]
                    S, eps = scores(qq, kk, b)
                    eps = np.where(np.isfinite(S), eps, 0.0).max(1, keepdims=True)
                    top = S.max(1, keepdims=True)
                    full = np.isfinite(top)
                    e = np.exp(S - np.where(full, top, 0.0))
                    den = e.sum(1, keepdims=True)
                    with np.errstate(divide="ignore"):
                        lse = np.where(full, top + np.log(np.where(full, den, 1.0)), -np.inf)
                    P = np.where(full, e / np.where(den == 0, 1.0, den), 0.0)
                    O = P @ vv
                    R.lse[w, h], R.lse_tol[w, h] = lse[:, 0], (eps + u + add + 2.0 ** -22 * np.abs(np.where(full, lse, 0.0)))[:, 0]
                    R.out[bi, ys, xs, c] = O
                    R.out_tol[bi, ys, xs, c] = 1.1 * (2 * eps + 2 * u + add) * (P @ np.abs(vv)) + u * np.abs(O)
                    if dout is None:
                        continue
                    if bwd_qkv is not None:
                        qq, kk, vv = (x[bi, ys, xs, c] for x in bwd_qkv)
                        S, eps2 = scores(qq, kk, b)
                        eps = np.maximum(eps, np.where(np.isfinite(S), eps2, 0.0).max(1, keepdims=True))
                    P = np.where(full, np.exp(S - np.where(full, lse, 0.0)), 0.0)
                    do, o = dout[bi, ys, xs, c], out[bi, ys, xs, c]
                    delta = (do * o).sum(1, keepdims=True)
                    dP = do @ vv.T
                    dS = P * (dP - delta)
                    # P's relative error, and what dP - delta is off by
                    t = 1.1 * (2 * eps + u + split * (1 + np.abs(np.where(full, lse, 0.0))) + add)
                    off = (split * np.abs(delta) + 2.0 ** -24 * (d + 4) * (np.abs(do) @ np.abs(vv).T + np.abs(do * o).sum(1, keepdims=True)))
                    eS = t * np.abs(dS) + 1.1 * P * off
                    r = u + add
                    for name, val, tol in (
                            ("dv", P.T @ do, (P * (t + r)).T @ np.abs(do)),
                            ("dq", scale * dS @ kk, abs(scale) * (eS + r * np.abs(dS)) @ np.abs(kk)),
                            ("dk", scale * dS.T @ qq, abs(scale) * (eS + 2 * r * np.abs(dS)).T @ np.abs(qq))):
                        getattr(R, name)[bi, ys, xs, c] = val
                        getattr(R, name + "_tol")[bi, ys, xs, c] = 1.05 * tol + u * np.abs(val) + 1e-30
                    np.add.at(R.dbias[h], rel.reshape(-1), dS.reshape(-1))
                    np.add.at(R.dbias_tol[h], rel.reshape(-1), (eS + 2.0 ** -22 * np.abs(dS)).reshape(-1))
                w += 1
    R.dbias_tol = 1.05 * R.dbias_tol + 2.0 ** -20 * np.abs(R.dbias) + 1e-30
    return R


def pack(x, heads, M, s):
    """(codes [units][N][dp] uint8, exponents [units][N] uint8) of a grid tensor [B][H][W][C] (fp64, storage values)."""
    B, H, W, C = x.shape
    d, N = C // heads, M * M
    dp = (d + 15) // 16 * 16
    nw = B * (H // M) * (W // M)
    codes, exps = np.full((nw * heads, N, dp), 128, np.uint8), np.zeros((nw * heads, N), np.uint8)
    w = 0
    for bi in range(B):
        for wy in range(H // M):
            for wx in range(W // M):
                ys, xs = pixels(H, W, M, s, wy, wx)
                for h in range(heads):
                    rows = x[bi, ys, xs, h * d:(h + 1) * d]
                    for n in range(N):
                        big = np.abs(rows[n]).max()
                        if not np.isfinite(rows[n]).all():
                            exps[w * heads + h, n] = 255
                            continue
                        if big == 0:
                            continue
                        e = 1
                        while big > 127 * 2.0 ** (e - 127):
                            e += 1
                        exps[w * heads + h, n] = e
                        codes[w * heads + h, n, :d] = (np.rint(rows[n] / 2.0 ** (e - 127)) + 128).astype(np.uint8)
                w += 1
    return codes, exps


def unpack(codes, exps, shape, heads, M, s):
    B, H, W, C = shape
    d = C // heads
    x = np.zeros(shape)
    step = np.where(exps == 0, 0.0, 2.0 ** (exps.astype(float) - 127))
    step[exps == 255] = np.nan
    w = 0
    for bi in range(B):
        for wy in range(H // M):
            for wx in range(W // M):
                ys, xs = pixels(H, W, M, s, wy, wx)
                for h in range(heads):
                    u = w * heads + h
                    x[bi, ys, xs, h * d:(h + 1) * d] = (codes[u, :, :d].astype(float) - 128) * step[u][:, None]
                w += 1
    return x
