"""What the rounding of the learned bias's kernels may change, term by term: tests/rpb_reference.py's attention in 64 bits, with the bounds
of kernels whose logits are not rounded.  Two bounds of each tensor, elementwise (the worst case) and of the 2-norm of the error.

H = 2^-24 is half a step of fp32.  In bf16 U = 2^-8, half a step of bf16, is what P, dS and the outputs are rounded to; fp32 rounds its outputs alone.

    a logit          a sum of d products and a bias, scaled: d + 8 roundings of H at the size of its terms, and 2^-22 for exp2: eps
    O                weights w (1 + e), |e| <= eps + U, over their own sum: sum of w |e| |v - O|; sums of N terms (two H a term: an instruction that adds
                     two values rounds up to 2.8 H)
    LSE              of P before it is rounded: max eps, sums, 8 H of itself, 2^-20 for the logarithm
    P in backward    t = eps + LSE's bound + 6 H |LSE| + 2^-22, relative
    dS               t |dS|, and P times the fp32 sums of d products in dP and delta (delta from O as it is stored)
    dv, dq, dk       sums of P (t + U) and of dS (.. + U), N roundings of H, and their own
    dbias            dS is not rounded there

The 2-norm: roundings to bf16 are independent, uniform within U of their value at most, so the error's expected square is U^2 / 3 times the sum of the
squared terms; 1.2 times its root leaves room for the sample, and what is not random (eps, t, H) is added as it is."""
import numpy as np

import rpb_reference as ref

H = 2.0 ** -24


class Bounds:
    pass


def attention(q, k, v, bias, heads, M, s, scale, bf16, out=None, dout=None, bwd_qkv=None):
    """As rpb_reference.attention; names with _tol (elementwise) and _norm (2-norm of the error)."""
    B, Hh, W, C = q.shape
    d, N = C // heads, M * M
    rel, L = ref.offsets(M), (2 * M - 1) ** 2
    U, Uo = (2.0 ** -8, 2.0 ** -8) if bf16 else (0.0, H)
    R = Bounds()
    nw = B * (Hh // M) * (W // M)
    R.lse, R.lse_tol = np.zeros((nw, heads, N)), np.zeros((nw, heads, N))
    names = ["out"] + (["dq", "dk", "dv"] if dout is not None else [])
    det, var = {}, dict.fromkeys(names, 0.0)
    for n in names:
        setattr(R, n, np.zeros(q.shape)), setattr(R, n + "_tol", np.zeros(q.shape))
        det[n] = np.zeros(q.shape)
    R.dbias, R.dbias_tol = np.zeros((heads, L)), np.zeros((heads, L))
    sums = (2 * N + d + 16) * H

    def logits(qq, kk, b):
        mag = abs(scale) * np.abs(qq) @ np.abs(kk).T + np.abs(np.where(np.isfinite(b), b, 0.0))
        S = scale * qq @ kk.T + b
        return S, np.where(np.isfinite(S), (d + 8) * H * mag + 2.0 ** -22, 0.0)

    def put(name, at, value, fixed, rounded, squares):
        """`fixed`: what is not random; `rounded`: sums of |terms| that are rounded to U; `squares`: of their squares."""
        getattr(R, name)[at] = value
        det[name][at] = 1.05 * fixed
        getattr(R, name + "_tol")[at] = 1.05 * (fixed + U * rounded) + Uo * np.abs(value) + 1e-30
        var[name] += (U * U * squares + Uo * Uo * value * value).sum() / 3

    w = 0
    for bi in range(B):
        for wy in range(Hh // M):
            for wx in range(W // M):
                ys, xs = ref.pixels(Hh, W, M, s, wy, wx)
                for h in range(heads):
                    at = (bi, ys, xs, slice(h * d, (h + 1) * d))
                    qq, kk, vv, b = q[at], k[at], v[at], bias[h][rel]
                    S, eps = logits(qq, kk, b)
                    top = S.max(1, keepdims=True)
                    full = np.isfinite(top)
                    e = np.exp(S - np.where(full, top, 0.0))
                    den = e.sum(1, keepdims=True)
                    lse = np.where(full, top + np.log(np.where(full, den, 1.0)), -np.inf)
                    P = np.where(full, e / np.where(den == 0, 1.0, den), 0.0)
                    O = P @ vv
                    # (sums over keys of w |v - O| and its square, channel by channel)
                    apart, apart_eps, apart2 = np.zeros(O.shape), np.zeros(O.shape), np.zeros(O.shape)
                    for c in range(d):
                        gap = np.abs(vv[None, :, c] - O[:, c, None])
                        apart[:, c], apart_eps[:, c], apart2[:, c] = (P * gap).sum(1), (P * eps * gap).sum(1), (P * P * gap * gap).sum(1)
                    put("out", at, O, apart_eps + sums * (P @ np.abs(vv)), apart, apart2)
                    R.lse[w, h] = lse[:, 0]
                    lse0 = np.abs(np.where(full, lse, 0.0))
                    ltol = eps.max(1, keepdims=True) + sums + 8 * H * lse0 + 2.0 ** -20
                    R.lse_tol[w, h] = ltol[:, 0]
                    if dout is None:
                        continue
                    if bwd_qkv is not None:
                        qq, kk, vv = (x[at] for x in bwd_qkv)
                        S, eps = logits(qq, kk, b)
                    P = np.where(full, np.exp(S - np.where(full, lse, 0.0)), 0.0)
                    do, o = dout[at], out[at]
                    delta = (do * o).sum(1, keepdims=True)
                    dS = P * (do @ vv.T - delta)
                    t = eps + ltol + 6 * H * lse0 + 2.0 ** -22
                    off = H * (d + 4) * (np.abs(do) @ np.abs(vv).T + np.abs(do * o).sum(1, keepdims=True))
                    eS = 1.05 * (t * np.abs(dS) + P * off)
                    aS = np.abs(dS)
                    put("dv", at, P.T @ do, (P * (t + sums)).T @ np.abs(do), P.T @ np.abs(do), (P * P).T @ (do * do))
                    put("dq", at, scale * dS @ kk, abs(scale) * (eS + sums * aS) @ np.abs(kk), abs(scale) * aS @ np.abs(kk), scale ** 2 * (dS * dS) @ (kk * kk))
                    put("dk", at, scale * dS.T @ qq, abs(scale) * (eS + sums * aS).T @ np.abs(qq), abs(scale) * aS.T @ np.abs(qq), scale ** 2 * (dS * dS).T @ (qq * qq))
                    np.add.at(R.dbias[h], rel.reshape(-1), dS.reshape(-1))
                    np.add.at(R.dbias_tol[h], rel.reshape(-1), (eS + (nw + 64) * H * aS).reshape(-1))
                w += 1
    for n in names:
        setattr(R, n + "_norm", 1.2 * np.sqrt(var[n]) + np.sqrt((det[n] ** 2).sum()) + 1e-30)
    R.dbias_tol = 1.05 * R.dbias_tol + 1e-30
    return R


def outside(name, got, R, times=1):
    """What of `got` lies outside R's bounds: a text, or None.  `times`: so many copies of R's images."""
    want, tol = times * getattr(R, name), times * getattr(R, name + "_tol")
    if times > 1:
        tol = tol + times * (times + 16) * H * np.abs(getattr(R, name))
    inf = np.isinf(want)
    if not np.array_equal(got[inf], want[inf]):
        return f"{name}: infinities"
    off = np.abs(np.where(inf, 0.0, got) - np.where(inf, 0.0, want))
    if not (off <= tol).all():
        worst = np.unravel_index(np.argmax(np.where(np.isnan(off), np.inf, off - tol)), off.shape)
        return f"{name} at {worst}: {got[worst]} for {want[worst]}, {off[worst]:.3g} off, {tol[worst]:.3g} allowed"
    most = getattr(R, name + "_norm", None)
    # (fewer than 2000 elements: a sample too small for the 1.2)
    if most is not None and off.size >= 2000 and np.sqrt((off ** 2).sum()) > most:
        return f"{name}: an error of {np.sqrt((off ** 2).sum()):.4g} in the 2-norm, {most:.4g} allowed"
    return None
