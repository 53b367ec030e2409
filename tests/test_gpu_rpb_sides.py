"""Windows of more than 96 tokens a side, up to the largest: one unit, every element, against 64 bits on the GPU."""
import pytest
import torch

from paper_2603_06738_amd import binding as rb
from test_gpu_rpb import DEV, Case, packed

pytestmark = pytest.mark.gpu
H = 2.0 ** -24


def diagonals(x):
    """[..., M, M] (query, key) -> [..., 2M-1]: sums over query minus key."""
    M = x.shape[-1]
    x = torch.nn.functional.pad(x.flip(-1), (0, M)).flatten(-2)[..., :M * (2 * M - 1)]
    return x.reshape(*x.shape[:-1], M, 2 * M - 1).sum(-2)


def reference(c, qkv):
    """Values, elementwise bounds and 2-norm bounds (the terms of rpb_bounds.py; of |v - O| only what bounds it, |v| + |O|) of one unit whose
    window is the whole grid, in blocks of window rows."""
    M, N, d, scale = c.M, c.N, c.d, c.p.scale_c
    U, Uo = (2.0 ** -8, 2.0 ** -8) if c.dtype == "bf16" else (0.0, H)
    flat = lambda x: torch.roll(x, (-c.s, -c.s), (1, 2)).reshape(N, d).double()        # noqa: E731
    q, k, v = (flat(x) for x in (c.q, c.k, c.v))
    q8, k8, v8 = (flat(x) for x in qkv)
    do, o = flat(c.dout), flat(c.out)
    table = c.bias[0].double()
    n = torch.arange(N, device=DEV)
    jy, jx = n // M, n % M
    sums, dots = (2 * N + d + 16) * H, H * (d + 4)
    got = {x: torch.empty(N, d, dtype=torch.float64, device=DEV) for x in ("out", "dq")}
    tol = {x: torch.empty_like(got["out"]) for x in got}
    for x in ("dk", "dv"):
        got[x], tol[x] = (torch.zeros(N, d, dtype=torch.float64, device=DEV) for _ in range(2))
    square = {x: torch.zeros((), dtype=torch.float64, device=DEV) for x in ("out", "dq", "dk", "dv")}
    lse, ltol = (torch.empty(N, dtype=torch.float64, device=DEV) for _ in range(2))
    dbias, btol = (torch.zeros(2 * M - 1, 2 * M - 1, dtype=torch.float64, device=DEV) for _ in range(2))
    rows = max(1, 4096 // M)
    for y0 in range(0, M, rows):
        i = n[y0 * M:min(M, y0 + rows) * M]
        b = table[(jy[i][:, None] - jy + M - 1) * (2 * M - 1) + jx[i][:, None] - jx + M - 1]
        b0 = torch.where(torch.isinf(b), torch.zeros_like(b), b).abs()
        S = scale * q[i] @ k.T.contiguous() + b
        eps = (d + 8) * H * (abs(scale) * q[i].abs() @ k.abs().T.contiguous() + b0) + 2.0 ** -22
        lse[i] = torch.logsumexp(S, 1)
        l = lse[i][:, None]
        P = torch.exp(S - l)
        e = eps.amax(1, keepdim=True)
        O, big = P @ v, P @ v.abs()
        got["out"][i], tol["out"][i] = O, 1.05 * ((e + U) * (big + O.abs()) + sums * big) + Uo * O.abs()
        P2 = P * P
        square["out"] += ((U * U * (P2 @ (v * v) - 2 * O * (P2 @ v) + O * O * P2.sum(1, keepdim=True)) + Uo * Uo * O * O) / 3).sum()
        lt = e + sums + 8 * H * l.abs() + 2.0 ** -20
        ltol[i] = lt[:, 0]
        S = scale * q8[i] @ k8.T.contiguous() + b
        P = torch.exp(S - l)
        delta = (do[i] * o[i]).sum(1, keepdim=True)
        dS = P * (do[i] @ v8.T.contiguous() - delta)
        aS = dS.abs()
        t = 1.05 * (e + lt + 6 * H * l.abs() + 2.0 ** -22)
        eS = t * aS + 1.05 * P * dots * (do[i].abs() @ v8.abs().T.contiguous() + (do[i] * o[i]).abs().sum(1, keepdim=True))
        dq = scale * dS @ k8
        got["dq"][i], tol["dq"][i] = dq, abs(scale) * (1.05 * (eS + (U + sums) * aS)) @ k8.abs() + Uo * dq.abs() + 1e-30
        square["dq"] += ((U * U * scale ** 2 * (dS * dS) @ (k8 * k8) + Uo * Uo * dq * dq) / 3).sum()
        Pt, St = P.T.contiguous(), dS.T.contiguous()
        got["dv"] += Pt @ do[i]
        tol["dv"] += (1.05 * P * (t + U + sums)).T.contiguous() @ do[i].abs()
        square["dv"] += (U * U / 3 * (Pt * Pt) @ (do[i] * do[i])).sum()
        got["dk"] += scale * St @ q8[i]
        tol["dk"] += abs(scale) * (1.05 * (eS + (U + sums) * aS)).T.contiguous() @ q8[i].abs()
        square["dk"] += (U * U / 3 * scale ** 2 * (St * St) @ (q8[i] * q8[i])).sum()
        for y in range(y0, min(M, y0 + rows)):
            at = slice((y - y0) * M, (y - y0 + 1) * M)
            for x, to in ((dS, dbias), (eS + 128 * H * aS, btol)):
                # [query column][key row][key column] -> [key row][column offset]; row offsets fall as the key row rises
                to[y:y + M] += diagonals(x[at].reshape(M, M, M).permute(1, 0, 2)).flip(0)
    for x in ("dk", "dv"):
        tol[x] += Uo * got[x].abs() + 1e-30
        square[x] += (Uo * Uo / 3 * got[x] * got[x]).sum()
    # (what is not random: the elementwise bounds without U; the norms use a hundredth of them, and the random part, only where U is the larger)
    norm = {x: 1.2 * float(square[x]) ** 0.5 + (float(((tol[x] if not U else 0.02 * tol[x]) ** 2).sum()) ** 0.5) for x in square}
    return got, tol, norm, lse, ltol, dbias, 1.05 * btol + 1e-30


@pytest.mark.parametrize("dtype,M,d,ckpt", [("bf16", 112, 30, False), ("bf16", 128, 30, True), ("bf16", 131, 8, False), ("bf16", 144, 9, False), ("bf16", 160, 64, False), ("bf16", 250, 8, True),
                                            ("bf16", 256, 16, False), ("f32", 128, 8, True), ("f32", 131, 30, False), ("f32", 255, 8, False), ("f32", 256, 8, False)])
def test_largest_sides(dtype, M, d, ckpt):
    c = Case(dtype, 1, M, M, 1, d, M, M // 3, buckets="near", seed=M) if M < 200 else Case(dtype, 1, M, M, 1, d, M, M // 3, seed=M)
    c.forward()
    held = (c.q, c.k, c.v)
    if ckpt:
        ck = packed(c)
        held = [torch.empty_like(c.q) for _ in range(3)]
        rb.rib_checkpoint_unpack(c.p, ck, *held)
        rb.rib_rpb_attn_bwd_ckpt(c.p, ck, c.bias, c.out, c.dout, c.lse, c.dq, c.dk, c.dv, c.dbias, c.ws)
    else:
        c.backward()
    want, tol, norm, lse, ltol, dbias, btol = reference(c, held)
    assert ((c.lse[0, 0].double() - lse).abs() <= ltol).all()
    assert ((c.dbias[0].double().reshape(dbias.shape) - dbias).abs() <= btol).all()
    for x in want:
        got = torch.roll(getattr(c, x), (-c.s, -c.s), (1, 2)).reshape(c.N, d).double()
        off = (got - want[x]).abs()
        assert (off <= tol[x]).all(), (x, float((off - tol[x]).max()))
        assert float(off.norm()) <= norm[x], (x, float(off.norm()), norm[x], float(want[x].norm()))
