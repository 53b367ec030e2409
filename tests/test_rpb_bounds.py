"""The bounds of rpb_bounds.py, on the CPU: a plain model of the bf16 kernels' arithmetic lies within them, and what a mistake in a kernel would
give does not."""
import numpy as np
import pytest
import torch

import rpb_bounds
import rpb_reference as ref

NAMES = ("lse", "out", "dq", "dk", "dv", "dbias")


def bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x)).float().to(torch.bfloat16).double().numpy()


def model(q, k, v, dout, bias, M, scale, mistake=None):
    """One window and head, N x d each, as the bf16 kernels round: P, dS and the outputs; everything else in 64 bits."""
    b = bias[0][ref.offsets(M)]
    S = scale * q @ k.T + b
    if mistake == "q rounded":
        S = bf16(scale * q) @ k.T + b
    if mistake == "key tile":
        S[:, 64:128] = -np.inf
    if mistake == "bias transposed":
        S = scale * q @ k.T + b.T
    top = S.max(1, keepdims=True)
    P = np.exp(S - top)
    R = bf16(P)
    if mistake == "half a merge":           # the two halves of a row's keys added up at maxima of their own
        half = np.arange(len(k)) % 64 < 32
        R = bf16(np.where(half, np.exp(S - S[:, half].max(1, keepdims=True)), np.exp(S - S[:, ~half].max(1, keepdims=True))))
    out = bf16(R @ v / R.sum(1, keepdims=True))
    lse = top[:, 0] + np.log((R if mistake == "rounded sum" else P).sum(1))
    P = np.exp(scale * q @ k.T + b - lse[:, None])
    dS = P * (dout @ v.T - (dout * (0 if mistake == "no delta" else out)).sum(1, keepdims=True))
    if mistake == "dq unscaled":
        scale = 1.0
    dbias = np.zeros((1, (2 * M - 1) ** 2))
    np.add.at(dbias[0], ref.offsets(M).reshape(-1), dS.reshape(-1))
    return dict(lse=lse[None, None], out=out, dq=bf16(scale * bf16(dS) @ k), dk=bf16(scale * bf16(dS).T @ q), dv=bf16(bf16(P).T @ dout), dbias=dbias)


def case(M, d, spread, std, scale, seed=0):
    rng = np.random.default_rng(seed)
    q, k, v = (bf16(rng.standard_normal((M * M, d)) * spread) for _ in range(3))
    return q, k, v, bf16(rng.standard_normal((M * M, d))), rng.standard_normal((1, (2 * M - 1) ** 2)).astype(np.float32).astype(float) * std, scale


CASES = {"ordinary": (16, 30, 1.0, 0.5, 30 ** -0.5), "narrow": (12, 16, 1.0, 0.5, 0.25), "wide": (16, 64, 1.0, 0.5, 0.125), "large logits": (16, 24, 8.0, 40.0, 1.0)}


def bounds(c, M, got):
    grid = lambda x: x.reshape(1, M, M, -1)             # noqa: E731
    q, k, v, dout, bias, scale = c
    return rpb_bounds.attention(*map(grid, (q, k, v)), bias, 1, M, 0, scale, True, out=grid(got["out"]), dout=grid(dout))


def found(got, R, M):
    return [n for n in NAMES if rpb_bounds.outside(n, got[n] if n in ("lse", "dbias") else got[n].reshape(1, M, M, -1), R)]


@pytest.mark.parametrize("name", list(CASES))
def test_the_kernels_arithmetic_is_within(name):
    M = CASES[name][0]
    c = case(*CASES[name])
    got = model(*c[:4], c[4], M, c[5])
    assert found(got, bounds(c, M, got), M) == []


WHERE = {"q rounded": {"lse"}, "key tile": {"out", "lse", "dq", "dk", "dv"}, "half a merge": {"out"}, "no delta": {"dq", "dk", "dbias"},
         "bias transposed": {"out", "lse", "dq"}, "rounded sum": {"lse"}, "dq unscaled": {"dq", "dk"}}


def shows(name, mistake):
    """A scale of one changes nothing, a power of two keeps q's digits, and with logits in the hundreds a row's largest P is 1 and the others
    next to nothing, so that their rounding is, too."""
    scale = CASES[name][4]
    return not (mistake == "dq unscaled" and scale == 1.0 or mistake == "q rounded" and np.log2(scale) % 1 == 0 or mistake == "rounded sum" and name == "large logits")


@pytest.mark.parametrize("name,mistake", [(n, m) for n in CASES for m in WHERE if shows(n, m)])
def test_mistakes_are_outside(name, mistake):
    M = CASES[name][0]
    c = case(*CASES[name])
    got = model(*c[:4], c[4], M, c[5], mistake)
    assert WHERE[mistake] <= set(found(got, bounds(c, M, got), M))


@pytest.mark.parametrize("name", list(CASES))
def test_zeros_are_outside(name):
    """Element by element: most zeros, wherever the value is not itself next to zero."""
    M = CASES[name][0]
    c = case(*CASES[name])
    got = model(*c[:4], c[4], M, c[5])
    R = bounds(c, M, got)
    for n in NAMES:
        want, tol = getattr(R, n), getattr(R, n + "_tol")
        assert rpb_bounds.outside(n, np.zeros_like(want), R)
        size = np.sqrt((want ** 2).mean())
        assert (tol <= 0.25 * size).mean() > 0.9 if n != "dbias" else (tol <= 0.25 * size).all(), n
