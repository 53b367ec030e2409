"""The learned bias's table: gradients of buckets that differ by many orders of magnitude, each to its own fp32 precision."""
import numpy as np
import pytest
import torch

import rpb_reference as ref
from paper_2603_06738_amd import binding as rb
from test_gpu_rpb import DEV, np64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,buckets", [(2, 3), (5, 7), (12, 40), (12, 529), (48, 625), (96, 5000), (256, 625)])
def test_small_gradients_beside_large_ones(dtype, M, buckets):
    """Buckets of 1e-30 to 1e30, in one head, of either sign.  A bucket's terms are whole multiples of a unit: the power of two above its
    largest over 2^(62 - bits of the number of offsets), 2^-43 of its largest at most; every term is half a unit off at most, and the sum is
    rounded to the table's type."""
    rng = np.random.default_rng(M)
    L, heads = (2 * M - 1) ** 2, 3
    index = rng.integers(-1, buckets + 1, L).astype(np.int32)
    size = 10.0 ** rng.uniform(-30, 30, buckets + 2)
    if dtype == "bf16":
        size = np.clip(size, 1e-30, 1e30)
    db = (rng.standard_normal((heads, L)) * size[index]).astype(np.float32)
    db[1] = np.abs(db[1])
    db[2, ::3] = 0
    tp = rb.make_rpb_params(M, heads, buckets, dtype)
    got = torch.full((heads, buckets), float("nan"), dtype=torch.float32 if dtype == "f32" else torch.bfloat16, device=DEV)
    rb.rib_rpb_table_bwd(tp, torch.from_numpy(db).to(DEV), torch.from_numpy(index).to(DEV), got)
    want, most, terms = np.zeros((heads, buckets)), np.zeros((heads, buckets)), np.zeros(buckets)
    for o in range(L):
        if 0 <= index[o] < buckets:
            want[:, index[o]] += db[:, o]
            most[:, index[o]] = np.maximum(most[:, index[o]], np.abs(db[:, o]))
            terms[index[o]] += 1
    u = 2.0 ** -24 if dtype == "f32" else 2.0 ** -8
    tol = 0.5 * terms * 2.0 ** -43 * most + u * np.abs(want) * (1 + 2.0 ** -20)
    assert (np.abs(np64(got) - want) <= tol).all()
    assert (np64(got)[:, terms == 0] == 0).all()


def test_largest_and_smallest_numbers():
    """Sums of the largest finite numbers overflow to infinity only where they must; denormal numbers are added exactly."""
    M, buckets = 3, 4
    index = np.arange(25).astype(np.int32) % buckets
    db = np.zeros((1, 25), np.float32)
    top = np.float32(3.4028235e38)
    db[0, [0, 4]] = top, -top                   # bucket 0: they cancel
    db[0, [1, 5]] = top, top                    # bucket 1: beyond fp32
    db[0, [2, 6, 10]] = 1e-45, 3e-45, -1e-45    # bucket 2: denormal
    db[0, [3, 7]] = 1.0, 2.0 ** -30             # bucket 3
    got = torch.empty(1, buckets, device=DEV)
    rb.rib_rpb_table_bwd(rb.make_rpb_params(M, 1, buckets), torch.from_numpy(db).to(DEV), torch.from_numpy(index).to(DEV), got)
    g = got.cpu().numpy()[0]
    assert g[0] == 0 and g[1] == np.inf and g[2] == np.float32(3e-45) and g[3] == 1.0
    assert ref.table_grad(db.astype(float), index, buckets)[0, 2] == pytest.approx(2 * 1.4e-45, rel=0.2)
