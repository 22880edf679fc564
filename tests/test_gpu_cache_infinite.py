"""Keys of infinity in the 8-bit paged cache's open blocks."""
import numpy as np
import pytest
import torch

from cache_reference import BLOCK, tolerance, values
from test_gpu_cache import Both

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("prec,dh,start,P", [("bf16", 64, 0, 40), ("bf16", 16, 50, 33), ("bf16", 128, 0, 20),
                                             ("fp32", 16, 60, 20), ("bf16", 64, 30, 150), ("fp32", 64, 10, 140)])
@pytest.mark.parametrize("came", ["before", "now"])
def test_infinite_keys(prec, dh, start, P, came):
    """A position that sees a key of infinity gets NaN, whatever the sign of its
    product (a score of -inf is no weight of 0); no other position does."""
    if came == "before" and start == 0:
        start = 21
    b = Both(1, 2, 2, dh, prec, 2, 300, seed=5)
    hk, hv = b.rand(2, max(start, 1), 2, dh), b.rand(2, max(start, 1), 2, dh)
    q, k, v = b.rand(2, P, 2, dh), b.rand(2, P, 2, dh), b.rand(2, P, 2, dh)
    at = start // BLOCK * BLOCK if came == "before" else start + 2      # (a position of the open block)
    x = (hk if came == "before" else k)[:, at if came == "before" else 2]
    x[0, 0, 1], x[1, 1, 3] = float("inf"), float("-inf")
    if start:
        b.begin(start)
        b.step(queries=False, rows=[(None, hk, hv)])
        b.commit()
    b.begin(P)
    got = values(b.c.tppsd_cache_attend(0, q, k, v))
    fine = torch.where(torch.isfinite(k), k, 0.0)
    b.r.rows = np.where(np.isfinite(b.r.rows), b.r.rows, 0.0)
    b.r.append(0, values(fine), values(v))
    want = np.zeros(got.shape)
    weight, score = b.r.attend(0, values(q), want, float(np.float32(dh ** -0.5)), False)
    nan = np.zeros(want.shape, bool)
    nan[0, max(at - start, 0):, 0] = nan[1, max(at - start, 0):, 1] = True
    assert np.array_equal(np.isnan(got), nan), np.argwhere(np.isnan(got) != nan)[:8]
    tol = tolerance(prec, dh, start + P, want, weight, score)
    assert (np.abs(got - want)[~nan] <= tol[~nan]).all()
