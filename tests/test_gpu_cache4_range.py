"""Attention over the cache held in 4 bits (sa_cache4_decode_fwd) at the ends of its range: values of V, scores and queries of any size.  Bounds
are those of tests/test_gpu_cache4.py unless a test says otherwise."""
import numpy as np
import pytest
import torch

from tests import gpu_util as U
from tests.test_gpu_cache4 import Setup, sa

pytestmark = pytest.mark.gpu


def held(c, x):
    t = c.dev(np.ascontiguousarray(x))
    return t, U.to_np64(t)


# ---- scores -------------------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("size", [2.0 ** 20, 2.0 ** 29, 2.0 ** 33, 2.0 ** 60, 2.0 ** 120, 1.3125 * 2.0 ** 126, -1.3125 * 2.0 ** 127, -2.0 ** 60, -2.0 ** 33, -2.0 ** 29])
def test_scores_of_any_size(dtype, d, size):
    """One element of q meets one of K, so that scores are single products k * size, far enough apart that one row takes all: its V comes back, to
    the product's rounding of a weight (2^-11, 2^-22) that the sum takes whole, and the result's."""
    c = Setup(1, 2, 1, d, 32, 12, dtype, seed=3, scale=1.0)
    n = 384
    k = np.zeros((1, 1, n, d), np.float32)
    grid = np.float32([0.5, 1, 1.5])
    k[0, 0, :, 5] = grid[c.rng.integers(0, 3, n)]
    best = {1: 0, 40: 17, 384: 300}   # rows seen -> the one that outscores them
    order = (2, 3, 4) if size > 0 else (0.5, 0.25, 0.125)
    if size < 0:
        k[0, 0, :, 5] = np.float32([1, 1.5])[c.rng.integers(0, 2, n)]
    for row, what in zip(best.values(), order):
        k[0, 0, row, 5] = what
    if abs(size) > 2.0 ** 124:       # one row: 1.3125 2^127 log2 e = 3.22e38 is a number still
        k *= 0.25 if size > 0 else 2
    c.write(held(c, k), c.rows(n))
    _, Vr = c.read(n, None, None)
    q = torch.zeros(1, 2, 1, d, device=U.DEV)
    q[..., 5] = size
    q = q.to(U.tdtype(dtype))
    p, half = (2.0 ** -11, 2.0 ** -8) if dtype == "bf16" else (2.0 ** -22, 2.0 ** -24)
    for rows, row in best.items():
        _, Y, L = c.decode(1, [rows], q=q)
        want = float(k[0, 0, row, 5]) * float(q[0, 0, 0, 5])
        assert (np.abs(Y[0, :, 0] - Vr[0, 0, row]) <= (half + 1.01 * p) * np.abs(Vr[0, 0, row])).all(), (rows, Y[0, 0, 0, :4], Vr[0, 0, row, :4])
        assert (np.abs(L / want - 1) <= 2.0 ** -21).all(), (rows, L, want)
