"""Attention over the cache held in 4 bits (sa_cache4_decode_fwd) at the ends of its range: values of V, scores and queries of any size.  Bounds
are those of tests/test_gpu_cache4.py unless a test says otherwise."""
import math

import numpy as np
import pytest
import torch

from oracle import cache4 as orc
from tests import gpu_util as U
from tests.test_gpu_cache4 import Setup, sa

pytestmark = pytest.mark.gpu


def held(c, x):
    t = c.dev(np.ascontiguousarray(x))
    return t, U.to_np64(t)


# ---- V ------------------------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("sizes", [(2.0 ** 109, 1.0), (2.0 ** 112, 2.0 ** 112), (2.0 ** 119, 2.0 ** 3), (2.0 ** 124, 2.0 ** 124), (2.0 ** 124, 2.0 ** -100)])
def test_large_values_of_v(dtype, d, sizes):
    """Both signs, the sizes in turn from tile to tile; one row, few, several tiles a wave"""
    c = Setup(1, 4, 1, d, 32, 9, dtype, seed=d)
    K = c.rows(288)
    V = c.rng.uniform(0.5, 1.5, (1, 1, 288, d)).astype(np.float32) * c.rng.choice([-1, 1], (1, 1, 288, d))
    V *= np.repeat(np.resize(np.float32(sizes), 9), 32)[:, None]
    c.write(K, held(c, V))
    for T, n in ((1, 1), (1, 20), (1, 288), (3, 2), (20, 288)):
        c.check(T, [n])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_the_largest_values_of_v_come_back_finite(dtype, d):
    """6 * 2^125 in all rows: the mean is that, however many there are.  Weights enter product and sum alike; the two are kept to n 2^-24 each, a
    weight's parts in the product to 2^-16 (bf16) and 2^-23 (fp32: three parts), and the quotient is rounded."""
    top = 6 * 2.0 ** 125
    for T, n in ((1, 1), (1, 33), (1, 20000), (20, 1500)):
        c = Setup(1, 4, 1, d, 64, -(-n // 64), dtype, seed=n)
        K = c.rows(n)[0]
        V = torch.full_like(K, top)
        V[..., 1::2] = -top
        sa().sa_cache4_write(c.desc, K, V, None, None, c.dev(c.table), c.pool)
        _, Y, L = c.decode(T, [n])
        want = V[0, 0, 0].double().cpu().numpy()
        parts, half = (2.0 ** -16, 2.0 ** -8) if dtype == "bf16" else (2.0 ** -23, 2.0 ** -24)
        assert np.isfinite(L).all() and (np.abs(Y / want - 1) <= half + parts + 2 * n * 2.0 ** -24).all(), (T, n, np.abs(Y / want - 1).max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_values_of_v_and_scores_that_rise(dtype):
    """The maximum is raised over sums that are large already; large rows that no query sees (behind the last, on a page that is not there)"""
    c = Setup(2, 4, 1, 64, 32, 12, dtype, seed=4, scale=0.5)
    K = c.rows(384)[0]
    K = (K.float() * torch.linspace(0.05, 12, 384, device=U.DEV)[:, None]).to(K.dtype)
    V = c.rows(384)[0]
    V[:, :, :64] *= 2.0 ** 124
    V[1, :, 64:] *= 2.0 ** 60
    V = V.clamp(-2.0 ** 126, 2.0 ** 126)
    c.write((K, U.to_np64(K)), (V, U.to_np64(V)))
    c.check(3, [384, 384])
    c.check(1, [100, 33])
    table = c.table.copy()
    table[0, :2] = -1
    q, Y, L = c.decode(3, [384, 384], table=table)
    assert np.abs(Y[0]).max() < 10 and np.isfinite(Y).all() and np.isfinite(L).all()


# ---- scores -------------------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("size", [2.0 ** 20, 2.0 ** 29, 2.0 ** 33, 2.0 ** 60, 2.0 ** 120, 1.3125 * 2.0 ** 126, -1.3125 * 2.0 ** 127, -2.0 ** 60, -2.0 ** 33, -2.0 ** 29])
@pytest.mark.parametrize("heads", [2, 40])
def test_scores_of_any_size(dtype, d, size, heads):
    """One element of q meets one of K, so that scores are single products k * size, far enough apart that one row takes all: its V comes back, to
    the product's rounding of a weight (2^-11, 2^-22) that the sum takes whole, and the result's."""
    c = Setup(1, heads, 1, d, 32, 12, dtype, seed=3, scale=1.0)
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
    q = torch.zeros(1, heads, 1, d, device=U.DEV)
    q[..., 5] = size
    q = q.to(U.tdtype(dtype))
    p, half = (2.0 ** -11, 2.0 ** -8) if dtype == "bf16" else (2.0 ** -22, 2.0 ** -24)
    for rows, row in best.items():
        _, Y, L = c.decode(1, [rows], q=q)
        want = float(k[0, 0, row, 5]) * float(q[0, 0, 0, 5])
        assert (np.abs(Y[0, :, 0] - Vr[0, 0, row]) <= (half + 1.01 * p) * np.abs(Vr[0, 0, row])).all(), (rows, Y[0, 0, 0, :4], Vr[0, 0, row, :4])
        assert (np.abs(L / want - 1) <= 2.0 ** -21).all(), (rows, L, want)


# ---- queries ------------------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,n", [(1, 1), (1, 40), (3, 40), (1, 9000), (40, 2000)])
@pytest.mark.parametrize("what", ["infinity", "overflow"])
def test_scores_that_are_all_below_every_number(dtype, T, n, what):
    """Softmax over scores that are all -infinity is 0/0, not that of a query without rows; rows of other heads, and queries that see nothing,
    are as they were"""
    c = Setup(2, 4, 2, 64, 32, -(-n // 32), dtype, seed=n)
    K, V = c.rows(n)[0], c.rows(n)[0]
    K[..., 9] = -4 if what == "infinity" else -2.0 ** 100
    table = c.dev(c.table)
    short = min(T, n) - 1                  # the second sequence: its first tokens see nothing
    sa().sa_cache4_write(c.desc, K, V, None, None, table, c.pool)
    q = c.dev(c.rng.standard_normal((2, 4, T, 64)).astype(np.float32))
    q[..., 9] = 0
    _, Y, L = c.decode(T, [n, short], q=q)
    q[:, 1, :, 9] = math.inf if what == "infinity" else 2.0 ** 100
    _, Y2, L2 = c.decode(T, [n, short], q=q)
    assert np.isnan(Y2[0, 1]).all() and np.isnan(L2[0, 1]).all()
    sees = T - short
    assert np.isnan(Y2[1, 1, sees:]).all() and np.isnan(L2[1, 1, sees:]).all()
    assert (Y2[1, 1, :sees] == 0).all() and np.isneginf(L2[1, 1, :sees]).all()
    assert np.array_equal(Y[:, 2:], Y2[:, 2:]) and np.array_equal(L[:, 2:], L2[:, 2:])
    # the head that shares tiles: its maximum is raised elsewhere, weights and sums are rounded anew
    p, half = (2.0 ** -11, 2.0 ** -8) if dtype == "bf16" else (2.0 ** -22, 2.0 ** -24)
    tol = 2 * half * np.abs(Y[:, 0]) + 2 * (p + 2 * n * 2.0 ** -24 + 2.0 ** -18) * 1.2 * float(V.abs().max())
    assert (np.abs(Y[:, 0] - Y2[:, 0]) <= tol).all() and np.array_equal(np.isneginf(L[:, 0]), np.isneginf(L2[:, 0]))


@pytest.mark.parametrize("T,n", [(1, 9000), (3, 100)])
def test_some_scores_below_every_number(T, n):
    """Rows whose score is -infinity weigh nothing beside others: as if their pages were not there"""
    c = Setup(1, 4, 2, 128, 32, -(-n // 32), "f32", seed=n)
    K, V = c.rows(n)[0], c.rows(n)[0]
    K[..., 9] = 0
    K[:, :, 32:96, 9] = -2.0 ** 100        # two whole pages
    sa().sa_cache4_write(c.desc, K, V, None, None, c.dev(c.table), c.pool)
    q = c.dev(c.rng.standard_normal((1, 4, T, 128)).astype(np.float32))
    q[..., 9] = 2.0 ** 100
    _, Y, L = c.decode(T, [n], q=q)
    table = c.table.copy()
    table[0, 1:3] = -1
    _, Y2, L2 = c.decode(T, [n], q=q, table=table)
    assert np.array_equal(Y, Y2) and np.array_equal(L, L2) and np.isfinite(Y).all()


def test_pages_that_are_not_there_leave_nothing_to_see():
    """Also where the first rows of a sequence would be in sight"""
    c = Setup(1, 4, 2, 64, 32, 300, "bf16", seed=2)
    table = np.full_like(c.table, -1)
    for T in (1, 3, 20):
        _, Y, L = c.decode(T, [9600], table=table)
        assert (Y == 0).all() and np.isneginf(L).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T", [1, 20])
def test_fp32_queries_next_to_the_largest_number(d, T):
    """Past bf16's largest number their first part of 8 bits is that one, and all three add up to the number as ever"""
    c = Setup(1, 4, 2, d, 32, 4, "f32", seed=d)
    c.write(c.rows(100, 2.0 ** -124), c.rows(100))
    q = c.rng.uniform(-1, 1, (1, 4, T, d)) * 2.0 ** 121
    top = float(np.finfo(np.float32).max)
    q[..., 3] = top
    q[..., 7] = -top * (1 - 2.0 ** -20)
    q[..., 11] = 3.3895e38                 # the first that is rounded up to an infinity is 3.3961e38
    q = c.dev(q.astype(np.float32))
    _, Y, L = c.decode(T, [100], q=q)
    Yr, Lr, A = orc.attention(c.oracle, c.table, U.to_np64(q), [100], 100, c.scale)
    delta = (d + 8) * 2.0 ** -24 * A + 2.0 ** -22 * (1 + A)
    assert (np.abs(Y - Yr) <= 2.0 ** -24 * np.abs(Yr) + ((2 * delta + 2.0 ** -22 + 200 * 2.0 ** -24) * c.vmax)[..., None]).all()
    assert (np.abs(L - Lr) <= delta + 100 * 2.0 ** -24 + 2.0 ** -22 * (1 + np.abs(Lr))).all()
