"""Rows held in 4 bits for every finite bf16 number (and the fp32 numbers next to them), against the definition in include/sa.h in fp64: to the bit."""
import numpy as np
import pytest
import torch

from oracle import cache4 as orc
from tests import gpu_util as U
from tests.test_gpu_cache4 import sa

pytestmark = pytest.mark.gpu


def all_bf16():
    """Every finite bf16 number as fp32, in ascending order of magnitude, both signs"""
    bits = np.arange(0x7f80, dtype=np.uint32) << 16
    x = bits.view(np.float32)
    return np.stack([x, -x], 1).reshape(-1)


def blocks(order):
    """Each number beside: its neighbours, numbers of all sizes, numbers of up to 3 binades more (where all codes occur)"""
    x = all_bf16()
    rng = np.random.default_rng(0)
    if order == "neighbours":
        return x.reshape(-1, 32)
    if order == "all sizes":
        return rng.permutation(x).reshape(-1, 32)
    binade = x.reshape(-1, 256)           # 255 of them, the first the subnormal numbers
    near = np.concatenate([binade[i:i + 4].reshape(-1) for i in range(len(binade) - 3)]).reshape(-1, 1024)
    return rng.permuted(near, axis=1).reshape(-1, 32)


@pytest.mark.parametrize("dtype,off", [("bf16", 0), ("f32", -1), ("f32", 0), ("f32", 1)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("order", ["neighbours", "all sizes", "near"])
def test_every_finite_bf16_number(order, d, dtype, off):
    """off: the fp32 number that many places above in magnitude, next to every tie and turn"""
    x = blocks(order)
    if off:
        x = (x.view(np.int32) + np.where((x == 0) & (off < 0), 0, off)).astype(np.int32).view(np.float32)
    x = np.concatenate([x, np.zeros((-len(x) % (1024 * d // 32), 32), np.float32)])
    T = len(x) * 32 // d
    desc = sa().make_cache4_desc(1, 1, 1, d, 1024, T // 1024, T // 1024, 1, sa().SA_BF16 if dtype == "bf16" else sa().SA_F32)
    pool = torch.full((sa().sa_cache4_pool_bytes(desc),), 255, dtype=torch.uint8, device=U.DEV)
    table = torch.arange(T // 1024, dtype=torch.int32, device=U.DEV).view(1, -1)
    K = torch.from_numpy(x.reshape(1, 1, T, d)).to(U.DEV).to(U.tdtype(dtype))
    V = K.flip(2).contiguous()
    k, v = torch.empty_like(K), torch.empty_like(K)
    sa().sa_cache4_write(desc, K, V, None, None, table, pool)
    sa().sa_cache4_read(desc, pool, table, None, None, k, v)
    want = orc.blocks_held(x.astype(np.float64)).reshape(T, d)
    for got, ref in ((k, want), (v, want[::-1])):
        got = U.to_np64(got)[0, 0]
        assert np.array_equal(got, ref), np.argwhere(got != ref)[:4]
        assert np.array_equal(np.signbit(got), np.signbit(ref))
