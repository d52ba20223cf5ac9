"""GPU parity of the K/V cache held in 4 bits (sa_cache4_write, _read, _decode_fwd) against the fp64 oracle, through the C ABI.

Bounds.  Rows are held to the bit.  Attention over the rows held, with n rows seen, A the largest scale * sum |q k| of a query and
v the largest |V|: a score is off by at most (d + 8) 2^-24 A (fp32 sums of d exact products), its exponential by that and 2^-22 (1 + A) relative
(rounded argument, hardware exponential), which enters numerator and denominator: 2 delta v.  A probability is a number of 11 bits (bf16:
half a step, 2^-12) or the sum of two (fp32: half a step of half a step, 2^-24, and 2^-24 for what the second part's subnormal numbers
leave), the sums over n rows are kept to n 2^-24, and the result is rounded to its type once, half a step."""
import numpy as np
import pytest
import torch

from oracle import cache4 as orc
from tests import gpu_util as U

pytestmark = pytest.mark.gpu


def sa():
    from paper_2604_00754_amd import binding
    return binding


class Setup:
    """A cache of random pages, everything in it 0xFF (codes -6, scale bytes 255) until it is written, with the oracle's beside it"""

    def __init__(self, B, Hq, Hkv, d, page_rows, max_pages, dtype, seed, scale=0.0, spare=3):
        print(f"case cache4 B{B} Hq{Hq} Hkv{Hkv} d{d} page_rows{page_rows} max_pages{max_pages} {dtype} seed{seed}", flush=True)
        self.rng = np.random.default_rng(seed)
        P = B * max_pages + spare
        self.B, self.Hq, self.Hkv, self.d, self.cap, self.dtype, self.P = B, Hq, Hkv, d, page_rows * max_pages, dtype, P
        self.table = self.rng.permutation(P)[:B * max_pages].reshape(B, max_pages).astype(np.int32)
        self.desc = sa().make_cache4_desc(B, Hq, Hkv, d, page_rows, P, max_pages, 1, sa().SA_BF16 if dtype == "bf16" else sa().SA_F32, scale)
        assert sa().sa_cache4_pool_bytes(self.desc) == P * Hkv * page_rows // 32 * 34 * d
        self.pool = torch.full((sa().sa_cache4_pool_bytes(self.desc),), 255, dtype=torch.uint8, device=U.DEV)
        self.oracle = orc.Cache(Hkv, d, page_rows, P)
        self.scale = scale or d ** -0.5
        self.vmax = 0.0

    def dev(self, x, dtype=None):
        t = torch.from_numpy(np.ascontiguousarray(x)).to(U.DEV)
        return t if t.dtype == torch.int32 else t.to(dtype or U.tdtype(self.dtype)).contiguous()

    def rows(self, T, scale=1.0):
        """-> device tensor [B, Hkv, T, d] and what it holds in fp64"""
        t = self.dev(self.rng.standard_normal((self.B, self.Hkv, T, self.d)).astype(np.float32) * np.float32(scale))
        return t, U.to_np64(t)

    def write(self, K, V, starts=None, counts=None, table=None):
        """On both sides; K, V: pairs as from rows()"""
        T = K[1].shape[2]
        self.vmax = max(self.vmax, 1.2 * np.abs(V[1][np.isfinite(V[1])]).max(initial=0))  # rounding raises a block's largest by a fifth at most
        table = self.table if table is None else table
        s, c = (None if x is None else self.dev(np.asarray(x, np.int32)) for x in (starts, counts))
        sa().sa_cache4_write(self.desc, K[0], V[0], s, c, self.dev(table), self.pool)
        orc.write(self.oracle, table, K[1], V[1], np.zeros(self.B, int) if starts is None else starts, np.full(self.B, T) if counts is None else counts)

    def assert_bytes(self):
        got = self.pool.cpu().numpy().reshape(self.oracle.bytes.shape)
        assert np.array_equal(got, self.oracle.bytes), np.argwhere(got != self.oracle.bytes)[:5]

    def read(self, T, starts, counts, table=None):
        """Of the device, rows not read hold 7"""
        K = torch.full((self.B, self.Hkv, T, self.d), 7.0, device=U.DEV, dtype=U.tdtype(self.dtype))
        V = torch.full_like(K, 7.0)
        s, c = (None if x is None else self.dev(np.asarray(x, np.int32)) for x in (starts, counts))
        sa().sa_cache4_read(self.desc, self.pool, self.dev(self.table if table is None else table), s, c, K, V)
        return U.to_np64(K), U.to_np64(V)

    def decode(self, T, lens, max_len=None, table=None, q=None, lse=True):
        table = self.table if table is None else table
        max_len = max(1, max(lens)) if max_len is None else max_len
        if q is None:
            q = self.dev(self.rng.standard_normal((self.B, self.Hq, T, self.d)).astype(np.float32))
        need = sa().sa_cache4_workspace_bytes(self.desc, sa().SA_OP_CACHE4_DECODE, T)
        ws = torch.full((max(need, 16),), 255, dtype=torch.uint8, device=U.DEV)  # NaN: what is read has been written
        Y = torch.full_like(q, float("nan"))
        L = torch.full(q.shape[:3], float("nan"), device=U.DEV) if lse else None
        sa().sa_cache4_decode_fwd(self.desc, q, self.pool, self.dev(table), self.dev(np.asarray(lens, np.int32)), max_len, Y, L, ws if need else None)
        torch.cuda.synchronize()
        return q, U.to_np64(Y), None if L is None else L.cpu().numpy().astype(np.float64)

    def check(self, T, lens, max_len=None, table=None):
        q, Y, L = self.decode(T, lens, max_len, table)
        bound = max(1, max(lens)) if max_len is None else max_len
        Yr, Lr, A = orc.attention(self.oracle, self.table if table is None else table, U.to_np64(q), lens, bound, self.scale)
        n = bound
        delta = (self.d + 8) * 2.0 ** -24 * A + 2.0 ** -22 * (1 + A)
        v = self.vmax
        p, half = (2.0 ** -12, 2.0 ** -8) if self.dtype == "bf16" else (2.0 ** -23, 2.0 ** -24)
        tol = half * np.abs(Yr) + ((2 * delta + p + 2 * n * 2.0 ** -24) * v)[..., None]
        assert np.array_equal(np.isnan(Y), np.isnan(Yr))
        off = np.where(np.isnan(Yr), 0, np.abs(Y - Yr) - tol)
        assert (off <= 0).all(), (off.max(), np.unravel_index(off.argmax(), off.shape))
        assert np.array_equal(np.isnan(L), np.isnan(Lr)) and np.array_equal(np.isneginf(L), np.isneginf(Lr))
        fine = np.isfinite(Lr)
        assert (np.abs(np.where(fine, L, 0) - np.where(fine, Lr, 0))[fine] <= (delta + n * 2.0 ** -24 + 2.0 ** -22 * (1 + np.abs(np.where(fine, Lr, 0))))[fine]).all()
        return Y, L


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page_rows,max_pages,T,starts,counts", [
    (32, 4, 1, [0, 31, 127], None),                  # single tokens: the first, the last of a page, the last of all
    (64, 2, 33, [0, 5, 95], [33, 32, 33]),           # over the edges of tiles and pages
    (256, 1, 100, [3, 60, 155], [0, 100, -4]),       # nothing of some sequences; a count below 0
    (32, 5, 160, None, None),                        # all of it
    (64, 2, 70, [-20, 100, 128], [70, 71, 70]),      # positions before the first, past the last; a count above T
    (1024, 1, 17, [1000, 1023, 2 ** 31 - 1], None),  # past the end of the range of positions
])
def test_rows_are_held_to_the_bit(dtype, d, page_rows, max_pages, T, starts, counts):
    c = Setup(3, 4, 2, d, page_rows, max_pages, dtype, seed=T)
    c.table[1, 0] = c.P if max_pages > 1 else c.table[1, 0]   # a page that is not there
    c.write(c.rows(T), c.rows(T), starts, counts)
    c.assert_bytes()
    K, V = c.read(T, starts, counts)
    Kr, Vr = np.full(K.shape, 7.0), np.full(V.shape, 7.0)
    orc.read(c.oracle, c.table, Kr, Vr, [0] * 3 if starts is None else starts, [T] * 3 if counts is None else counts)
    assert np.array_equal(K, Kr, equal_nan=True) and np.array_equal(V, Vr, equal_nan=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_values_at_the_edges_of_the_format(dtype):
    """Ties, magnitudes around 7/4 of a power, zeros of either sign, blocks of zeros, the smallest and largest numbers"""
    c = Setup(1, 1, 1, 64, 32, 1, dtype, seed=0)
    x = np.zeros((1, 1, 32, 64), np.float32)
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, 0.2500001, 0.7499999, 5.0000005, 4.9999995], np.float32)
    for i, e in enumerate((-140, -126, -125, -124, -30, -1, 0, 1, 30, 120, 124)):
        with np.errstate(over="ignore"):
            row = np.resize(np.concatenate([ties, -ties]), 32) * np.float32(2.0) ** np.float32(e)
        x[0, 0, i, :32] = np.where(np.isfinite(row), row, 1)
        x[0, 0, i, 32:] = np.resize([1.0, -0.0, 0.0, 1e-45, -1e-45, 1.75, 1.7500001], 32) * np.float32(2.0) ** np.float32(min(e, 100))
    x[0, 0, 12] = np.float32(3.0e38)
    x[0, 0, 13] = np.float32(1.7500001)
    x[0, 0, 14] = np.float32(1.75)
    x[0, 0, 15] = np.float32(-2.0 ** -149)
    x[0, 0, 16, 3] = np.float32(2.0 ** 127)
    t = c.dev(x)
    c.write((t, U.to_np64(t)), (t, U.to_np64(t)))
    c.assert_bytes()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_the_largest_rows_come_back_finite(dtype, d):
    """Above 7 * 2^125 the next power of two would hold 4 * 2^126, which is no number: 6 * 2^125 is held.  Queries of zeros see them evenly."""
    c = Setup(1, 2, 1, d, 32, 2, dtype, seed=1)
    top = torch.finfo(U.tdtype(dtype)).max
    t = torch.full((1, 1, 40, d), top, device=U.DEV, dtype=U.tdtype(dtype))
    t[:, :, 1::2] *= -1
    zero = torch.zeros_like(t)
    c.write((t, U.to_np64(t)), (zero, U.to_np64(zero)))
    c.assert_bytes()
    K, V = c.read(40, [0], None)
    assert np.array_equal(K, np.sign(U.to_np64(t)) * 6 * 2.0 ** 125) and not V.any()
    q = torch.zeros((1, 2, 1, d), device=U.DEV, dtype=U.tdtype(dtype))
    _, Y, L = c.decode(1, [40], q=q)
    assert not Y.any() and np.allclose(L, np.log(40), rtol=2.0 ** -20, atol=0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_bf16_value_is_rounded_as_defined(dtype):
    """All magnitudes of one binade beside a largest of each of 8 kinds"""
    c = Setup(1, 1, 1, 128, 128, 1, dtype, seed=1)
    x = np.zeros((128, 4, 32), np.float32)
    small = np.arange(0, 128 * 31 * 4).reshape(128, 4, 31) % 1024
    x[..., 1:] = small / 1024 * 8 * np.where(small & 1, -1, 1)
    x[..., 0] = np.resize([4, 4.5, 5, 5.5, 6, 6.5, 7, 7.5], (128, 4))
    x = x.reshape(1, 1, 128, 128) * np.float32(0.125)
    t = c.dev(x)
    c.write((t, U.to_np64(t)), (t, U.to_np64(t)))
    c.assert_bytes()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_rows_with_infinities_and_nan(dtype, d):
    """Held as such in the head they are in; seen by the queries that see the row and by no other"""
    c = Setup(2, 4, 2, d, 32, 3, dtype, seed=d)
    K, V = c.rows(50), c.rows(50)
    for x, b, h, t, e, what in ((K, 0, 0, 20, 3, np.inf), (V, 0, 1, 47, d - 1, np.nan), (V, 1, 0, 49, 0, -np.inf)):
        x[0][b, h, t, e] = float(what)
        x[1][b, h, t, e] = what
    c.write(K, V)
    c.assert_bytes()
    k, v = c.read(50, None, None)
    bad = np.zeros((2, 2, 50), bool)
    bad[0, 0, 20] = bad[0, 1, 47] = bad[1, 0, 49] = True
    assert np.array_equal(np.isnan(k), np.broadcast_to(bad[..., None], k.shape)) and np.array_equal(np.isnan(v), np.isnan(k))
    Y, _ = c.check(5, [50, 50])
    nan = np.isnan(Y).all(-1)
    assert np.array_equal(nan, np.isnan(Y).any(-1)) and nan[0, :2].all() and np.array_equal(nan[0, 2:], [[False, False, True, True, True]] * 2)
    assert np.array_equal(nan[1], [[False] * 4 + [True]] * 2 + [[False] * 5] * 2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,Hq,Hkv,d,page_rows,max_pages,T,lens", [
    (2, 4, 4, 64, 32, 4, 1, [128, 1]),             # one query head per KV head
    (2, 8, 2, 128, 64, 4, 1, [200, 33]),           # four
    (1, 8, 1, 64, 256, 1, 1, [77]),                # eight
    (1, 12, 1, 128, 32, 3, 1, [96]),               # twelve
    (1, 40, 1, 64, 32, 3, 1, [90]),                # forty: three blocks of rows for one token
    (3, 4, 2, 128, 64, 2, 3, [2, 0, 128]),         # fewer rows than tokens, none at all
    (2, 8, 2, 64, 32, 5, 5, [160, 41]),            # 20 query rows a KV head: two blocks of 16
    (1, 6, 2, 128, 32, 4, 7, [100]),               # 21
    (1, 8, 2, 128, 64, 3, 13, [190]),              # 52: four blocks
    (1, 4, 4, 64, 32, 5, 70, [150]),               # 70: a second set of rows
    (1, 8, 2, 128, 32, 5, 37, [159]),              # 148, heads and sets out of step
    (2, 2, 1, 64, 32, 3, 90, [90, 60]),            # a prompt over itself, with tokens before its first row
])
def test_attention(dtype, B, Hq, Hkv, d, page_rows, max_pages, T, lens):
    c = Setup(B, Hq, Hkv, d, page_rows, max_pages, dtype, seed=T + d)
    n = max(lens)
    c.write(c.rows(n), c.rows(n), None, lens)
    c.check(T, lens)


@pytest.mark.parametrize("d", [64, 128])
def test_lengths_around_the_edges_of_tiles(d):
    c = Setup(1, 4, 1, d, 64, 6, "bf16", seed=d)
    c.write(c.rows(384), c.rows(384))
    for n in (1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 160, 255, 257, 384):
        c.check(1, [n])
        c.check(3, [n])


def test_the_rows_of_many_pieces():
    """Workspace sized by the capacity, pieces by the length at hand"""
    for Hkv, cap, lens in ((1, 64 * 40, [2501]), (2, 64 * 40, [97]), (1, 64 * 40, [2560])):
        c = Setup(1, 4 * Hkv, Hkv, 64, 64, cap // 64, "bf16", seed=cap)
        c.write(c.rows(max(lens)), c.rows(max(lens)), None, lens)
        c.check(1, lens)
        c.check(1, lens, max_len=cap)


def test_pages_that_are_not_there_and_lengths_out_of_range():
    c = Setup(3, 4, 2, 128, 32, 4, "bf16", seed=5)
    c.write(c.rows(128), c.rows(128))
    table = c.table.copy()
    table[0, 1], table[1, 0], table[1, 3], table[2] = -1, c.P, 2 ** 31 - 1, -(2 ** 31)
    Y, L = c.check(2, [128, 120, 100], table=table)
    assert (Y[2] == 0).all() and np.isneginf(L[2]).all()
    Y, L = c.check(2, [2 ** 31 - 1, -7, 50], max_len=128)
    assert (Y[1] == 0).all() and np.isneginf(L[1]).all()


def test_the_same_page_named_twice():
    c = Setup(2, 2, 1, 64, 32, 2, "bf16", seed=6)
    c.write(c.rows(64), c.rows(64))
    table = c.table.copy()
    table[1] = table[0, 0]
    c.check(1, [64, 64], table=table)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_far_apart_and_a_given_scale(dtype):
    """Later rows outscore earlier ones by ever more: the running maximum is raised in nearly every tile, for some rows only"""
    c = Setup(1, 4, 2, 64, 32, 8, dtype, seed=7, scale=0.5)
    K, V = c.rows(256), c.rows(256)
    ramp = torch.linspace(0.05, 12, 256, device=U.DEV)[None, None, :, None]
    K = ((K[0].float() * ramp).to(K[0].dtype),) * 2
    K = (K[0], U.to_np64(K[0]))
    c.write(K, V)
    c.check(3, [256])
    c.check(1, [130])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("sizes", [(2.0 ** -19, 1.0), (2.0 ** -21, 2.0 ** -17), (2.0 ** 13, 2.0 ** 10), (2.0 ** 16, 2.0 ** 16), (1e-30, 1e30), (2.0 ** -120, 0.0)])
def test_values_of_any_size(dtype, d, sizes):
    """Scales of V on either side of what f16 holds (2^-19 .. 2^12), the sizes in turn from tile to tile and zeros between: the bound is
    relative to the largest value seen"""
    c = Setup(1, 4, 1, d, 32, 8, dtype, seed=d)
    K = c.rows(250)
    V = c.rng.standard_normal((1, 1, 250, d)).astype(np.float32)
    V *= np.resize(np.repeat(np.float32(sizes), 32), 250)[:, None]
    V[0, 0, 40:50] = 0
    V = (c.dev(V),)
    c.write(K, (V[0], U.to_np64(V[0])))
    c.assert_bytes()
    c.check(1, [250])
    c.check(20, [250])


@pytest.mark.parametrize("B,Hq,Hkv,d,dtype,T,lens,kernel", [
    (1, 8, 2, 128, "bf16", 300, [6500], 2),         # pieces
    (1, 32, 8, 128, "bf16", 200, [5000], 2),        # more workgroups than fit
    (2, 8, 2, 128, "bf16", 511, [9001, 300], 2),    # a sequence shorter than its tokens, which see rows in part or none
    (1, 8, 2, 64, "bf16", 300, [6500], 2),
    (1, 8, 2, 128, "f32", 300, [6500], 2),
    (1, 8, 1, 64, "f32", 65, [20011], 2),
    (1, 32, 4, 128, "bf16", 1, [40001], 1),
    (3, 12, 12, 64, "bf16", 1, [30000, 1, 777], 1),                  # pieces dealt by length, as in those below
    (12, 32, 8, 128, "bf16", 1, [1000] * 5 + [16384] + [1001] * 6, 1),
    (32, 32, 8, 128, "bf16", 1, [600] * 31 + [12000], 1),            # sequences of one piece beside others
    (64, 4, 1, 64, "f32", 1, [40] * 20 + [14000] + [33] * 43, 1),
    (9, 32, 8, 128, "bf16", 6, [7, 12000, 6, 3001, 64, 9, 100, 5, 700], 2),
    (40, 8, 4, 64, "f32", 16, [30, 8192] + [41] * 37 + [3001], 2),
])
def test_many_rows(B, Hq, Hkv, d, dtype, T, lens, kernel):
    """Long caches and many tokens against fp64 on the rows as they are read back; some elements of q 60 times as large as others, some a
    millionth"""
    n = max(lens)
    c = Setup(B, Hq, Hkv, d, 64, -(-n // 64), dtype, seed=T + d)
    assert sa().cache4_plan(c.desc, T, n)[0] == kernel
    g = torch.Generator(device=U.DEV).manual_seed(T)
    K, V = (torch.randn(B, Hkv, n, d, device=U.DEV, generator=g).to(U.tdtype(dtype)) for _ in "KV")
    table = c.dev(c.table)
    sa().sa_cache4_write(c.desc, K, V, None, c.dev(np.array(lens, np.int32)), table, c.pool)
    sa().sa_cache4_read(c.desc, c.pool, table, None, None, K, V)
    q = torch.randn(B, Hq, T, d, device=U.DEV, generator=g)
    q[..., 5] *= 60
    q[..., 37] *= 1e-6
    q, Y, L = c.decode(T, lens, q=q.to(U.tdtype(dtype)))
    for b in range(B):
        m = lens[b]
        k, v, x = K[b, :, :m].double(), V[b, :, :m].double(), q[b].double().view(Hkv, -1, T, d)
        S = (x.reshape(Hkv, -1, d) @ k.transpose(1, 2) * c.scale).view(Hkv, -1, T, m)
        S = S.masked_fill(torch.arange(m, device=U.DEV) > m - T + torch.arange(T, device=U.DEV)[:, None], -torch.inf)
        top = S.amax(-1, keepdim=True).clamp(min=-1e300)
        w = (S - top).exp()
        l = w.sum(-1, keepdim=True)
        Yr = ((w.view(Hkv, -1, m) @ v).view(Hkv, -1, T, d) / l.clamp(min=1e-300)).view(Hq, T, d).cpu().numpy()
        Lr = (top + l.log()).view(Hq, T).cpu().numpy()
        A = c.scale * (x.abs().reshape(Hkv, -1, d) @ k.abs().transpose(1, 2)).amax(-1).view(Hq, T).cpu().numpy()
        delta = (d + 8) * 2.0 ** -24 * A + 2.0 ** -22 * (1 + A)
        p, half = (2.0 ** -12, 2.0 ** -8) if dtype == "bf16" else (2.0 ** -23, 2.0 ** -24)
        tol = half * np.abs(Yr) + ((2 * delta + p + 2 * m * 2.0 ** -24) * float(v.abs().max()))[..., None]
        assert np.isfinite(Y[b]).all() and (np.abs(Y[b] - Yr) <= tol).all(), (np.abs(Y[b] - Yr) - tol).max()
        assert np.array_equal(np.isneginf(L[b]), np.isneginf(Lr))
        seen = np.isfinite(Lr)
        assert (np.abs(L[b][seen] - Lr[seen]) <= (delta + m * 2.0 ** -24 + 2.0 ** -22 * (1 + np.abs(Lr)))[seen]).all()


@pytest.mark.parametrize("what", [float("inf"), float("nan")])
@pytest.mark.parametrize("T,n", [(1, 300), (5, 300), (300, 6500)])
def test_queries_with_infinities_and_nan(what, T, n):
    """Their own results are NaN, the others' are as if they were not there"""
    c = Setup(1, 8, 2, 128, 64, -(-n // 64), "bf16", seed=T)
    c.dev(c.table)
    K, V = (torch.randn(1, 2, n, 128, device=U.DEV).to(torch.bfloat16) for _ in "KV")
    sa().sa_cache4_write(c.desc, K, V, None, None, c.dev(c.table), c.pool)
    q, Y, L = c.decode(T, [n])
    q[0, 3, T // 2, 77] = what
    _, Y2, L2 = c.decode(T, [n], q=q)
    assert np.isnan(Y2[0, 3, T // 2]).all() and np.isnan(L2[0, 3, T // 2])
    Y2[0, 3, T // 2], L2[0, 3, T // 2] = Y[0, 3, T // 2], L[0, 3, T // 2]
    assert np.array_equal(Y, Y2) and np.array_equal(L, L2)


def test_one_cached_row_comes_back_as_it_is():
    c = Setup(1, 4, 2, 128, 32, 1, "bf16", seed=8)
    c.write(c.rows(1), c.rows(1))
    _, V = c.read(1, None, None)
    _, Y, _ = c.decode(1, [1])
    assert np.array_equal(Y[0, :, 0], np.repeat(V[0, :, 0], 2, axis=0))
    q, Y2, L = c.decode(1, [1], lse=False)
    assert L is None and np.array_equal(Y, Y2)


def test_a_sequence_does_not_depend_on_the_others():
    """Alone, in a batch, under another bound of the lengths: within the rounding of differently cut sums; twice: the same bits"""
    c = Setup(3, 8, 2, 128, 64, 8, "bf16", seed=9)
    c.write(c.rows(512), c.rows(512))
    q, Y, L = c.decode(1, [300, 512, 17])
    for lens, bound in (([300, 1, 1], 300), ([300, 512, 17], 512)):
        _, Y2, L2 = c.decode(1, lens, bound, q=q)
        assert np.abs(Y2[0] - Y[0]).max() <= 2.0 ** -7 * np.abs(Y[0]).max()
    assert np.array_equal(Y2, Y) and np.array_equal(L2, L)


@pytest.mark.parametrize("B,Hq,Hkv,d,dtype,T", [(64, 4, 2, 64, "bf16", 1), (33, 32, 8, 128, "bf16", 1), (7, 40, 8, 64, "f32", 5)])
def test_lengths_far_below_their_bound(B, Hq, Hkv, d, dtype, T):
    """Pieces dealt by length, empty sequences and lengths out of range among them, pages missing: as calls for each sequence alone, and the
    same bits twice"""
    n, R = 8192, 64
    c = Setup(B, Hq, Hkv, d, R, n // R, dtype, seed=B)
    assert sa().cache4_dealt(c.desc, T, n) > 0
    g = torch.Generator(device=U.DEV).manual_seed(B)
    lens = c.rng.integers(0, 300, B)
    lens[[0, 2, B - 1]], lens[1], lens[3], lens[4] = 0, 10 ** 9, -5, 5000
    c.table[1, 7] = -1
    table = c.dev(c.table)
    # any codes, with scales of 2^-2 .. 2: what is held is up to 12
    c.pool.copy_(torch.randint(0, 256, c.pool.shape, device=U.DEV, generator=g, dtype=torch.uint8))
    tiles = c.pool.view(-1, 34 * d)
    tiles[:, 32 * d:] = 125 + tiles[:, 32 * d:] % 4
    q = torch.randn(B, Hq, T, d, device=U.DEV, generator=g).to(U.tdtype(dtype))
    _, Y, L = c.decode(T, lens.tolist(), n, q=q)
    _, Y2, L2 = c.decode(T, lens.tolist(), n, q=q)
    assert np.array_equal(Y, Y2) and np.array_equal(L, L2)
    one = sa().make_cache4_desc(1, Hq, Hkv, d, R, c.P, n // R, 1, c.desc.dtype, 0.0)
    ws = torch.empty(max(16, sa().sa_cache4_workspace_bytes(one, sa().SA_OP_CACHE4_DECODE, T)), dtype=torch.uint8, device=U.DEV)
    assert sa().cache4_dealt(one, T, n) == 0
    for b in range(B):
        y, l = torch.empty_like(q[b:b + 1]), torch.empty(1, Hq, T, device=U.DEV)
        sa().sa_cache4_decode_fwd(one, q[b:b + 1].contiguous(), c.pool, table[b:b + 1].contiguous(), c.dev(lens[b:b + 1].astype(np.int32)), n, y, l, ws)
        y, l = U.to_np64(y)[0], l[0].cpu().numpy().astype(np.float64)
        m = min(max(int(lens[b]), 0), n)
        assert np.array_equal(np.isneginf(l), np.isneginf(L[b])) and np.isneginf(l).any() == (m < T or m == 0)
        assert (Y[b][np.isneginf(l)] == 0).all()
        # both sides: probabilities of 11 bits (fp32: 22 or more) and sums of m rows cut differently, values up to 6 * 2; scores and LSE are
        # sums of the same products in the same order, exponentials of arguments up to 128 rounded to 2^-24 of themselves
        p, half = (2.0 ** -12, 2.0 ** -8) if dtype == "bf16" else (2.0 ** -23, 2.0 ** -24)
        tol = 2 * half * np.abs(y) + 2 * 12 * (p + 2 * m * 2.0 ** -24 + 2.0 ** -16)
        assert (np.abs(Y[b] - y) <= tol).all(), (b, np.abs(Y[b] - y).max())
        fine = np.isfinite(l)
        assert (np.abs(L[b][fine] - l[fine]) <= 2 * m * 2.0 ** -24 + 2.0 ** -16).all()


def test_replays_deal_the_pieces_of_their_own_lengths():
    """One recorded call, even lengths and very different ones in turn, each replay against an eager call with a workspace of its own"""
    B, Hq, Hkv, d, n = 16, 16, 4, 64, 16384
    c = Setup(B, Hq, Hkv, d, 64, n // 64, "bf16", seed=3)
    assert sa().cache4_dealt(c.desc, 1, n) > 0
    g = torch.Generator(device=U.DEV).manual_seed(3)
    c.pool.copy_(torch.randint(0, 256, c.pool.shape, device=U.DEV, generator=g, dtype=torch.uint8))
    tiles = c.pool.view(-1, 34 * d)
    tiles[:, 32 * d:] = 125 + tiles[:, 32 * d:] % 4
    q = torch.randn(B, Hq, 1, d, device=U.DEV, generator=g).to(torch.bfloat16)
    lens, table = torch.full((B,), n, dtype=torch.int32, device=U.DEV), c.dev(c.table)
    need = sa().sa_cache4_workspace_bytes(c.desc, sa().SA_OP_CACHE4_DECODE, 1)
    ws, ws2 = (torch.empty(need, dtype=torch.uint8, device=U.DEV) for _ in range(2))
    Y, Y2 = torch.empty_like(q), torch.empty_like(q)
    L, L2 = (torch.empty(B, Hq, 1, device=U.DEV) for _ in range(2))
    sa().sa_cache4_decode_fwd(c.desc, q, c.pool, table, lens, n, Y, L, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sa().sa_cache4_decode_fwd(c.desc, q, c.pool, table, lens, n, Y, L, ws)
    for k, rows in enumerate(([n] * B, [100] * 15 + [n], [0] * 16, [n, 1] * 8, [900 * i for i in range(16)], [n] * B)):
        lens.copy_(torch.tensor(rows, dtype=torch.int32))
        ws2.fill_(255)
        graph.replay()
        sa().sa_cache4_decode_fwd(c.desc, q, c.pool, table, lens, n, Y2, L2, ws2)
        torch.cuda.synchronize()
        assert torch.equal(Y, Y2) and torch.equal(L, L2) and torch.isfinite(Y).all(), k


def test_decode_continues_a_prompt_pass():
    """Attention over rows written and read back equals the framework's dense decoding step on the rows as read."""
    B, Hq, Hkv, d, n = 2, 8, 2, 128, 700
    c = Setup(B, Hq, Hkv, d, 128, 6, "bf16", seed=10)
    K, V = c.rows(n)[0], c.rows(n)[0]
    t = c.dev(c.table)
    sa().sa_cache4_write(c.desc, K, V, None, None, t, c.pool)
    sa().sa_cache4_read(c.desc, c.pool, t, None, None, K, V)
    q, Y, L = c.decode(1, [n, n])
    dense = sa().make_desc(B, Hq, Hkv, n, d, 2)
    ws = torch.empty(sa().sa_workspace_bytes(dense, sa().SA_OP_DECODE), dtype=torch.uint8, device=U.DEV)
    Yd, Ld = torch.empty_like(q), torch.empty(B, Hq, device=U.DEV)
    sa().sa_decode_fwd(dense, q, K, V, n, Yd, Ld, ws)
    torch.cuda.synchronize()
    U.assert_close(Y, U.to_np64(Yd), "bf16", "Y")
    assert np.abs(L[..., 0] - Ld.cpu().numpy()).max() <= 1e-3
