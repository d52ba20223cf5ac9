"""The page tables of the caches held in 4 bits (sa_pages_*) against the oracle's entry-by-entry form: whole numbers and moved bytes,
all equal; and the calls of a serving loop together."""
import numpy as np
import pytest
import torch

from oracle import cache4 as orc
from tests import gpu_util as U

pytestmark = pytest.mark.gpu


def sa():
    from paper_2604_00754_amd import binding
    return binding


class Tables:
    def __init__(self, B, max_pages, spare=4, page_rows=32, layers=2, Hkv=1, d=64, seed=0, lens=None):
        print(f"case pages B{B} max_pages{max_pages} spare{spare} page_rows{page_rows} layers{layers} seed{seed}", flush=True)
        self.rng = np.random.default_rng(seed)
        self.B, self.M, self.P, self.R, self.layers = B, max_pages, B * max_pages + spare, page_rows, layers
        self.lens = self.rng.integers(0, max_pages * page_rows + 1, B).astype(np.int32) if lens is None else np.array(lens, np.int32)
        self.table = np.full((B, max_pages), -1, np.int32)
        ids = iter(self.rng.permutation(self.P))
        for b in range(B):
            for e in range(-(-max(0, int(self.lens[b])) // page_rows)):
                if e < max_pages:
                    self.table[b, e] = next(ids)
        self.refs = self.counts()
        self.desc = sa().make_cache4_desc(B, Hkv, Hkv, d, page_rows, self.P, max_pages, layers)
        size = sa().sa_cache4_pool_bytes(self.desc)
        self.pool = torch.from_numpy(self.rng.integers(0, 256, size, dtype=np.uint8)).to(U.DEV)
        self.host_pool = self.pool.cpu().numpy().reshape(layers, self.P, -1)
        self.info = torch.full((2,), -9, dtype=torch.int32, device=U.DEV)

    def counts(self):
        x = self.table[(self.table >= 0) & (self.table < self.P)]
        return np.bincount(x, minlength=self.P).astype(np.int32)

    def share(self, parents):
        self.table, self.lens, self.refs = orc.fork(parents, self.table, self.lens, self.refs, self.R)

    def ws(self, op):
        return torch.full((sa().sa_cache4_workspace_bytes(self.desc, op, 1),), 255, dtype=torch.uint8, device=U.DEV)

    def move(self, pairs):
        for a, b in pairs:
            self.host_pool[:, b] = self.host_pool[:, a]

    def assert_pool(self):
        assert np.array_equal(self.pool.cpu().numpy().reshape(self.host_pool.shape), self.host_pool)


def dev(x):
    return torch.from_numpy(np.array(x, np.int32)).to(U.DEV)


def same(t, x):
    return np.array_equal(t.cpu().numpy(), np.asarray(x))


def run_fork(t, parents, in_place=False):
    table, lens, refs = dev(t.table), dev(t.lens), dev(t.refs)
    to, lo = torch.full_like(table, 99), torch.full_like(lens, 99)
    ro = refs if in_place else torch.full_like(refs, 99)
    sa().sa_pages_fork(t.desc, dev(parents), table, lens, refs, to, lo, ro)
    want = orc.fork(parents, t.table, t.lens, t.refs, t.R)
    assert same(to, want[0]) and same(lo, want[1]) and same(ro, want[2])
    assert same(table, t.table) and same(lens, t.lens)
    t.table, t.lens, t.refs = want


def run_free(t, keep):
    table, refs = dev(t.table), dev(t.refs)
    sa().sa_pages_free(t.desc, dev(keep), table, refs)
    want = orc.free(keep, t.table, t.refs, t.R)
    assert same(table, want[0]) and same(refs, want[1])
    t.table, t.refs = want


def run_extend(t, lens, add):
    table, refs = dev(t.table), dev(t.refs)
    sa().sa_pages_extend(t.desc, dev(lens), dev(add), table, refs, t.pool, t.info, t.ws(sa().SA_OP_PAGES_EXTEND))
    *want, info, copies = orc.extend(lens, add, t.table, t.refs, t.R)
    assert same(t.info, info), (t.info.tolist(), info)
    assert same(table, want[0]) and same(refs, want[1])
    t.move(copies)
    t.assert_pool()
    t.table, t.refs = want
    return info, copies


def run_compact(t, max_moves, in_place=False):
    table, refs = dev(t.table), dev(t.refs)
    to, ro = (table, refs) if in_place else (torch.full_like(table, 99), torch.full_like(refs, 99))
    sa().sa_pages_compact(t.desc, max_moves, table, refs, to, ro, t.pool, t.info, t.ws(sa().SA_OP_PAGES_COMPACT))
    *want, info, moves = orc.compact(max_moves, t.table, t.refs)
    assert same(t.info, info) and same(to, want[0]) and same(ro, want[1])
    t.move(moves)
    t.assert_pool()
    t.table, t.refs = want
    return info


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B,M,parents", [
    (1, 1, [0]), (1, 3, [-1]), (4, 5, [0, 0, 0, 0]), (4, 5, [1, 2, 3, 0]), (5, 300, [4, -1, 2, 5, 2 ** 31 - 1]), (3, 2, [-(2 ** 31), 1, 1]),
    (70, 7, list(range(35)) * 2),
])
def test_fork(B, M, parents, in_place):
    t = Tables(B, M, seed=B + M)
    run_fork(t, parents, in_place)
    assert same(dev(t.refs), t.counts())
    run_fork(t, parents, in_place)   # pages shared by more than two


def test_fork_of_reserved_and_missing_pages():
    """Entries behind a parent's rows are its own; entries that name no page stay without one; lengths out of range"""
    t = Tables(4, 6, seed=3, lens=[100, 192, 40, 0])
    t.table[0, 5] = 7
    t.table[1, 2], t.table[2, 0] = t.P, -5
    t.refs = t.counts()
    t.lens = np.array([100, 10 ** 9, -3, 0], np.int32)
    run_fork(t, [1, 0, 2, 1])


@pytest.mark.parametrize("B,M,keep", [(1, 1, [0]), (3, 5, [0, 33, 10 ** 9]), (4, 300, [-1, 1, 32, 4000]), (2, 4, [64, 65])])
def test_free(B, M, keep):
    t = Tables(B, M, seed=B + M)
    t.share([max(0, b - 1) for b in range(B)])
    t.table[0, M - 1] = -8
    run_free(t, keep)
    run_free(t, keep)


@pytest.mark.parametrize("B,M,R,lens,add", [
    (1, 1, 32, [0], [1]),
    (3, 4, 32, [0, 31, 32], [1, 1, 1]),                   # a new page, room on the page, past its edge
    (3, 4, 64, [100, 128, 256], [60, 0, 5]),              # over an edge; nothing asked; full
    (4, 3, 32, [90, 5, 96, 64], [100, -3, 2 ** 31 - 1, 2 ** 31 - 1]),
    (2, 100, 32, [10, 1000], [3000, 1500]),               # long prompts: more entries than 16 lanes look at at once
    (80, 3, 32, [20] * 80, [50] * 80),                    # more sequences than are looked at at once
])
def test_extend_without_sharing(B, M, R, lens, add):
    t = Tables(B, M, spare=B * M, page_rows=R, lens=lens)
    info, copies = run_extend(t, lens, add)
    assert info[1] == 0 and not copies
    assert run_extend(t, lens, add)[0] == (0, 0)          # it is there now


@pytest.mark.parametrize("lens,add", [([50, 50, 50], [1, 1, 1]), ([64, 64, 64], [1, 0, 40]), ([50, 20, 50], [100, 1, 0]), ([0, 50, 50], [96, 14, 15])])
def test_extend_copies_shared_pages(lens, add):
    t = Tables(3, 6, spare=20, layers=3, Hkv=2, d=128, lens=[70, 0, 0], seed=sum(lens))
    t.share([0, 0, 0])
    run_extend(t, lens, add)
    run_extend(t, lens, add)


def test_extend_copies_a_page_that_is_held_from_outside():
    t = Tables(1, 3, spare=5, lens=[40])
    t.refs[t.table[0, 1]] += 1
    _, copies = run_extend(t, [40], [1])
    assert len(copies) == 1


def test_extend_with_too_few_pages_changes_nothing():
    t = Tables(2, 8, spare=-12, lens=[32, 32])    # four pages, two in use
    assert run_extend(t, [32, 32], [33, 33])[0] == (0, 2)
    assert run_extend(t, [32, 32], [32, 31])[0] == (2, 0)
    assert run_extend(t, [256, 256], [1, 1])[0] == (0, 0)
    t = Tables(3, 1000, spare=-2990, lens=[5, 0, 0])
    t.share([0, 0, 0])
    assert run_extend(t, [5, 5, 5], [31000] * 3)[0][1] > 0


def test_extend_takes_the_lowest_pages_of_a_large_pool():
    t = Tables(2, 40, spare=20000, layers=1, lens=[1200, 1000])
    t.refs[:17000] = 1
    t.refs[5], t.refs[9999] = 0, -2
    run_extend(t, [1200, 1000], [80, 280])
    assert t.table[0, 38] == 5 and t.table[0, 39] == 9999 and (t.table[1, 32:40] >= 17000).all()


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B,M,spare,max_moves", [(1, 1, 0, 9), (4, 6, 30, 10 ** 9), (4, 6, 30, 3), (4, 6, 30, 0), (30, 40, 9000, 2 ** 31 - 1)])
def test_compact(B, M, spare, max_moves, in_place):
    t = Tables(B, M, spare=spare, layers=2, seed=B + spare)
    t.share([max(0, b - b % 2) for b in range(B)])
    t.table[0, M - 1] = t.P + 3 if M > 1 else t.table[0, M - 1]
    t.refs = t.counts()
    t.refs[-1] += 2     # held from outside
    info = run_compact(t, max_moves, in_place)
    if max_moves > t.P:
        assert (t.refs[:info[0]] > 0).all() and (t.refs[info[0]:] <= 0).all()
        assert run_compact(t, max_moves, in_place)[1] == 0


@pytest.mark.parametrize("used", [0, 1])
def test_compact_of_empty_and_full_pools(used):
    t = Tables(2, 3, spare=0, lens=[96 * used] * 2)
    assert run_compact(t, 100) == (6 * used, 0)


def test_pieces_of_pages_that_end_inside_a_copy():
    """Pages of 3 and 17 KB and of many pieces: the last piece of each is short"""
    for Hkv, d, R in ((1, 64, 32), (4, 128, 32), (5, 128, 128)):
        t = Tables(2, 3, spare=6, page_rows=R, layers=2, Hkv=Hkv, d=d, lens=[2 * R + 1, 0])
        t.share([0, 0])
        run_extend(t, [2 * R + 1, R + 3], [1, 1])
        run_compact(t, 100)


def decode(desc, q, pool, table, lens, max_len):
    need = sa().sa_cache4_workspace_bytes(desc, sa().SA_OP_CACHE4_DECODE, q.shape[2])
    Y = torch.empty_like(q)
    sa().sa_cache4_decode_fwd(desc, q, pool, table, lens, max_len, Y, None, torch.empty(max(need, 16), dtype=torch.uint8, device=U.DEV))
    return Y


def test_pools_beyond_4_gib():
    """Pages whose bytes lie past 2^32 of a layer: written, read, attended to, copied and moved as in a small pool"""
    Hkv, d, R, M, P = 8, 128, 64, 4, 66000
    big, small = (sa().make_cache4_desc(2, 16, Hkv, d, R, p, M, 1) for p in (P, 8))
    assert sa().sa_cache4_pool_bytes(big) > 1.05 * 2 ** 32
    pool = torch.zeros(sa().sa_cache4_pool_bytes(big), dtype=torch.uint8, device=U.DEV)
    near = torch.zeros(sa().sa_cache4_pool_bytes(small), dtype=torch.uint8, device=U.DEV)
    far_table, near_table = dev([[P - 1, 5, P - 2, 61700], [P - 3, P - 1, -1, -1]]), dev([[0, 1, 2, 3], [4, 0, -1, -1]])
    g = torch.Generator(device=U.DEV).manual_seed(3)
    K, V = (torch.randn(2, Hkv, 256, d, device=U.DEV, generator=g).to(torch.bfloat16) for _ in "KV")
    q = torch.randn(2, 16, 3, d, device=U.DEV, generator=g).to(torch.bfloat16)
    counts, lens = dev([256, 64]), dev([250, 100])

    def read(desc, pool, table):
        k, v = torch.zeros_like(K), torch.zeros_like(K)
        sa().sa_cache4_read(desc, pool, table, None, lens, k, v)
        return k, v, decode(desc, q, pool, table, lens, 256)

    for desc, p, table in ((big, pool, far_table), (small, near, near_table)):
        sa().sa_cache4_write(desc, K, V, None, counts, table, p)
    want = read(small, near, near_table)
    for a, b in zip(read(big, pool, far_table), want):
        assert torch.equal(a, b)
    # a page of its own for the second sequence's rows past 100, copied from the last page of the pool into the last but ten
    refs = torch.ones(P, dtype=torch.int32, device=U.DEV)
    refs[P - 1], refs[P - 11] = 2, 0
    info = torch.zeros(2, dtype=torch.int32, device=U.DEV)
    ws = torch.empty(max(sa().sa_cache4_workspace_bytes(big, op) for op in (sa().SA_OP_PAGES_EXTEND, sa().SA_OP_PAGES_COMPACT)), dtype=torch.uint8, device=U.DEV)
    sa().sa_pages_extend(big, lens, dev([0, 9]), far_table, refs, pool, info, ws)
    assert info.tolist() == [1, 0] and far_table.tolist() == [[P - 1, 5, P - 2, 61700], [P - 3, P - 11, -1, -1]]
    for a, b in zip(read(big, pool, far_table), want):
        assert torch.equal(a, b)
    # only the pages in the table stay: they move to the front
    refs.zero_()
    refs[far_table[far_table >= 0].long()] = 1
    sa().sa_pages_compact(big, P, far_table, refs, far_table, refs, pool, info, ws)
    assert info.tolist() == [6, 5] and int(far_table.max()) == 5 and refs.tolist()[:7] == [1] * 6 + [0]
    pool[6 * (pool.numel() // P):] = 255
    for a, b in zip(read(big, pool, far_table), want):
        assert torch.equal(a, b)


def test_a_serving_loop():
    """Prompts, beams that share them, drafted tokens that are taken back, a sequence that ends, compaction in between: after every
    step each sequence's attention is, bit for bit, what a cache of its own with the same rows gives."""
    B, Hq, Hkv, d, R, M, layers, P = 4, 8, 2, 64, 32, 8, 2, 26
    desc = sa().make_cache4_desc(B, Hq, Hkv, d, R, P, M, layers)
    alone = sa().make_cache4_desc(B, Hq, Hkv, d, R, B * M, M, 1)
    g = torch.Generator(device=U.DEV).manual_seed(1)
    normal = lambda *s: torch.randn(s, device=U.DEV, generator=g).to(torch.bfloat16)  # noqa: E731
    pool = torch.full((layers, sa().sa_cache4_pool_bytes(desc) // layers), 255, dtype=torch.uint8, device=U.DEV)
    table, refs = torch.full((B, M), -1, dtype=torch.int32, device=U.DEV), torch.zeros(P, dtype=torch.int32, device=U.DEV)
    lens = torch.zeros(B, dtype=torch.int32, device=U.DEV)
    info = torch.zeros(2, dtype=torch.int32, device=U.DEV)
    ws = torch.empty(max(sa().sa_cache4_workspace_bytes(desc, op) for op in (sa().SA_OP_PAGES_EXTEND, sa().SA_OP_PAGES_COMPACT)),
                     dtype=torch.uint8, device=U.DEV)
    kept = [[[torch.zeros(Hkv, 0, d, device=U.DEV, dtype=torch.bfloat16) for _ in "KV"] for _ in range(layers)] for _ in range(B)]  # dense

    def append(counts):
        nonlocal lens
        T = max(counts)
        sa().sa_pages_extend(desc, lens, dev(counts), table, refs, pool, info, ws)
        assert info.tolist()[1] == 0
        for layer in range(layers):
            K, V = normal(B, Hkv, T, d), normal(B, Hkv, T, d)
            sa().sa_cache4_write(desc, K, V, lens, dev(counts), table, pool[layer])
            for b in range(B):
                for i, x in enumerate((K, V)):
                    kept[b][layer][i] = torch.cat([kept[b][layer][i], x[b, :, :counts[b]]], 1)
        lens = lens + dev(counts)

    def check():
        counted = np.bincount(table[table >= 0].cpu().numpy(), minlength=P)
        assert same(refs, counted)
        n = lens.tolist()
        T = max(max(n), 1)
        for layer in range(layers):
            own = torch.full((sa().sa_cache4_pool_bytes(alone),), 255, dtype=torch.uint8, device=U.DEV)
            own_table = torch.arange(B * M, dtype=torch.int32, device=U.DEV).view(B, M).contiguous()
            K, V = (torch.zeros(B, Hkv, T, d, device=U.DEV, dtype=torch.bfloat16) for _ in "KV")
            for b in range(B):
                assert kept[b][layer][0].shape[1] == n[b]
                K[b, :, :n[b]], V[b, :, :n[b]] = kept[b][layer]
            sa().sa_cache4_write(alone, K, V, None, lens, own_table, own)
            for t in (1, 3):
                q = normal(B, Hq, t, d)
                Y, ref = decode(desc, q, pool[layer], table, lens, T), decode(alone, q, own, own_table, lens, T)
                assert torch.equal(Y, ref)

    def fork(parents):
        nonlocal table, lens, kept
        to, lo = torch.empty_like(table), torch.empty_like(lens)
        sa().sa_pages_fork(desc, dev(parents), table, lens, refs, to, lo, refs)
        table, lens = to, lo
        empty = [[torch.zeros(Hkv, 0, d, device=U.DEV, dtype=torch.bfloat16) for _ in "KV"] for _ in range(layers)]
        kept = [[list(x) for x in (kept[p] if p >= 0 else empty)] for p in parents]

    def compact():
        sa().sa_pages_compact(desc, 1000, table, refs, table, refs, pool, info, ws)
        assert info.tolist()[0] == int((refs > 0).sum()) and (refs[info.tolist()[0]:] == 0).all()

    def cut(n):
        nonlocal lens
        lens = (lens - dev(n)).contiguous()
        sa().sa_pages_free(desc, lens, table, refs)
        for b in range(B):
            for layer in range(layers):
                kept[b][layer] = [x[:, :int(lens[b])] for x in kept[b][layer]]

    append([70, 0, 33, 0])
    check()
    fork([0, 0, 2, 2])
    check()
    for step in range(4):
        append([1, 1, 1, 1])
    check()
    append([5, 5, 0, 5])
    check()
    cut([3, 5, 0, 1])
    check()
    fork([1, 1, -1, 0])
    compact()
    check()
    append([40, 1, 64, 20])
    compact()
    check()


def test_calls_of_a_decoding_step_replay_from_a_graph():
    """Extend, write and attend recorded once, replayed with eager work and a synchronisation in between, against eager calls"""
    B, Hq, Hkv, d, R, M, P = 3, 4, 2, 128, 32, 6, 30
    desc = sa().make_cache4_desc(B, Hq, Hkv, d, R, P, M, 1)
    g = torch.Generator(device=U.DEV).manual_seed(2)
    normal = lambda *s: torch.randn(s, device=U.DEV, generator=g).to(torch.bfloat16)  # noqa: E731
    i32 = {"dtype": torch.int32, "device": U.DEV}

    def fresh():
        s = {"pool": torch.full((sa().sa_cache4_pool_bytes(desc),), 255, dtype=torch.uint8, device=U.DEV), "table": torch.full((B, M), -1, **i32),
             "refs": torch.zeros(P, **i32), "lens": torch.tensor([0, 31, 60], **i32), "one": torch.ones(B, **i32), "info": torch.zeros(2, **i32),
             "K": torch.empty(B, Hkv, 1, d, device=U.DEV, dtype=torch.bfloat16), "V": torch.empty(B, Hkv, 1, d, device=U.DEV, dtype=torch.bfloat16),
             "q": torch.empty(B, Hq, 1, d, device=U.DEV, dtype=torch.bfloat16), "Y": torch.empty(B, Hq, 1, d, device=U.DEV, dtype=torch.bfloat16),
             "ws": torch.empty(max(sa().sa_cache4_workspace_bytes(desc, sa().SA_OP_PAGES_EXTEND), sa().sa_cache4_workspace_bytes(desc, sa().SA_OP_CACHE4_DECODE, 1)),
                               dtype=torch.uint8, device=U.DEV)}
        K = torch.linspace(-1, 1, B * Hkv * 60 * d, device=U.DEV).to(torch.bfloat16).view(B, Hkv, 60, d)
        sa().sa_pages_extend(desc, torch.zeros(B, **i32), s["lens"], s["table"], s["refs"], s["pool"], s["info"], s["ws"])
        sa().sa_cache4_write(desc, K, K.flip(2).contiguous(), None, s["lens"], s["table"], s["pool"])
        return s

    def step(s):
        sa().sa_pages_extend(desc, s["lens"], s["one"], s["table"], s["refs"], s["pool"], s["info"], s["ws"])
        sa().sa_cache4_write(desc, s["K"], s["V"], s["lens"], None, s["table"], s["pool"])
        s["lens"].add_(1)
        sa().sa_cache4_decode_fwd(desc, s["q"], s["pool"], s["table"], s["lens"], M * R, s["Y"], None, s["ws"])

    a, e, warm = fresh(), fresh(), fresh()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step(warm)
    torch.cuda.current_stream().wait_stream(stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a)
    for k in range(40):   # over the edges of pages
        x = {n: normal(*a[n].shape) for n in ("K", "V", "q")}
        for s in (a, e):
            for n in x:
                s[n].copy_(x[n])
        graph.replay()
        step(e)
        torch.cuda.synchronize()
        for n in ("Y", "table", "refs", "lens", "pool", "info"):
            assert torch.equal(a[n], e[n]), (k, n)
