"""Page tables (sa_pages_*) of many sequences and many pages, and whole rounds of a serving loop recorded and replayed, against the oracle's
entry-by-entry form: whole numbers and moved bytes, all equal."""
import numpy as np
import pytest
import torch

from oracle import cache4 as orc
from tests import gpu_util as U
from tests.test_gpu_pages import Tables, dev, run_compact, run_extend, run_fork, run_free, sa, same

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,M,share", [
    (2500, 2, False),     # more sequences than are kept near
    (2500, 2, True),
    (5, 1000, False),     # more pages dealt at once than are kept near
    (1300, 3, True),      # both a second turn of the prefix sums and pages from far away
])
def test_extend_of_many(B, M, share):
    t = Tables(B, M, spare=B, layers=1, lens=[(7 * b) % 50 for b in range(B)], seed=B)
    if share:
        t.share([b - b % 2 for b in range(B)])
    add = [M * 32 if M > 3 else (5 * b) % 40 for b in range(B)]
    info, copies = run_extend(t, t.lens, add)
    assert info[0] > (2048 if M > 3 else 800) and (len(copies) > 500) == share
    assert run_extend(t, t.lens, add)[0] == (0, 0)


@pytest.mark.parametrize("B,M", [(2500, 2), (3, 1500)])
def test_the_other_calls_with_many(B, M):
    t = Tables(B, M, spare=20000, layers=1, seed=B)
    rng = np.random.default_rng(B)
    run_fork(t, rng.integers(-1, B, B).astype(np.int32))
    run_free(t, np.maximum(0, t.lens - rng.integers(0, 40, B)).astype(np.int32))
    assert run_compact(t, 5)[1] == 5
    run_compact(t, 10 ** 9, in_place=True)


def test_rounds_of_beams_replay_from_a_graph():
    """Fork, free, extend, write, attend and compact recorded once.  Parents, rows taken back, rows added and the rows themselves change between
    the replays, with eager work and a synchronisation in between; tables after every round as the oracle's, everything as eager calls give it."""
    B, Hq, Hkv, d, R, M, P, T, layers = 6, 4, 2, 64, 32, 8, 60, 12, 2
    desc = sa().make_cache4_desc(B, Hq, Hkv, d, R, P, M, layers)
    g = torch.Generator(device=U.DEV).manual_seed(5)
    rng = np.random.default_rng(5)
    i32 = {"dtype": torch.int32, "device": U.DEV}
    ws_bytes = max(sa().sa_cache4_workspace_bytes(desc, op) for op in (sa().SA_OP_PAGES_EXTEND, sa().SA_OP_PAGES_COMPACT, sa().SA_OP_CACHE4_DECODE))

    def fresh():
        s = {"pool": torch.full((layers, sa().sa_cache4_pool_bytes(desc) // layers), 255, dtype=torch.uint8, device=U.DEV),
             "table": torch.full((B, M), -1, **i32), "refs": torch.zeros(P, **i32), "lens": torch.zeros(B, **i32), "info": torch.zeros(2, **i32),
             "info2": torch.zeros(2, **i32), "parents": torch.arange(B, **i32), "cut": torch.zeros(B, **i32), "add": torch.zeros(B, **i32),
             "ws": torch.zeros(ws_bytes, dtype=torch.uint8, device=U.DEV)}
        for name in ("table", "refs", "lens"):
            s[name + "2"] = torch.zeros_like(s[name])
        s["keep"] = torch.zeros_like(s["lens"])
        for name, heads, n in (("K", Hkv, T), ("V", Hkv, T), ("q", Hq, 1), ("Y", Hq, 1)):
            s[name] = torch.zeros(layers, B, heads, n, d, device=U.DEV, dtype=torch.bfloat16)
        return s

    def step(s):
        sa().sa_pages_fork(desc, s["parents"], s["table"], s["lens"], s["refs"], s["table2"], s["lens2"], s["refs2"])
        torch.sub(s["lens2"], s["cut"], out=s["keep"])
        torch.clamp(s["keep"], min=0, out=s["keep"])
        sa().sa_pages_free(desc, s["keep"], s["table2"], s["refs2"])
        sa().sa_pages_extend(desc, s["keep"], s["add"], s["table2"], s["refs2"], s["pool"], s["info"], s["ws"])
        torch.add(s["keep"], s["add"], out=s["lens"])
        for layer in range(layers):
            sa().sa_cache4_write(desc, s["K"][layer], s["V"][layer], s["keep"], s["add"], s["table2"], s["pool"][layer])
            sa().sa_cache4_decode_fwd(desc, s["q"][layer], s["pool"][layer], s["table2"], s["lens"], M * R, s["Y"][layer], None, s["ws"])
        sa().sa_pages_compact(desc, 1000, s["table2"], s["refs2"], s["table"], s["refs"], s["pool"], s["info2"], s["ws"])

    a, e, warm = fresh(), fresh(), fresh()
    step(warm)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a)
    table, refs, lens = np.full((B, M), -1, np.int32), np.zeros(P, np.int32), np.zeros(B, np.int32)
    for k in range(60):
        parents = np.arange(B) if k % 3 else rng.integers(0 if k % 2 else -1, B, B)
        table, lens, refs = orc.fork(parents, table, lens, refs, R)
        cut = rng.integers(0, 5, B)
        keep = np.maximum(lens - cut, 0)
        table, refs = orc.free(keep, table, refs, R)
        add = np.minimum(rng.integers(0, T + 1, B) if k else np.full(B, T), M * R - keep)
        table, refs, info, _ = orc.extend(keep, add, table, refs, R)
        assert info[1] == 0
        lens = (keep + add).astype(np.int32)
        table, refs, info2, _ = orc.compact(1000, table, refs)
        x = {"parents": dev(parents), "cut": dev(cut), "add": dev(add)}
        for name in ("K", "V", "q"):
            x[name] = torch.randn(a[name].shape, device=U.DEV, generator=g).to(torch.bfloat16)
        for s in (a, e):
            for name in x:
                s[name].copy_(x[name])
        graph.replay()
        step(e)
        torch.cuda.synchronize()
        for name in ("Y", "table", "refs", "lens", "pool", "info", "info2"):
            assert torch.equal(a[name], e[name]), (k, name)
        assert same(a["table"], table) and same(a["refs"], refs) and same(a["lens"], lens), k
        assert same(a["info"], info) and same(a["info2"], info2), k
        assert torch.isfinite(a["Y"].float()).all()
