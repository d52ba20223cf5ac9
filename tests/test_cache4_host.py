"""Caches held in 4 bits, without a GPU: the oracle against facts about the format, and the refusals of the entry points."""
import ctypes as C

import numpy as np
import pytest

from oracle import cache4 as orc
from paper_2604_00754_amd import binding as sa

FAKE = C.c_void_p(4096)  # never dereferenced: every call below fails validation first
FAR = C.c_void_p(1 << 40)


# ---- the oracle ---------------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("e", [-125, -20, 0, 5, 120])
def test_what_the_format_holds_stays_as_it_is(e):
    x = np.array([s * m * 2.0 ** e for s in (1, -1) for m in orc.MAGNITUDES] * 2)
    (codes, byte), _ = orc.quantise_row(x, x)
    assert byte == [e + 127] and [orc.value(c, byte[0]) for c in codes] == list(x)


def test_ties_go_to_the_even_code_and_the_scale_turns_at_seven():
    codes = [orc.element_code(v, 0) for v in (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.5)]
    assert codes == [0, 2, 2, 4, 4, 6, 6, 7]
    assert orc.block_exponent(7.0) == 0 and orc.block_exponent(np.nextafter(7.0, 8)) == 1
    assert orc.block_exponent(4.0) == 0 and orc.block_exponent(np.nextafter(4.0, 0)) == 0  # 3.99.. / 2^-1 > 7
    assert orc.block_exponent(3.5) == -1 and orc.block_exponent(2.0 ** -149) == -125 and orc.block_exponent(0.0) == 0


def test_normal_rows_are_held_as_well_as_the_better_of_two_powers_holds_them():
    """Relative error 0.112 of N(0,1) rows, within 1 % of choosing the power of every block by its error."""
    x = np.random.default_rng(0).standard_normal((300, 32))
    err = best = 0.0
    for row in x:
        by = {}
        e = orc.block_exponent(np.abs(row).max())
        for k in (e - 1, e, e + 1):
            by[k] = sum((orc.value(orc.element_code(v, k), k + 127) - v) ** 2 for v in row)
        err += by[e]
        best += min(by.values())
    assert err <= 1.02 * best and np.sqrt(err / (x ** 2).sum()) < 0.115


def test_the_largest_numbers_are_held_as_numbers():
    for amax in (7 * 2.0 ** 125, np.nextafter(7 * 2.0 ** 125, np.inf), float(np.finfo(np.float32).max)):
        e = orc.block_exponent(amax)
        assert e == 125 and orc.value(orc.element_code(amax, e), e + 127) == 6 * 2.0 ** 125


@pytest.mark.parametrize("spread", [0, 1, 3, 30, 120])
def test_blocks_at_once_and_element_by_element(spread):
    rng = np.random.default_rng(spread)
    x = rng.choice([-1, 1], (200, 32)) * (1 + rng.integers(0, 128, (200, 32)) / 128) * 2.0 ** rng.integers(-126 + spread, 128 - spread // 2, (200, 1))
    x = x.astype(np.float32).astype(np.float64) * 2.0 ** -rng.integers(0, spread + 1, (200, 32)).astype(np.float64)
    x[rng.random(x.shape) < 0.1] = 0
    x[0], x[1, 1:], x[2] = 0, 0, -0.0
    e = [orc.block_exponent(np.abs(b).max()) for b in x]
    want = np.array([[orc.value(orc.element_code(v, k), k + 127) for v in b] for b, k in zip(x, e)])
    got = orc.blocks_held(x)
    assert np.array_equal(got, want) and np.array_equal(np.signbit(got), np.signbit(want))


@pytest.mark.parametrize("d", [64, 128])
def test_every_byte_of_a_tile_has_one_place(d):
    c = orc.Cache(1, d, 32, 1)
    places = np.concatenate([np.concatenate(c._places(r)) for r in range(32)])
    assert sorted(places) == list(range(34 * d))


# ---- refusals -----------------------------------------------------------------------------------------------------------------


def desc(**kw):
    a = dict(B=2, Hq=8, Hkv=2, d=128, page_rows=64, pages=40, max_pages=16, layers=3, dtype=sa.SA_BF16, scale=0.0)
    a.update(kw)
    return sa.make_cache4_desc(**a)


def calls(d, **kw):
    """Every entry point with good arguments but those in kw, by name -> status"""
    a = dict(K=FAKE, V=FAKE, T=5, starts=FAKE, counts=FAKE, table=FAKE, pool=FAKE, q=FAKE, lens=FAKE, max_len=1000, Y=FAKE, LSE=FAKE, ws=FAKE,
             ws_bytes=1 << 40, parents=FAKE, refs=FAKE, table_out=FAR, lens_out=FAR, refs_out=FAKE, keep=FAKE, add=FAKE, info=FAKE, max_moves=9)
    a.update(kw)
    p = C.byref(d) if d is not None else None
    lib = sa.raw()
    order = {"sa_cache4_write": "K V T starts counts table pool", "sa_cache4_read": "pool table T starts counts K V",
             "sa_cache4_decode_fwd": "q T pool table lens max_len Y LSE ws ws_bytes",
             "sa_pages_fork": "parents table lens refs table_out lens_out refs_out", "sa_pages_free": "keep table refs",
             "sa_pages_extend": "lens add table refs pool info ws ws_bytes",
             "sa_pages_compact": "max_moves table refs table_out refs_out pool info ws ws_bytes"}
    out = {}
    for name, args in order.items():
        args = args.split()
        if not kw or any(k in args for k in kw):
            out[name] = getattr(lib, name)(p, *[a[k] for k in args], None)
    return out


def test_null_descriptor():
    assert set(calls(None).values()) == {sa.SA_ERR_NULL}


@pytest.mark.parametrize("field,value,status", [
    ("B", 0, sa.SA_ERR_SHAPE), ("Hq", 0, sa.SA_ERR_SHAPE), ("Hkv", 3, sa.SA_ERR_SHAPE), ("pages", 0, sa.SA_ERR_SHAPE),
    ("max_pages", 0, sa.SA_ERR_SHAPE), ("layers", 0, sa.SA_ERR_SHAPE), ("layers", -1, sa.SA_ERR_SHAPE), ("scale", float("inf"), sa.SA_ERR_SHAPE),
    ("scale", float("nan"), sa.SA_ERR_SHAPE), ("d", 96, sa.SA_ERR_UNSUPPORTED), ("dtype", 2, sa.SA_ERR_UNSUPPORTED),
    ("page_rows", 16, sa.SA_ERR_UNSUPPORTED), ("page_rows", 96, sa.SA_ERR_UNSUPPORTED), ("page_rows", 2048, sa.SA_ERR_UNSUPPORTED),
    ("page_rows", 0, sa.SA_ERR_UNSUPPORTED), ("page_rows", -64, sa.SA_ERR_UNSUPPORTED),
    ("max_pages", (1 << 30) // 64 + 1, sa.SA_ERR_SHAPE), ("B", 1 << 27, sa.SA_ERR_SHAPE), ("pages", 1 << 29, sa.SA_ERR_SHAPE),
    ("B", 65536, sa.SA_ERR_SHAPE), ("layers", 65536, sa.SA_ERR_SHAPE), ("Hkv", 2 * 123362, sa.SA_ERR_SHAPE),
])
def test_bad_descriptors(field, value, status):
    d = desc(**{field: value}, **({"Hq": value} if field == "Hkv" and value > 3 else {}))
    assert set(calls(d).values()) == {status}
    assert sa.sa_cache4_pool_bytes(d) == 0 and sa.sa_cache4_workspace_bytes(d, sa.SA_OP_CACHE4_DECODE, 1) == 0


@pytest.mark.parametrize("arg", "K V table pool q lens Y parents refs table_out lens_out refs_out keep add info".split())
def test_null_arguments(arg):
    got = calls(desc(), **{arg: None})
    assert got and set(got.values()) == {sa.SA_ERR_NULL}


@pytest.mark.parametrize("arg", "K V pool q Y ws".split())
def test_addresses_off_the_16_byte_grid(arg):
    got = calls(desc(), **{arg: C.c_void_p(4096 + 8)})
    assert got and set(got.values()) == {sa.SA_ERR_UNSUPPORTED}


@pytest.mark.parametrize("arg", "table lens LSE starts counts parents refs table_out lens_out keep add info".split())
def test_addresses_off_the_4_byte_grid(arg):
    got = calls(desc(), **{arg: C.c_void_p(4096 + 2)})
    assert got and set(got.values()) == {sa.SA_ERR_UNSUPPORTED}


def test_token_counts_and_lengths():
    for T in (0, -1):
        assert set(calls(desc(), T=T).values()) == {sa.SA_ERR_SHAPE}
        assert sa.sa_cache4_workspace_bytes(desc(), sa.SA_OP_CACHE4_DECODE, T) == 0
    assert set(calls(desc(), T=1 << 28).values()) == {sa.SA_ERR_SHAPE}  # 2 * 8 * 2^28 rows
    for n in (0, -5, 16 * 64 + 1):
        assert set(calls(desc(), max_len=n).values()) == {sa.SA_ERR_SHAPE}
    assert set(calls(desc(), max_moves=-1).values()) == {sa.SA_ERR_SHAPE}


def test_workspaces():
    d = desc(B=1, Hq=32, Hkv=8, max_pages=512, pages=512)
    need = sa.sa_cache4_workspace_bytes(d, sa.SA_OP_CACHE4_DECODE, 1)
    assert need > 0
    for op, name in ((sa.SA_OP_CACHE4_DECODE, "sa_cache4_decode_fwd"), (sa.SA_OP_PAGES_EXTEND, "sa_pages_extend"),
                     (sa.SA_OP_PAGES_COMPACT, "sa_pages_compact")):
        need = sa.sa_cache4_workspace_bytes(d, op, 5)
        assert need > 0 and calls(d, ws_bytes=need - 1)[name] == sa.SA_ERR_WORKSPACE and calls(d, ws=None)[name] == sa.SA_ERR_WORKSPACE
    assert sa.sa_cache4_workspace_bytes(d, 99, 1) == 0


@pytest.mark.parametrize("B,Hq,Hkv,d,dtype,T,n,kernel,pieces", [
    (1, 32, 8, 128, 0, 1, 300, 1, 1),          # three tiles a wave at most: one launch
    (1, 32, 8, 128, 0, 1, 1100, 1, 5),         # a tile a wave
    (1, 32, 4, 128, 0, 1, 131072, 1, 64),      # two waves a SIMD
    (16, 32, 8, 128, 0, 1, 8192, 1, 2),
    (64, 16, 16, 64, 0, 1, 131072, 1, 8),      # 64 tiles a wave and no more
    (4, 32, 8, 128, 0, 5, 8192, 2, 8),         # one wave a SIMD
    (1, 32, 8, 128, 0, 64, 32768, 2, 8),       # two
    (1, 32, 8, 128, 0, 509, 32768, 2, 2),      # two whole rounds
    (1, 32, 8, 128, 1, 509, 32768, 2, 2),
    (1, 16, 16, 64, 0, 512, 512, 2, 1),
    (1, 2, 1, 128, 0, 2000, 1 << 20, 2, 64),   # 128 tiles a wave and no more
])
def test_how_attention_is_dealt(B, Hq, Hkv, d, dtype, T, n, kernel, pieces):
    c = desc(B=B, Hq=Hq, Hkv=Hkv, d=d, dtype=dtype, max_pages=-(-n // 64), pages=100)
    assert sa.cache4_plan(c, T, n) == (kernel, pieces)


@pytest.mark.parametrize("B,Hq,Hkv,T,n,pieces,dealt", [
    (1, 32, 8, 1, 32768, 32, 0),     # alone
    (16, 32, 8, 1, 8192, 2, 2),
    (12, 32, 8, 1, 16384, 3, 3),
    (2, 32, 8, 1, 20000, 16, 0),     # few tiles a wave
    (32, 32, 8, 1, 12000, 1, 2),     # a slot more
    (32, 32, 8, 1, 4000, 1, 0),
    (64, 32, 8, 1, 32768, 2, 2),
    (65, 32, 8, 1, 32768, 2, 0),     # more sequences than lanes
    (12, 32, 8, 6, 16384, 5, 5),
    (12, 32, 8, 16, 16384, 5, 0),    # two blocks of query rows
])
def test_where_pieces_may_be_dealt_by_length(B, Hq, Hkv, T, n, pieces, dealt):
    c = desc(B=B, Hq=Hq, Hkv=Hkv, d=128, max_pages=-(-n // 64), pages=100)
    assert sa.cache4_plan(c, T, n) == (1 if T == 1 else 2, pieces) and sa.cache4_dealt(c, T, n) == dealt
    if dealt:
        assert sa.sa_cache4_workspace_bytes(c, sa.SA_OP_CACHE4_DECODE, T) >= 512 + B * Hq * T * dealt * 130 * 4


def test_workspaces_cover_every_length():
    rng = np.random.default_rng(0)
    for _ in range(300):
        Hkv, g, M = int(rng.integers(1, 9)), int(rng.integers(1, 9)), int(np.exp(rng.uniform(0, 8)))
        c = desc(B=int(rng.integers(1, 20)), Hq=Hkv * g, Hkv=Hkv, d=int(rng.choice([64, 128])), dtype=int(rng.integers(0, 2)), max_pages=M, pages=9)
        T = int(np.exp(rng.uniform(0, 6)))
        need = sa.sa_cache4_workspace_bytes(c, sa.SA_OP_CACHE4_DECODE, T)
        for n in {1, 64 * M, *np.exp(rng.uniform(0, np.log(64 * M), 20)).astype(int).tolist()}:
            kernel, pieces = sa.cache4_plan(c, T, n)
            tiles, waves = -(-n // 32), 8 if kernel == 1 else 4
            assert pieces <= -(-tiles // waves) and -(-tiles // pieces) <= waves * (64 if kernel == 1 else 128)
            assert pieces == 1 or need >= c.B * c.Hq * T * pieces * (c.d + 2) * 4
            slots = sa.cache4_dealt(c, T, n)
            assert slots == 0 or slots >= pieces and need >= 512 + c.B * c.Hq * T * slots * (c.d + 2) * 4


@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 33, 40])
def test_rows_that_are_loaded_are_rows_that_are_written(T):
    """Whatever start and count are: no row in front of the sequence's or past its count is touched, a sequence without rows touches none"""
    for start in [*range(64), -1, -20, -32, -33, 2 ** 31 - 1, -(2 ** 31)]:
        for count in [*range(T + 1), -1, -(2 ** 31), T + 1, 2 ** 31 - 1]:
            rows = min(max(count, 0), T)
            seen = set()
            for half in sa.cache4_loaded_rows(start, count, T):
                assert half is None or 0 <= min(half) and max(half) < rows, (start, count, half)
                seen.update(half or ())
            assert seen == set(range(rows)), (start, count)


def test_outputs_that_overlap_inputs():
    d = desc()
    name = "sa_pages_fork"
    assert calls(d, table_out=FAKE)[name] == sa.SA_ERR_UNSUPPORTED
    assert calls(d, table_out=C.c_void_p(4096 + 2 * 16 * 4 - 4))[name] == sa.SA_ERR_UNSUPPORTED
    assert calls(d, lens_out=C.c_void_p(4096 + 4))[name] == sa.SA_ERR_UNSUPPORTED
    assert calls(d, refs_out=C.c_void_p(4096 - 4))[name] == sa.SA_ERR_UNSUPPORTED
    name = "sa_pages_compact"
    assert calls(d, table_out=C.c_void_p(4096 + 4))[name] == sa.SA_ERR_UNSUPPORTED
    assert calls(d, refs_out=C.c_void_p(4096 + 39 * 4))[name] == sa.SA_ERR_UNSUPPORTED


def test_sizes_at_their_limits():
    """Accepted: the next argument error is what is reported (sizes are judged before the tensors)"""
    for d in (desc(B=65535, max_pages=16), desc(layers=65535), desc(pages=(1 << 31) // 4 - 1, layers=1), desc(max_pages=(1 << 30) // 64, B=1),
              desc(Hkv=123361, Hq=123361, page_rows=64, B=1, pages=2, layers=1)):
        assert set(calls(d, table=None).values()) == {sa.SA_ERR_NULL} and sa.sa_cache4_pool_bytes(d) > 0
    for d in (desc(pages=40000, layers=60000), desc(pages=1 << 30, Hkv=1, layers=1)):
        assert set(calls(d, table=None).values()) == {sa.SA_ERR_SHAPE}


def test_calls_that_need_more_workgroups_than_a_launch_holds():
    d = desc(B=1, Hq=1, Hkv=1, max_pages=1 << 24, layers=1)
    got = calls(d, T=(1 << 31) - 1)
    assert got["sa_cache4_write"] == got["sa_cache4_read"] == sa.SA_ERR_UNSUPPORTED


def test_pool_size():
    assert sa.sa_cache4_pool_bytes(desc()) == 3 * 40 * 2 * 2 * 34 * 128
    # a quarter of the bf16 rows, and a sixteenth of that for the scales
    assert 34 * 128 * 16 == 17 * (2 * 32 * 128 * 2) // 4


def test_binding_raises_with_status():
    import torch
    x = torch.zeros(1, 1, 1, 64, dtype=torch.bfloat16)
    t = torch.zeros(1, 1, dtype=torch.int32)
    with pytest.raises(sa.SaError) as e:
        sa.sa_cache4_write(desc(d=32), x, x, None, None, t, x)
    assert e.value.status == sa.SA_ERR_UNSUPPORTED and "sa_cache4_write" in str(e.value)
