"""The operators of a K/V cache held in 4 bits and in pages, as cases to be timed.

A case is one pass of one of four kinds:
  write    rows of K and V go into the cache and come back as the values that it stands for
  attend   T query tokens of every sequence attend to the cache, themselves included
  step     a round of beam search or of drafted tokens: the page tables are dealt anew (fork), pages past the rows that stay are
           given back (free), the next rows get room (extend, which copies pages that are shared)
  compact  the pages in use move to the front of the pool

Format: an element is E2M1 (sign, magnitudes 0 .5 1 1.5 2 3 4 6), 32 elements of a row share a power of two, held as a byte e + 127.
A tile holds 32 rows of a head: K codes [row][d/2] | V codes [g 4][r 16][half 2][i 4][d/32], row 16 half + 4 g + i, bytes r d/32 .. of it |
K scales [d/32][row % 16][row / 16] | V scales [d/32][g][half][i].  A page is [Hkv][page_rows/32] tiles, a pool [layers][pages] of them.
"""
import math

import torch

own = False

# (query heads, KV heads, head size) of the configurations in synth.WORKLOADS
HEADS = [(32, 8, 128), (32, 4, 128), (12, 12, 64), (16, 16, 64)]


def _case(kind, B, heads, cap, **more):
    c = {"kind": kind, "B": B, "Hq": heads[0], "Hkv": heads[1], "d": heads[2], "cap": cap, "page_rows": 64, "layers": 1, "dtype": "bf16",
         "T": 1, "len": cap, "varlen": False, "spare": 0}
    c.update(more)
    return c


def listed():
    grouped8, grouped4, small12, wide16 = HEADS
    cases = [
        # one generated token of each sequence of a serving batch goes into the cache
        ("write_token", _case("write", 16, grouped8, 8192, varlen=True)),
        # the long prompt goes into the cache
        ("write_prompt", _case("write", 1, grouped8, 32768, T=32768)),
        # fp32 rows, prompts of different odd lengths behind rows that are there already
        ("write_f32", _case("write", 3, wide16, 4096, T=2039, len=3950, varlen=True, dtype="f32")),
        # a token generated early in a conversation: the smallest call
        ("attend_early", _case("attend", 1, grouped8, 32768, len=1100)),
        # a serving batch whose sequences have different lengths
        ("attend_batch", _case("attend", 16, grouped8, 8192, varlen=True)),
        # the token after the longest prompt
        ("attend_128k", _case("attend", 1, grouped4, 131072)),
        # five drafted tokens of each sequence are looked at together, fp32, one query head per KV head
        ("attend_draft", _case("attend", 4, wide16, 4096, T=5, len=2039, varlen=True, dtype="f32")),
        # a follow-up question to the long prompt
        ("attend_question", _case("attend", 1, grouped8, 32768, T=509)),
        # four beams of one layer, short pages
        ("step_beams", _case("step", 4, small12, 2048, len=1500, page_rows=32, spare=16)),
        # a batch of forty sequences, four layers of caches
        ("step_batch", _case("step", 40, grouped8, 8192, len=4800, layers=4, spare=100)),
        # a small pool after some sequences have ended
        ("compact_small", _case("compact", 6, small12, 2048, len=1000, page_rows=32, spare=100)),
        # a pool of four layers, half of it in use
        ("compact_large", _case("compact", 24, grouped8, 4096, len=3900, layers=4, spare=1000)),
    ]
    return [dict(c, name=name) for name, c in cases]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        c = _draw(rng)
        if _cost(c) <= most:
            return c


def _draw(rng):
    kind = rng.choice(["write", "write", "attend", "attend", "attend", "step", "compact"])
    heads, page_rows = rng.choice(HEADS), rng.choice([32, 64, 128, 256])
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    if kind in ("step", "compact"):
        cap = _log_int(rng, 2, 64) * page_rows
        return _case(kind, rng.randint(2, 40), heads, cap, page_rows=page_rows, len=_log_int(rng, page_rows, cap), layers=rng.randint(1, 4),
                     spare=rng.randint(40, 400), varlen=rng.random() < 0.7)
    n = _log_int(rng, 1, 131072)
    B = rng.randint(1, max(1, min(24, 131072 // n)))
    cap = -(-rng.randint(n, 2 * n) // page_rows) * page_rows
    if kind == "write":
        T = 1 if rng.random() < 0.4 else _log_int(rng, 1, n)
    else:
        T = rng.choice([1, 1, 1, _log_int(rng, 1, min(n, 16)), _log_int(rng, 1, min(n, 512))])
    return _case(kind, B, heads, cap, page_rows=page_rows, len=n, T=T, dtype=dtype, varlen=B > 1 and rng.random() < 0.7)


class _State:
    pass


def _tdtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _page_bytes(c):
    return c["Hkv"] * (c["page_rows"] // 32) * 34 * c["d"]


def _pages(c):
    return c["B"] * (c["cap"] // c["page_rows"]) + c["spare"]


def prepare(case, seed):
    c, s = case, _State()
    s.case = c
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    B, Hq, Hkv, d, T, R = c["B"], c["Hq"], c["Hkv"], c["d"], c["T"], c["page_rows"]
    M, P = c["cap"] // R, _pages(c)
    i32 = {"device": dev, "dtype": torch.int32}

    def normal(*shape, dtype=torch.float32):
        return torch.randn(shape, device=dev, generator=g).to(dtype)

    # rows of every sequence: `len`, or from a quarter of that upwards with one sequence of that length
    lens = torch.full((B,), c["len"], **i32)
    if c["varlen"]:
        lens = torch.randint(max(1, min(T if c["kind"] == "attend" else 1, c["len"]), c["len"] // 4), c["len"] + 1, (B,), generator=g, **i32)
        lens[seed % B] = c["len"]
    s.lens, s.max_len = lens, c["len"]
    own_pages = torch.randperm(P, device=dev, generator=g)[:B * M].to(torch.int32).view(B, M)
    entry = torch.arange(M, device=dev)
    s.table = own_pages.contiguous()
    if c["kind"] in ("write", "attend"):
        shape = (P, Hkv, R // 32, 34 * d)
        s.pool = torch.empty(shape, device=dev, dtype=torch.uint8)
        if c["kind"] == "write":
            s.K, s.V = normal(B, Hkv, T, d, dtype=_tdtype(c)), normal(B, Hkv, T, d, dtype=_tdtype(c))
            s.counts = lens.clamp(max=T)  # prompts shorter than T end early
            s.starts = (lens - s.counts).contiguous()
            s.K_out, s.V_out = torch.zeros_like(s.K), torch.zeros_like(s.V)
            s.pool.zero_()
        else:
            s.q = normal(B, Hq, T, d, dtype=_tdtype(c))
            s.Y = torch.empty_like(s.q)
            s.LSE = torch.empty(B, Hq, T, device=dev, dtype=torch.float32)
            tile = s.pool.view(-1, 34 * d)
            step = max(1, (1 << 26) // (32 * d))
            for at in range(0, tile.shape[0], step):  # N(0, 1) rows, held in 4 bits
                n = min(step, tile.shape[0] - at)
                tile[at:at + n] = _tiles(normal(n, 32, d), normal(n, 32, d))
        s.ws = None
        return s

    # page tables: pages behind the rows in use are not there
    have = entry < ((lens + R - 1) // R)[:, None]
    s.table = torch.where(have, s.table, -1).contiguous()
    s.refs = _counts(s.table, P).to(torch.int32)
    s.pool = torch.randint(0, 1 << 62, (c["layers"], P, _page_bytes(c) // 8), device=dev, generator=g, dtype=torch.int64).view(torch.uint8)
    s.table_out, s.refs_out = torch.empty_like(s.table), torch.empty_like(s.refs)
    s.info = torch.zeros(2, **i32)
    if c["kind"] == "step":
        # every second sequence, in an order of the seed's, becomes a copy of the one before it
        order = torch.randperm(B, device=dev, generator=g).to(torch.int32)
        s.parents = torch.arange(B, **i32)
        s.parents[order[1::2].long()] = order[0:2 * (B // 2):2]
        s.lens_out = torch.empty_like(lens)
        new = lens[s.parents.long()]
        cut = torch.randint(0, 6, (B,), generator=g, **i32)  # drafted tokens that are not kept
        s.keep = (new - cut).clamp(min=0).contiguous()
        s.add = torch.randint(1, 6, (B,), generator=g, **i32)
    else:
        s.max_moves = P
    s.ws = None
    return s


# ---- the format, in elementary operations -------------------------------------------------------------------------------------


def _power(byte):
    """2^(byte - 127) in fp32, exact"""
    return torch.exp2(torch.arange(-127, 129, device=byte.device, dtype=torch.float64)).float()[byte.int()].unsqueeze(-1)


def _quantise(x):
    """fp32 [..., d] -> codes 0..15 and scale bytes [..., d/32]"""
    x = x.unflatten(-1, (-1, 32))
    m, ex = torch.frexp(x.abs().amax(-1))  # amax = m 2^ex, m in [0.5, 1)
    byte = (ex - 3 + 127 + (m > 0.875).to(ex.dtype)).clamp(2, 254)
    v = x.abs() / _power(byte)
    code = ((v > 0.25).int() + (v >= 0.75).int() + (v > 1.25).int() + (v >= 1.75).int() + (v > 2.5).int() + (v >= 3.5).int() + (v > 5).int())
    return (code + 8 * (x < 0).int()).flatten(-2), byte


def _values(code, byte):
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], device=code.device)
    return (grid[code].unflatten(-1, (-1, 32)) * _power(byte)).flatten(-2)


def _tiles(K, V):
    """[n, 32, d] rows -> [n, 34 d] bytes"""
    n, _, d = K.shape
    out = []
    for x in (K, V):
        code, byte = _quantise(x)
        out += [(code[..., 0::2] | (code[..., 1::2] << 4)).to(torch.uint8), byte.to(torch.uint8)]
    kc, ks, vc, vs = out
    vc = vc.view(n, 2, 4, 4, 16, d // 32).permute(0, 2, 4, 1, 3, 5)  # half g i r b -> g r half i b
    ks = ks.view(n, 2, 16, d // 32).permute(0, 3, 2, 1)
    vs = vs.view(n, 2, 4, 4, d // 32).permute(0, 4, 2, 1, 3)
    return torch.cat([x.reshape(n, -1) for x in (kc, vc, ks, vs)], 1)


def _rows(pool, table, n, c):
    """The first n rows of every sequence as fp32 K, V [B, Hkv, n', d], n' = whole pages"""
    B, Hkv, d, R = c["B"], c["Hkv"], c["d"], c["page_rows"]
    t = pool[table[:, :-(-n // R)].long()]  # [B, pages, Hkv, tiles, 34 d]
    t = t.permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, 34 * d)
    two = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], device=t.device)
    two = torch.stack([two.repeat(16), two.repeat_interleave(16)], 1)  # both values of a byte
    lead = t.shape[:3]
    kc, vc, ks, vs = t[..., :16 * d], t[..., 16 * d:32 * d], t[..., 32 * d:33 * d], t[..., 33 * d:]
    vc = vc.reshape(*lead, 4, 16, 2, 4, d // 32).permute(0, 1, 2, 5, 3, 6, 4, 7)  # half g i r b
    ks = ks.reshape(*lead, d // 32, 16, 2).permute(0, 1, 2, 5, 4, 3)
    vs = vs.reshape(*lead, d // 32, 4, 2, 4).permute(0, 1, 2, 5, 4, 6, 3)
    out = []
    for code, scale in ((kc, ks), (vc, vs)):
        x = two[code.reshape(*lead, 32, d // 2).int()].reshape(*lead, 32, d // 32, 32)
        out.append((x * _power(scale.reshape(*lead, 32, d // 32))).reshape(B, Hkv, -1, d))
    return out


# ---- the plain forms ----------------------------------------------------------------------------------------------------------


def _plain_write(s):
    c = s.case
    t = torch.arange(c["T"], device=s.K.device)
    at = s.starts.long()[:, None] + t
    seen = (t < s.counts[:, None]) & (at >= 0) & (at < c["cap"])
    for x, y in ((s.K, s.K_out), (s.V, s.V_out)):
        back = _values(*_quantise(x.float())).to(x.dtype)
        torch.where(seen[:, None, :, None], back, y, out=y)
    return {"K": s.K_out, "V": s.V_out}


def _plain_attend(s):
    c = s.case
    B, Hq, Hkv, d, T = c["B"], c["Hq"], c["Hkv"], c["d"], c["T"]
    K, V = _rows(s.pool, s.table, c["len"], c)
    n = K.shape[2]
    q = s.q.float().view(B, Hkv, Hq // Hkv * T, d)
    S = torch.matmul(q, K.transpose(-1, -2)).mul_(d ** -0.5).view(B, Hq, T, n)
    last = s.lens.long()[:, None] - T + torch.arange(T, device=S.device)  # [B, T]: the last row that a token sees
    S.masked_fill_((torch.arange(n, device=S.device) > last[..., None])[:, None], -math.inf)
    m = S.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    P = S.sub_(m).exp_()
    l = P.sum(-1, keepdim=True)
    Y = torch.matmul(P.view(B, Hkv, -1, n), V).view(B, Hq, T, d) / torch.where(l > 0, l, torch.ones_like(l))
    return {"Y": Y.to(s.q.dtype), "LSE": (m + l.log()).squeeze(-1)}


def _there(table, P):
    return (table >= 0) & (table < P)


def _counts(entries, P):
    """How many entries name each page"""
    e = torch.where(_there(entries, P), entries, P).flatten().long()
    return torch.zeros(P + 1, device=e.device, dtype=torch.int64).index_add_(0, e, torch.ones_like(e))[:P]


def _plain_step(s):
    c = s.case
    B, R, P = c["B"], c["page_rows"], _pages(c)
    M = s.table.shape[1]
    entry, seq = torch.arange(M, device=s.table.device), torch.arange(B, device=s.table.device)
    # fork
    p = s.parents.long()
    named = (p >= 0) & (p < B)
    p0 = p.clamp(0, B - 1)
    held = (s.lens[p0].clamp(0, c["cap"]) + R - 1) // R
    new = torch.where(named[:, None] & (entry < held[:, None]) & _there(s.table[p0], P), s.table[p0], -1)
    same = p == seq
    table = torch.where(same[:, None], s.table, new)
    lens = torch.where(same, s.lens, torch.where(named, s.lens[p0], 0))
    refs = s.refs + _counts(torch.where(same[:, None], -1, table), P) - _counts(torch.where(same[:, None], -1, s.table), P)
    # free
    past = entry >= ((s.keep.clamp(0, c["cap"]) + R - 1) // R)[:, None]
    refs = refs - _counts(torch.where(past, table, -1), P)
    table = torch.where(past, -1, table)
    # extend
    a = s.keep.long().clamp(0, c["cap"])
    b = (a + s.add.clamp(min=0)).clamp(max=c["cap"])
    touched = (entry >= (a // R)[:, None]) & (entry < ((b + R - 1) // R)[:, None]) & (b > a)[:, None]
    shared = _there(table, P) & (refs[table.clamp(0, P - 1).long()] > 1)
    need = touched & (shared | ~_there(table, P))
    free = (refs <= 0).nonzero().flatten()
    total = int(need.sum())
    lacking = max(0, total - free.numel())
    if not lacking:
        taken = torch.where(need, free[(need.flatten().long().cumsum(0) - 1).clamp(min=0).view(B, M)], table.long()) if total else table.long()
        copied = need & shared & (entry == (a // R)[:, None]) & (a % R > 0)[:, None]
        s.pool[:, taken[copied]] = s.pool[:, table[copied].long()]
        refs = refs - _counts(torch.where(need & shared, table, -1), P)
        refs = torch.where(_counts(torch.where(need, taken, -1), P) > 0, 1, refs)
        table = taken
    info = torch.tensor([0 if lacking else total, lacking], dtype=torch.int32)
    return {"table": table.to(torch.int32), "lens": lens.to(torch.int32), "refs": refs.to(torch.int32), "pool": s.pool, "info": info.to(table.device)}


def _plain_compact(s):
    P = _pages(s.case)
    used = s.refs > 0
    U = int(used.sum())
    page = torch.arange(P, device=s.refs.device)
    src = (used & (page >= U)).nonzero().flatten().flip(0)[:s.max_moves]
    dst = (~used & (page < U)).nonzero().flatten()[:s.max_moves]
    s.pool[:, dst] = s.pool[:, src]
    to = page.clone()
    to[src] = dst
    refs = s.refs.clone()
    refs[dst], refs[src] = s.refs[src], torch.zeros_like(s.refs[src])
    there = _there(s.table, P)
    table = torch.where(there, to[s.table.clamp(0, P - 1).long()], s.table.long())
    return {"table": table.to(torch.int32), "refs": refs, "pool": s.pool, "info": torch.tensor([U, src.numel()], dtype=torch.int32, device=page.device)}


# ---- the package's calls ------------------------------------------------------------------------------------------------------


def _own(s):
    from paper_2604_00754_amd import binding as sa
    c = s.case
    if s.ws is None:  # descriptor and workspace: made once, as a program does
        s.desc = sa.make_cache4_desc(c["B"], c["Hq"], c["Hkv"], c["d"], c["page_rows"], _pages(c), c["cap"] // c["page_rows"], c["layers"],
                                     sa.SA_BF16 if c["dtype"] == "bf16" else sa.SA_F32)
        op = {"write": None, "attend": sa.SA_OP_CACHE4_DECODE, "step": sa.SA_OP_PAGES_EXTEND, "compact": sa.SA_OP_PAGES_COMPACT}[c["kind"]]
        size = 0 if op is None else sa.sa_cache4_workspace_bytes(s.desc, op, c["T"])
        s.ws = torch.empty(max(size, 256), device=s.table.device, dtype=torch.uint8)
    if c["kind"] == "write":
        sa.sa_cache4_write(s.desc, s.K, s.V, s.starts, s.counts, s.table, s.pool)
        sa.sa_cache4_read(s.desc, s.pool, s.table, s.starts, s.counts, s.K_out, s.V_out)
        return {"K": s.K_out, "V": s.V_out}
    if c["kind"] == "attend":
        sa.sa_cache4_decode_fwd(s.desc, s.q, s.pool, s.table, s.lens, s.max_len, s.Y, s.LSE, s.ws)
        return {"Y": s.Y, "LSE": s.LSE}
    if c["kind"] == "step":
        sa.sa_pages_fork(s.desc, s.parents, s.table, s.lens, s.refs, s.table_out, s.lens_out, s.refs_out)
        sa.sa_pages_free(s.desc, s.keep, s.table_out, s.refs_out)
        sa.sa_pages_extend(s.desc, s.keep, s.add, s.table_out, s.refs_out, s.pool, s.info, s.ws)
        return {"table": s.table_out, "lens": s.lens_out, "refs": s.refs_out, "pool": s.pool, "info": s.info}
    sa.sa_pages_compact(s.desc, s.max_moves, s.table, s.refs, s.table_out, s.refs_out, s.pool, s.info, s.ws)
    return {"table": s.table_out, "refs": s.refs_out, "pool": s.pool, "info": s.info}


def run(state):
    if own:
        return _own(state)
    return {"write": _plain_write, "attend": _plain_attend, "step": _plain_step, "compact": _plain_compact}[state.case["kind"]](state)


def _rows_in_use(c):
    return c["len"] + (c["B"] - 1) * (c["len"] * 5 // 8 if c["varlen"] else c["len"])  # lengths spread over a quarter to all


def work(case):
    """Every input read once, every output written once.  write: the rows in, the codes out and in, the rows out."""
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    held = c["d"] + c["d"] // 16  # bytes of a row of K and V in 4 bits
    if c["kind"] == "write":
        rows = min(_rows_in_use(c), c["B"] * c["T"]) * c["Hkv"]
        return {"bytes": rows * (4 * c["d"] * e + 2 * held), "flops": 0}
    if c["kind"] == "attend":
        rows = _rows_in_use(c)
        pairs = c["T"] * rows - c["B"] * c["T"] * (c["T"] - 1) // 2
        return {"bytes": rows * c["Hkv"] * held + 2 * c["B"] * c["Hq"] * c["T"] * c["d"] * e, "flops": 4 * max(pairs, 1) * c["Hq"] * c["d"]}
    ints = 8 * (c["B"] * (c["cap"] // c["page_rows"]) + _pages(c))
    if c["kind"] == "step":  # nearly every sequence that takes part in a fork has a page that it shares and has begun
        return {"bytes": ints + 2 * 2 * (c["B"] // 2) * c["layers"] * _page_bytes(c), "flops": 0}
    used, P = _rows_in_use(c) // c["page_rows"], _pages(c)
    return {"bytes": ints + 2 * used * max(0, P - used) // P * c["layers"] * _page_bytes(c), "flops": 0}


def _cost(case):
    """What bounds the draw: seconds at 8 TB/s and 2.5 PFLOP/s (fp32: 0.15)."""
    w = work(case)
    return w["bytes"] / 8e12 + w["flops"] / (2.5e15 if case["dtype"] == "bf16" else 1.5e14)


# ---- in 64 bits, from the definitions -----------------------------------------------------------------------------------------


def _nearest(x):
    """fp64 [..., d]: the value that the format holds for each element, by looking at every magnitude"""
    x = x.unflatten(-1, (-1, 32))
    top = x.abs().amax(-1, keepdim=True)
    e = torch.floor(torch.log2(top.clamp(min=2.0 ** -130)))
    e = torch.where(torch.exp2(e) > top.clamp(min=2.0 ** -130), e - 1, e)
    e = torch.where(torch.exp2(e + 1) <= top, e + 1, e) - 2
    e = torch.where(top > 7 * torch.exp2(e), e + 1, e).clamp(min=-125)
    best, value = torch.full_like(x, math.inf), torch.zeros_like(x)
    for magnitude in (0, 1, 2, 4, 0.5, 1.5, 3, 6):  # even codes first: a tie goes to them
        off = (x.abs() - magnitude * torch.exp2(e)).abs()
        value = torch.where(off < best, magnitude * torch.exp2(e), value)
        best = torch.minimum(off, best)
    return (torch.sign(x) * value).flatten(-2)


def exact(case, seed):
    c = case
    if c["kind"] in ("step", "compact"):
        return None  # whole numbers
    s = prepare(case, seed)
    if c["kind"] == "write":
        out = {}
        for name, x in (("K", s.K), ("V", s.V)):
            y = torch.zeros(x.shape, device=x.device, dtype=torch.float64)
            for b in range(c["B"]):
                m = int(s.counts[b])
                y[b, :, :m] = _nearest(x[b, :, :m].double())
            out[name] = y
        return out
    B, Hq, Hkv, d, T, R = c["B"], c["Hq"], c["Hkv"], c["d"], c["T"], c["page_rows"]
    Y = torch.zeros(B, Hq, T, d, device=s.q.device, dtype=torch.float64)
    LSE = torch.full((B, Hq, T), -math.inf, device=s.q.device, dtype=torch.float64)
    magnitude = [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    low = torch.tensor([(-1) ** (b >> 3 & 1) * magnitude[b & 7] for b in range(256)], device=s.q.device, dtype=torch.float64)
    high = torch.tensor([(-1) ** (b >> 7) * magnitude[b >> 4 & 7] for b in range(256)], device=s.q.device, dtype=torch.float64)
    for b in range(B):
        n = int(s.lens[b])
        row = torch.arange(n, device=s.q.device)
        page, tile, r = s.table[b].long()[row // R], row % R // 32, row % 32
        half, g, i = r // 16, r % 16 // 4, r % 4
        e = torch.arange(d, device=s.q.device)
        for h in range(Hkv):
            t = s.pool[page, h, tile]  # [n, 34 d]
            kb = (r[:, None] * (d // 2) + e // 2).long()
            vb = 16 * d + ((((g[:, None] * 16 + e // (d // 16)) * 2 + half[:, None]) * 4 + i[:, None]) * (d // 32) + e % (d // 16) // 2)
            ks = 32 * d + (e // 32 * 16 + r[:, None] % 16) * 2 + half[:, None]
            vs = 33 * d + ((e // 32 * 4 + g[:, None]) * 2 + half[:, None]) * 4 + i[:, None]
            K, V = (torch.where(e % 2 == 0, low[t.gather(1, at).long()], high[t.gather(1, at).long()]) *
                    torch.exp2(t.gather(1, sc).double() - 127) for at, sc in ((kb, ks), (vb, vs)))
            q = s.q[b, h * (Hq // Hkv):(h + 1) * (Hq // Hkv)].double()  # [g, T, d]
            S = q @ K.T / math.sqrt(d)
            S = torch.where(row <= n - T + torch.arange(T, device=S.device)[:, None], S, -math.inf)
            top = S.max(-1, keepdim=True).values.clamp(min=-1e300)
            w = torch.exp(S - top)
            total = w.sum(-1, keepdim=True)
            Y[b, h * (Hq // Hkv):(h + 1) * (Hq // Hkv)] = w @ V / total.clamp(min=1e-300)
            LSE[b, h * (Hq // Hkv):(h + 1) * (Hq // Hkv)] = (top + torch.log(total)).squeeze(-1)
    return {"Y": Y, "LSE": LSE}
