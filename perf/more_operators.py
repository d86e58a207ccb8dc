"""The paged cache in 4 bits and the GPU-side planning of a batch's pages, as measured cases: appending rows quantised to 4 bits
(by block table or by slot), reading them back, the attention of new tokens over such a cache, and the step's plan - row offsets,
positions, slots and pages from the requests' lengths and a pool of free pages.

A cached 4-bit row is two halves (the first and the second half of the head dims), each with a scale s and a smallest value m,
both bfloat16: value = code * s + m, codes 0 to 15.  Pages: [n_pages, n_kv_heads, page, head_dim / 2] bytes, byte i holds the code of
dim i in its low and of dim i + head_dim / 2 in its high bits; parameters: [n_pages, n_kv_heads, page, 2, 2] (half, (s, m)).

Notation: B sequences, sequence b has lens[b] cached tokens and new[b] new ones, whose rows lie one sequence after the other
in the [n_tokens, heads, head_dim] tensors (row offsets `cu`).
"""
import math
import random

import torch

own = False

FLOATS = {"f32": torch.float32, "bf16": torch.bfloat16}
SMALLEST = 2.0 ** -60  # smallest scale
RELEASE = -1           # new[b] of a request that is finished: its pages go back to the pool


def listed():
    return [
        # one layer's cache update of a decode step: 64 sequences, one token each (grouped-query 64/8 heads, head_dim 128)
        dict(name="append_decode", op="write", by="slots", dtype="bf16", B=64, nkv=8, d=128, page=16, lo=512, hi=1023, new_lo=1, new_hi=1, layout=1),
        # prompts entering the cache of a 40-head multi-head model, 16 of about 1024 tokens
        dict(name="store_prompts", op="write", by="table", dtype="bf16", B=16, nkv=40, d=128, page=16, lo=0, hi=0, new_lo=700, new_hi=1024, layout=2),
        # a batch's contexts copied out, ragged
        dict(name="read_batch", op="read", dtype="bf16", B=16, nkv=40, d=128, page=16, lo=300, hi=1279, new_lo=0, new_hi=0, layout=3),
        # single-token step of one sequence: the smallest attention call, latency counts
        dict(name="decode_one", op="attend", dtype="bf16", B=1, nq=64, nkv=8, d=128, page=16, lo=2048, hi=2048, new_lo=1, new_hi=1, window=0, sinks=0, layout=4),
        # single-token step of a batch of 64 ragged sequences
        dict(name="decode_64", op="attend", dtype="bf16", B=64, nq=64, nkv=8, d=128, page=16, lo=129, hi=1023, new_lo=1, new_hi=1, window=0, sinks=0, layout=5),
        # long contexts, what 4 bits are for: the cache read is the cost
        dict(name="decode_long", op="attend", dtype="bf16", B=32, nq=64, nkv=8, d=128, page=16, lo=9000, hi=16383, new_lo=1, new_hi=1, window=0, sinks=0, layout=6),
        # drafted tokens checked in one pass: five new tokens per sequence
        dict(name="verify_5", op="attend", dtype="bf16", B=32, nq=64, nkv=8, d=128, page=16, lo=500, hi=2300, new_lo=5, new_hi=5, window=0, sinks=0, layout=7),
        # a chunk of a long prompt on the context before it: the largest call
        dict(name="chunk_2048", op="attend", dtype="bf16", B=1, nq=64, nkv=8, d=128, page=16, lo=14336, hi=14336, new_lo=2048, new_hi=2048, window=0, sinks=0, layout=8),
        # ragged chunks of a mixed batch on a multi-head cache
        dict(name="chunks_ragged", op="attend", dtype="bf16", B=12, nq=40, nkv=40, d=128, page=16, lo=0, hi=1000, new_lo=1, new_hi=700, window=0, sinks=0, layout=9),
        # float32 stack at the small configuration's head size, sliding window with three first tokens that stay visible
        dict(name="chunk_f32_d64", op="attend", dtype="f32", B=4, nq=8, nkv=4, d=64, page=16, lo=50, hi=900, new_lo=30, new_hi=256, window=200, sinks=3, layout=10),
        # the plan of a decode step: one token for each of 256 requests
        dict(name="plan_decode", op="plan", B=256, page=16, lo=100, hi=2000, chunk=0.0, done=0.0, new_hi=1, short=0, layout=11),
        # the plan of a mixed step of a large server: finished requests, single tokens, chunks of prompts
        dict(name="plan_mixed", op="plan", B=2048, page=16, lo=0, hi=6000, chunk=0.15, done=0.05, new_hi=512, short=0, layout=12),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["write", "read", "attend", "attend", "attend", "attend", "plan"])
        layout = rng.randrange(1, 1 << 20)
        if op == "plan":
            c = dict(op=op, B=_spread(rng, 64, 4096), page=rng.choice([1, 8, 16, 16, 32, 64]), lo=0, hi=_spread(rng, 16, 6000),
                     chunk=rng.choice([0.0, rng.random() * 0.3]), done=rng.choice([0.0, rng.random() * 0.2]), new_hi=_spread(rng, 1, 700),
                     short=rng.choice([0, 0, 1]), layout=layout)
            if work(c)["bytes"] <= 8_000_000:
                return c
            continue
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        nkv, group = rng.choice([1, 2, 4, 8, 10, 16, 32, 40]), rng.choice([1, 1, 2, 4, 5, 8])
        c = dict(op=op, dtype=dtype, B=_spread(rng, 1, 64), nkv=nkv, d=rng.choice([64, 128, 128]), page=rng.choice([16, 16, 16, 32, 64]), layout=layout)
        if dtype == "f32":
            c["B"] = min(c["B"], 8)
        top = _spread(rng, 4, 2000 if dtype == "f32" else 12000)
        c["lo"], c["hi"] = rng.randrange(0, top + 1), top
        if op == "write":
            c["by"] = rng.choice(["slots", "table"])
        if op == "read":
            c["lo"], c["new_lo"], c["new_hi"] = max(1, c["lo"]), 0, 0
        else:
            c["new_hi"] = rng.choice([1, 1, _spread(rng, 2, 16), _spread(rng, 17, 300 if dtype == "f32" else 1500)])
            c["new_lo"] = 1 if rng.random() < 0.5 else c["new_hi"]
        if op == "attend":
            c["nq"] = nkv * group
            c["window"] = rng.choice([0, 0, 0, _spread(rng, 1, 3000)])
            c["sinks"] = rng.choice([0, rng.randrange(1, 40)]) if c["window"] else 0
        w = work(c)
        T, L = c["hi"] + c["new_hi"], max(1, c["new_hi"])
        cached = c["B"] * T * nkv * c["d"]
        scores = c["B"] * c.get("nq", 0) * L * T * (20 if dtype == "f32" else 1)
        if 150_000 <= w["bytes"] <= 300_000_000 and w["flops"] <= 8e11 and cached <= 300_000_000 and scores <= 1_500_000_000:
            return c


def _lengths(case):
    """(cached tokens, new tokens) of every sequence: part of the case, not of the seed."""
    rng = random.Random(case["layout"])
    lens = [rng.randint(case["lo"], case["hi"]) for _ in range(case["B"])]
    if case["op"] != "plan":
        return lens, [rng.randint(case["new_lo"], case["new_hi"]) for _ in range(case["B"])]
    new = []
    for _ in lens:
        x = rng.random()
        new.append(RELEASE if x < case["done"] else rng.randint(1, case["new_hi"]) if x < case["done"] + case["chunk"] else 1)
    return lens, new


def _pages(n, page):
    return -(-n // page)


def _plan_sizes(case):
    """(rows of the step, new pages, pages that come back, pages of all requests before the step)"""
    lens, new = _lengths(case)
    page = case["page"]
    rows = sum(n for n in new if n > 0)
    take = sum(_pages(a + n, page) - _pages(a, page) for a, n in zip(lens, new) if n > 0)
    back = sum(_pages(a, page) for a, n in zip(lens, new) if n < 0)
    return rows, take, back, sum(_pages(a, page) for a in lens)


def work(case):
    if case["op"] == "plan":
        rows, take, back, _ = _plan_sizes(case)
        # lengths in, offsets and next lengths out; a position and a slot per row; table entries of the rows' pages and of returned ones; the pool
        return {"bytes": 16 * case["B"] + 8 * rows + 4 * (rows // case["page"] + case["B"]) + 8 * take + 8 * back, "flops": 4 * rows}
    lens, new = _lengths(case)
    nkv, d, e = case["nkv"], case["d"], 4 if case["dtype"] == "f32" else 2
    row = 2 * nkv * (d // 2 + 8)  # K and V of one cached token
    if case["op"] == "write":  # new rows in, cached rows out; and read back
        n = sum(new)
        return {"bytes": 2 * n * (2 * nkv * d * e + row), "flops": 6 * n * nkv * d}
    if case["op"] == "read":
        n = sum(lens)
        return {"bytes": n * (2 * nkv * d * e + row), "flops": 4 * n * nkv * d}
    w, s, keys, pairs = case["window"], case["sinks"], 0, 0
    for a, n in zip(lens, new):
        first = max(0, a - w + 1) if w else 0  # keys from here on, and the sinks before it
        keys += a + n - first + min(s, first)
        k = min(n, max(0, w - a)) if w else n  # queries that still see everything before them
        pairs += k * a + k * (k + 1) // 2
        pairs += sum(w + min(s, a + i + 1 - w) for i in range(k, n))
    return {"bytes": keys * row + 2 * sum(new) * case["nq"] * d * e, "flops": 4 * pairs * case["nq"] * d}


def _dev():
    return "cuda"


def _quantise(x):
    """float32 rows [..., d] -> (packed codes uint8 [..., d / 2], parameters bfloat16 [..., 2, 2]).  Per half: m is its smallest value rounded
    down to bfloat16, s = (largest - m) / 15 rounded to bfloat16, at least SMALLEST; code = (x - m) / s rounded to nearest, half to even."""
    h = x.unflatten(-1, (2, x.shape[-1] // 2))
    lo, hi = h.amin(-1), h.amax(-1)
    bits = lo.view(torch.int32)
    m = (torch.where(lo < 0, bits + 0xFFFF, bits) & -0x10000).view(torch.float32)
    r = hi - m
    s = (r / torch.full_like(r, 15)).to(torch.bfloat16).float().clamp(min=SMALLEST)
    bad = ~torch.isfinite(r).all(-1, keepdim=True)
    codes = torch.round((h - m[..., None]) / s[..., None]).clamp(0, 15).masked_fill(bad[..., None], 0).to(torch.uint8)
    p = torch.stack([s, m], -1).masked_fill(bad[..., None], math.nan).to(torch.bfloat16)
    return codes[..., 0, :] | (codes[..., 1, :] << 4), p


def _values(codes, p):
    """float32 values of cached rows: codes uint8 [..., d / 2], parameters [..., 2, 2]."""
    p = p.float()
    return torch.cat([(codes & 15).float() * p[..., 0, :1] + p[..., 0, 1:], (codes >> 4).float() * p[..., 1, :1] + p[..., 1, 1:]], -1)


def _prepare_plan(case, seed):
    dev, page, B = _dev(), case["page"], case["B"]
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    lens, new = _lengths(case)
    rows, take, back, used = _plan_sizes(case)
    spare = take // 2 if case["short"] else take + 50  # short: the pool does not last for the last requests
    n_pages = used + spare
    width = max(1, max(_pages(a + max(0, n), page) for a, n in zip(lens, new)))
    perm = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32)
    ln = torch.tensor(lens, dtype=torch.int32, device=dev)
    have = (ln.long() + page - 1) // page
    col = torch.arange(width, device=dev)
    owned = col < have[:, None]
    at = (torch.cumsum(have, 0) - have)[:, None] + col
    table = torch.where(owned, perm[at.clamp(max=n_pages - 1)], torch.full_like(perm[:1], -1)).contiguous()
    free = torch.zeros(n_pages, dtype=torch.int32, device=dev)
    free[:spare] = perm[used:]
    return dict(case=case, lens=ln, new=torch.tensor(new, dtype=torch.int32, device=dev), table=table, free=free,
                n_free=torch.tensor([spare], dtype=torch.int32, device=dev), n_pages=n_pages, n_tokens=rows + 7,
                err=torch.zeros(1, dtype=torch.int32, device=dev))


def prepare(case, seed):
    if case["op"] == "plan":
        return _prepare_plan(case, seed)
    dev = _dev()
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    lens, new = _lengths(case)
    B, nkv, d, page, dtype = case["B"], case["nkv"], case["d"], case["page"], FLOATS[case["dtype"]]
    need = [_pages(a + n, page) for a, n in zip(lens, new)]
    width = max(1, max(need))
    n_pages = sum(need) + 3  # a few pages belong to nobody
    perm = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32)
    table, at = torch.zeros((B, width), dtype=torch.int32, device=dev), 0
    for b, k in enumerate(need):  # scattered pages, as a pool hands them out
        table[b, :k] = perm[at:at + k]
        at += k
    st = dict(case=case, B=B, table=table, max_context=max(a + n for a, n in zip(lens, new)), max_new=max(1, max(new)))
    st["lens"] = torch.tensor(lens, dtype=torch.int32, device=dev)
    cu = [0]
    for n in (lens if case["op"] == "read" else new):
        cu.append(cu[-1] + n)
    st["cu"], st["n"] = torch.tensor(cu, dtype=torch.int32, device=dev), cu[-1]
    st["starts"] = torch.zeros(B, dtype=torch.int32, device=dev)
    st["err"] = torch.zeros(1, dtype=torch.int32, device=dev)

    # keys: dimensions of unequal size and offset, as rotary models have them, and rows of unequal size; values ~ N(0, 1)
    def rows(shape, uneven):
        x = torch.randn(shape, generator=g, device=dev)
        if uneven:
            x *= torch.exp(0.5 * torch.randn(shape[-1:], generator=g, device=dev)) * torch.exp(0.3 * torch.randn(shape[:-1] + (1,), generator=g, device=dev))
            x += 0.5 * torch.randn(shape[-1:], generator=g, device=dev)
        return x.to(dtype)

    for n, uneven in (("k", True), ("v", False)):
        if case["op"] == "write":
            st[n + "_pages"] = torch.zeros((n_pages, nkv, page, d // 2), dtype=torch.uint8, device=dev)
            st[n + "_scales"] = torch.ones((n_pages, nkv, page, 2, 2), dtype=torch.bfloat16, device=dev)
        else:
            st[n + "_pages"], st[n + "_scales"] = _quantise(rows((n_pages, nkv, page, d), uneven).float())
    if case["op"] == "write":  # K and V as the slices of one projection output [q | k | v], q as wide as k
        qkv = torch.cat([rows((st["n"], nkv, d), True) for _ in range(2)] + [rows((st["n"], nkv, d), False)], 1)
        st["k"], st["v"] = qkv[:, nkv:2 * nkv], qkv[:, 2 * nkv:]
        _, _, pg, r = _where(st, st["lens"], st["n"])
        st["slots"] = (pg * page + r).to(torch.int32)  # of a plan made once per step, for all layers
    if case["op"] == "attend":
        st["q"] = rows((st["n"], case["nq"], d), False)
    return st


def _where(st, offsets, n):
    """(sequence, position, page, row of the page) of token rows 0 .. n-1; sequence b's first row is at position offsets[b]."""
    cu, page = st["cu"].long(), st["case"]["page"]
    row = torch.arange(n, device=cu.device)
    b = torch.searchsorted(cu, row, right=True) - 1
    pos = offsets.long()[b] + row - cu[b]
    return b, pos, st["table"][b, pos // page].long(), pos % page


def _plan(st):
    """Elementary form of the step's plan.  All pages of finished requests join the free ones first, in the requests' order; then the requests
    take theirs from the end.  A request that the pool or the rows do not last for gets nothing, and so does a later one that needs pages."""
    B, page, T = st["case"]["B"], st["case"]["page"], st["n_tokens"]
    dev = st["lens"].device
    lens, new, table, free = st["lens"].long(), st["new"].long(), st["table"], st["free"]
    n_free = st["n_free"].long()
    width = table.shape[1]
    have = (lens + page - 1) // page
    done = new < 0
    n = new.clamp(min=0)
    col = torch.arange(width, device=dev)
    gone = torch.where(done, have, torch.zeros_like(have))
    first = n_free + torch.cumsum(gone, 0) - gone  # where a finished request's pages go
    put = (first[:, None] + col).where(col < gone[:, None], torch.full_like(col, free.numel()))
    pool = torch.cat([free, free.new_zeros(1)])
    pool[put.flatten()] = table.flatten()
    free.copy_(pool[:-1])
    have_free = n_free + gone.sum()
    take = torch.where(n > 0, (lens + n + page - 1) // page - have, torch.zeros_like(n))
    cum_take, cum_rows = torch.cumsum(take, 0), torch.cumsum(n, 0)
    ok = ((take == 0) | (cum_take <= have_free)) & (cum_rows <= T)
    n = torch.where(ok, n, torch.zeros_like(n))
    take = torch.where(ok, take, torch.zeros_like(take))
    cu = torch.cat([torch.zeros_like(n[:1]), torch.cumsum(n, 0)])
    k = (torch.cumsum(take, 0) - take)[:, None] + col - have[:, None]
    fresh = (col >= have[:, None]) & (col < (have + take)[:, None])
    table.copy_(torch.where(fresh, free[(have_free - 1 - k).clamp(0, free.numel() - 1)], table))
    row = torch.arange(T, device=dev)
    b = (torch.searchsorted(cu, row, right=True) - 1).clamp(max=B - 1)
    live = row < cu[-1]
    pos = lens[b] + row - cu[b]
    slot = table[b, (pos // page).clamp(max=width - 1)].long() * page + pos % page
    none = torch.full_like(row, -1)
    after = torch.where(done, torch.zeros_like(lens), lens + n)
    i32 = lambda x: x.to(torch.int32)  # noqa: E731
    return (i32(cu), i32(torch.where(live, pos, none)), i32(torch.where(live, slot, none)), i32(after), i32(have_free - take.sum()), table, free)


def run(state):
    st, case = state, state["case"]
    if own:
        import paper_2502_20727_b200 as spd
        if case["op"] == "plan":
            p = spd.plan_batch(st["lens"], st["new"], st["table"], st["free"], st["n_free"], page=case["page"], n_pages=st["n_pages"],
                               n_tokens=st["n_tokens"], err=st["err"])
            return p.cu_new, p.positions, p.slots, p.next_lens, p.n_free, st["table"], st["free"]
        dtype = FLOATS[case["dtype"]]
        kv = dict(k_scales=st["k_scales"], v_scales=st["v_scales"], err=st["err"])
        if case["op"] == "attend":
            return spd.paged_attention(st["q"], st["k_pages"], st["v_pages"], st["cu"], st["lens"], st["table"], max_new=st["max_new"],
                                       max_context=st["max_context"], window=case["window"], sinks=case["sinks"], **kv)
        if case["op"] == "write":
            if case["by"] == "slots":
                spd.kv_write_slots(st["k"], st["v"], st["k_pages"], st["v_pages"], st["slots"], **kv)
            else:
                spd.kv_write(st["k"], st["v"], st["k_pages"], st["v_pages"], st["cu"], st["lens"], st["table"], **kv)
            return spd.kv_read(st["k_pages"], st["v_pages"], st["cu"], st["lens"], st["table"], n_tokens=st["n"], dtype=dtype, **kv)
        return spd.kv_read(st["k_pages"], st["v_pages"], st["cu"], st["starts"], st["table"], n_tokens=st["n"], dtype=dtype, **kv)

    if case["op"] == "plan":
        return _plan(st)
    dtype = FLOATS[case["dtype"]]
    if case["op"] == "write":
        if case["by"] == "slots":
            page, row = st["slots"].long() // case["page"], st["slots"].long() % case["page"]
        else:
            _, _, page, row = _where(st, st["lens"], st["n"])
        for t in ("k", "v"):
            st[t + "_pages"][page, :, row], st[t + "_scales"][page, :, row] = _quantise(st[t].float())
    elif case["op"] == "read":
        _, _, page, row = _where(st, st["starts"], st["n"])
    if case["op"] != "attend":
        return tuple(_values(st[t + "_pages"][page, :, row], st[t + "_scales"][page, :, row]).to(dtype) for t in ("k", "v"))

    B, nq, nkv, d, page, T, L = st["B"], case["nq"], case["nkv"], case["d"], case["page"], st["max_context"], st["max_new"]
    dev = st["q"].device
    key = torch.arange(T, device=dev)
    pages = st["table"][:, :-(-T // page)].long()
    kv = [_values(st[t + "_pages"][pages], st[t + "_scales"][pages]).transpose(1, 2).reshape(B, nkv, -1, d)[:, :, :T] for t in ("k", "v")]
    cu, lens = st["cu"].long(), st["lens"].long()
    i = torch.arange(L, device=dev)
    live = i < (cu[1:] - cu[:-1])[:, None]  # [B, L]
    src = torch.where(live, cu[:-1, None] + i, torch.zeros_like(i))
    q = st["q"].float()[src].view(B, L, nkv, nq // nkv, d).permute(0, 2, 1, 3, 4).reshape(B, nkv, -1, d)
    s = torch.matmul(q, kv[0].transpose(-1, -2)) * (1.0 / math.sqrt(d))
    pos = (lens[:, None] + i)[..., None]
    seen = key <= pos
    if case["window"]:
        seen &= (key > pos - case["window"]) | (key < case["sinks"])
    s = s.view(B, nkv, L, nq // nkv, T).masked_fill_(~seen[:, None, :, None], -math.inf)
    s = torch.exp(s.sub_(s.amax(-1, keepdim=True)))
    s /= s.sum(-1, keepdim=True)
    o = torch.matmul(s.view(B, nkv, -1, T), kv[1])
    o = o.view(B, nkv, L, nq // nkv, d).permute(0, 2, 1, 3, 4).reshape(B, L, nq, d)
    return o[live].to(dtype)


def _exact_plan(case, seed):
    """Request by request, on the host."""
    st = prepare(case, seed)
    lens, new, table, free, n_free = st["lens"].tolist(), st["new"].tolist(), st["table"].tolist(), st["free"].tolist(), int(st["n_free"])
    page, T = case["page"], st["n_tokens"]
    for b, n in enumerate(new):
        if n < 0:
            for j in range(_pages(lens[b], page)):
                free[n_free] = table[b][j]
                n_free += 1
    cu, positions, slots, after, wanted, rows, top = [0], [], [], [], 0, 0, n_free
    for b, n in enumerate(new):
        a = lens[b]
        if n < 0:
            after.append(0)
            cu.append(cu[-1])
            continue
        fresh = range(_pages(a, page), _pages(a + n, page))
        wanted, rows = wanted + len(fresh), rows + n
        if (len(fresh) and wanted > top) or rows > T:
            n, fresh = 0, ()
        for j in fresh:
            n_free -= 1
            table[b][j] = free[n_free]
        for t in range(a, a + n):
            positions.append(t)
            slots.append(table[b][t // page] * page + t % page)
        after.append(a + n)
        cu.append(cu[-1] + n)
    pad = [-1] * (T - len(slots))
    t = lambda x: torch.tensor(x, dtype=torch.int32, device=_dev())  # noqa: E731
    return t(cu), t(positions + pad), t(slots + pad), t(after), t([n_free]), t(table), t(free)


def exact(case, seed):
    """The definition in float64, sequence by sequence."""
    if case["op"] == "plan":
        return _exact_plan(case, seed)
    st = prepare(case, seed)
    lens, new = _lengths(case)
    page, d, nkv = case["page"], case["d"], case["nkv"]
    half = d // 2

    def dequantised(t, b, first, count):
        where = torch.arange(first, first + count, device=st["table"].device)
        pg, r = st["table"][b].long()[where // page], where % page
        byte, p = st[t + "_pages"][pg, :, r].to(torch.int64), st[t + "_scales"][pg, :, r].double()
        x = torch.empty(byte.shape[:-1] + (d,), dtype=torch.float64, device=byte.device)
        x[..., :half] = (byte % 16).double() * p[..., 0, 0, None] + p[..., 0, 1, None]
        x[..., half:] = (byte // 16).double() * p[..., 1, 0, None] + p[..., 1, 1, None]
        return x

    if case["op"] == "read":
        parts = [[dequantised(t, b, 0, a) for b, a in enumerate(lens) if a] for t in ("k", "v")]
        return tuple(torch.cat(p) for p in parts)
    if case["op"] == "write":
        out = []
        for t in ("k", "v"):
            x = st[t].double()
            y = torch.empty_like(x)
            for dims in (slice(0, half), slice(half, d)):
                z = x[..., dims]
                low, high = z.min(-1, keepdim=True).values, z.max(-1, keepdim=True).values
                m = low.to(torch.bfloat16)  # rounded down
                m = torch.where(m.double() > low, torch.nextafter(m, torch.full_like(m, -math.inf)), m).double()
                step = ((high - m) / 15).to(torch.bfloat16).double().clamp(min=SMALLEST)
                y[..., dims] = torch.round((z - m) / step).clamp(0, 15) * step + m
            out.append(y)
        return tuple(out)
    out, at = [], 0
    for b, (a, n) in enumerate(zip(lens, new)):
        if not n:
            continue
        k, v = dequantised("k", b, 0, a + n), dequantised("v", b, 0, a + n)
        t = torch.arange(a + n, device=k.device)[None]
        p = torch.arange(a, a + n, device=k.device)[:, None]
        hidden = t > p
        if case["window"]:
            hidden |= (t <= p - case["window"]) & (t >= case["sinks"])
        group = case["nq"] // nkv
        heads = []
        for h in range(case["nq"]):
            logits = st["q"][at:at + n, h].double() @ k[:, h // group].t() / d ** 0.5
            heads.append(torch.softmax(logits.masked_fill(hidden, -math.inf), -1) @ v[:, h // group])
        out.append(torch.stack(heads, 1))
        at += n
    return torch.cat(out)
