"""The paged-cache operators of the library as measured cases: appending new tokens to a paged K/V cache (plain or
quantised to 8 bits), reading cached tokens back, and the attention of a chunk of new tokens per sequence over such a cache
(causal, optionally a sliding window with always-visible first tokens).

Notation: B sequences, sequence b has lens[b] cached tokens and new[b] new ones, whose rows lie one sequence after the other
in the [n_tokens, heads, head_dim] tensors (row offsets `cu`).  Pages: [n_pages, n_kv_heads, page, head_dim], the 8-bit
formats with one float32 scale per cached row in [n_pages, n_kv_heads, page].
"""
import math
import random

import torch

own = False

NP_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}
ES = {"f32": 4, "bf16": 2, "e4m3": 1, "int8": 1}


def listed():
    head = dict(page=16)
    return [
        # one layer's cache update of a decode step: 64 sequences, one token each (grouped-query 64/8 heads, head_dim 128)
        dict(head, name="append_decode_e4m3", op="write", dtype="bf16", fmt="e4m3", B=64, nkv=8, d=128, lo=512, hi=1023, new_lo=1, new_hi=1, layout=1),
        # prompts entering the cache of a 40-head multi-head model, 16 of about 1024 tokens
        dict(head, name="store_prompts_int8", op="write", dtype="bf16", fmt="int8", B=16, nkv=40, d=128, lo=0, hi=0, new_lo=700, new_hi=1024, layout=2),
        # one sequence's context copied out of the cache (moved to another pool, or inspected)
        dict(head, name="read_one_e4m3", op="read", dtype="bf16", fmt="e4m3", B=1, nkv=8, d=128, lo=2048, hi=2048, new_lo=0, new_hi=0, layout=3),
        # a batch's contexts copied out, ragged
        dict(head, name="read_batch_int8", op="read", dtype="bf16", fmt="int8", B=16, nkv=40, d=128, lo=300, hi=1279, new_lo=0, new_hi=0, layout=4),
        # single-token step of one sequence: the smallest attention call, latency counts
        dict(head, name="decode_one_bf16", op="attend", dtype="bf16", fmt="bf16", B=1, nq=64, nkv=8, d=128, lo=2048, hi=2048, new_lo=1, new_hi=1, window=0, sinks=0, layout=5),
        # single-token step of a batch of 64 ragged sequences on an 8-bit cache
        dict(head, name="decode_64_e4m3", op="attend", dtype="bf16", fmt="e4m3", B=64, nq=64, nkv=8, d=128, lo=129, hi=1023, new_lo=1, new_hi=1, window=0, sinks=0, layout=6),
        # long contexts, 8-bit cache: the cache read is the cost
        dict(head, name="decode_long_int8", op="attend", dtype="bf16", fmt="int8", B=32, nq=64, nkv=8, d=128, lo=9000, hi=16383, new_lo=1, new_hi=1, window=0, sinks=0, layout=7),
        # drafted tokens checked in one pass: five new tokens per sequence
        dict(head, name="verify_5_bf16", op="attend", dtype="bf16", fmt="bf16", B=32, nq=64, nkv=8, d=128, lo=500, hi=2300, new_lo=5, new_hi=5, window=0, sinks=0, layout=8),
        # a chunk of a long prompt on the context before it: the largest call
        dict(head, name="chunk_2048_bf16", op="attend", dtype="bf16", fmt="bf16", B=1, nq=64, nkv=8, d=128, lo=14336, hi=14336, new_lo=2048, new_hi=2048, window=0, sinks=0, layout=9),
        # ragged chunks of a mixed batch on a multi-head 8-bit cache
        dict(head, name="chunks_ragged_e4m3", op="attend", dtype="bf16", fmt="e4m3", B=12, nq=40, nkv=40, d=128, lo=0, hi=1000, new_lo=1, new_hi=700, window=0, sinks=0, layout=10),
        # sliding window with four first tokens that stay visible
        dict(head, name="window_sinks_bf16", op="attend", dtype="bf16", fmt="bf16", B=2, nq=32, nkv=32, d=128, lo=5000, hi=6000, new_lo=1500, new_hi=2048, window=1024, sinks=4, layout=11),
        # float32 stack at the small configuration's head size
        dict(head, name="chunk_f32_d64", op="attend", dtype="f32", fmt="f32", B=4, nq=8, nkv=4, d=64, lo=50, hi=900, new_lo=30, new_hi=256, window=200, sinks=3, layout=12),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["write", "read", "attend", "attend", "attend"])
        fmt = rng.choice(["bf16", "e4m3", "int8", "f32"])
        dtype = "f32" if fmt == "f32" else "bf16"
        nkv, group = rng.choice([1, 2, 4, 8, 10, 16, 32, 40]), rng.choice([1, 1, 2, 4, 5, 8])
        c = dict(op=op, dtype=dtype, fmt=fmt, B=_spread(rng, 1, 64), nkv=nkv, d=rng.choice([64, 128, 128]), page=rng.choice([16, 16, 16, 32, 64]),
                 layout=rng.randrange(1, 1 << 20))
        if dtype == "f32":
            c["B"] = min(c["B"], 8)
        top = _spread(rng, 4, 2000 if dtype == "f32" else 12000)
        c["lo"], c["hi"] = rng.randrange(0, top + 1), top
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
        if 300_000 <= w["bytes"] <= 400_000_000 and w["flops"] <= 8e11 and cached <= 300_000_000 and scores <= 1_500_000_000:
            return c


def _lengths(case):
    """(cached tokens, new tokens) of every sequence: part of the case, not of the seed."""
    rng = random.Random(case["layout"])
    lens = [rng.randint(case["lo"], case["hi"]) for _ in range(case["B"])]
    new = [rng.randint(case["new_lo"], case["new_hi"]) for _ in range(case["B"])]
    return lens, new


def work(case):
    lens, new = _lengths(case)
    nkv, d, e, f = case["nkv"], case["d"], ES[case["dtype"]], ES[case["fmt"]]
    row = 2 * nkv * (d * f + (4 if f == 1 else 0))  # K and V of one cached token
    if case["op"] == "write":  # new rows in, cached rows out; and read back
        n = sum(new)
        return {"bytes": 2 * n * (2 * nkv * d * e + row), "flops": 4 * n * nkv * d}
    if case["op"] == "read":
        n = sum(lens)
        return {"bytes": n * (2 * nkv * d * e + row), "flops": 2 * n * nkv * d}
    w, s, keys, pairs = case["window"], case["sinks"], 0, 0
    for a, n in zip(lens, new):
        if not n:
            continue
        first = max(0, a - w + 1) if w else 0  # keys from here on, and the sinks before it
        keys += a + n - first + min(s, first)
        k = min(n, max(0, w - a)) if w else n  # queries that still see everything before them
        pairs += k * a + k * (k + 1) // 2
        late = n - k
        if late:
            pairs += late * w + (late * s if a + k + 1 - w >= s else sum(min(s, a + i + 1 - w) for i in range(k, n)))
    return {"bytes": keys * row + 2 * sum(new) * case["nq"] * d * e, "flops": 4 * pairs * case["nq"] * d}


def _dev():
    return "cuda"


def _quantise(x, fmt):
    """float32 rows -> (codes, one scale per row).  e4m3: the smallest power of two that brings the row under 448;
    int8: the row's largest magnitude / 127.  Rows of zeros keep scale 1; scales are at least 2^-126."""
    amax = x.abs().amax(-1)
    if fmt == "e4m3":
        m, ex = torch.frexp(amax)  # amax = m 2^ex, 0.5 <= m < 1; 448 = 0.875 * 2^9
        k = (ex - 9 + (m > 0.875).to(ex.dtype)).clamp(min=-126)
        s = torch.ldexp(torch.ones_like(amax), k)
        s = torch.where(amax > 0, s, torch.ones_like(s))
        return (x / s[..., None]).to(torch.float8_e4m3fn), s
    s = torch.where(amax > 0, (amax / 127).clamp(min=2.0 ** -126), torch.ones_like(amax))
    inv = torch.where(amax > 0, 127 / amax.clamp(min=127 * 2.0 ** -126), torch.ones_like(amax))
    return torch.round(x * inv[..., None]).clamp(-127, 127).to(torch.int8), s


def prepare(case, seed):
    dev = _dev()
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    lens, new = _lengths(case)
    B, nkv, d, page, fmt, dtype = case["B"], case["nkv"], case["d"], case["page"], case["fmt"], NP_TORCH[case["dtype"]]
    need = [-(-(a + n) // page) for a, n in zip(lens, new)]
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

    # cached keys: dimensions of unequal size, as rotary models have them, and rows of unequal size; values ~ N(0, 1)
    def rows(shape, uneven):
        x = torch.randn(shape, generator=g, device=dev)
        if uneven:
            x *= torch.exp(0.5 * torch.randn(shape[-1:], generator=g, device=dev)) * torch.exp(0.3 * torch.randn(shape[:-1] + (1,), generator=g, device=dev))
        return x.to(dtype)

    for n, uneven in (("k", True), ("v", False)):
        st[n + "_scales"] = None
        if case["op"] == "write":
            st[n + "_pages"] = torch.zeros((n_pages, nkv, page, d), dtype=torch.int8 if ES[fmt] == 1 else NP_TORCH[fmt], device=dev)
            if ES[fmt] == 1:
                st[n + "_pages"] = st[n + "_pages"].view(NP_TORCH[fmt])
                st[n + "_scales"] = torch.ones((n_pages, nkv, page), device=dev)
        else:
            x = rows((n_pages, nkv, page, d), uneven)
            if ES[fmt] == 1:
                st[n + "_pages"], st[n + "_scales"] = _quantise(x.float(), fmt)
            else:
                st[n + "_pages"] = x
    if case["op"] == "write":  # K and V as the slices of one projection output [q | k | v], q as wide as k
        qkv = torch.cat([rows((st["n"], nkv, d), True) for _ in range(2)] + [rows((st["n"], nkv, d), False)], 1)
        st["k"], st["v"] = qkv[:, nkv:2 * nkv], qkv[:, 2 * nkv:]
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


def _codes(pages):
    return pages.view(torch.int8) if pages.element_size() == 1 else pages


def _read(st, n, page, row, dtype):
    """Rows (page, row) of both caches in float32, rounded once to dtype."""
    out = []
    for t in ("k", "v"):
        p, s = st[t + "_pages"], st[t + "_scales"]
        x = _codes(p)[page, :, row].view(p.dtype).float()
        out.append((x if s is None else x * s[page, :, row][..., None]).to(dtype))
    return out


def run(state):
    st, case = state, state["case"]
    dtype = NP_TORCH[case["dtype"]]
    if own:
        import paper_2502_20727_b200 as spd
        kv = dict(k_scales=st["k_scales"], v_scales=st["v_scales"], err=st["err"])
        if case["op"] == "attend":
            return spd.paged_attention(st["q"], st["k_pages"], st["v_pages"], st["cu"], st["lens"], st["table"], max_new=st["max_new"],
                                       max_context=st["max_context"], window=case["window"], sinks=case["sinks"], **kv)
        if case["op"] == "write":
            spd.kv_write(st["k"], st["v"], st["k_pages"], st["v_pages"], st["cu"], st["lens"], st["table"], **kv)
            return spd.kv_read(st["k_pages"], st["v_pages"], st["cu"], st["lens"], st["table"], n_tokens=st["n"], dtype=dtype, **kv)
        return spd.kv_read(st["k_pages"], st["v_pages"], st["cu"], st["starts"], st["table"], n_tokens=st["n"], dtype=dtype, **kv)

    if case["op"] == "write":
        _, _, page, row = _where(st, st["lens"], st["n"])
        for t in ("k", "v"):
            p = st[t + "_pages"]
            if st[t + "_scales"] is None:
                p[page, :, row] = st[t].to(p.dtype)
            else:
                codes, s = _quantise(st[t].float(), case["fmt"])
                _codes(p)[page, :, row] = _codes(codes)
                st[t + "_scales"][page, :, row] = s
        return tuple(_read(st, st["n"], page, row, dtype))
    if case["op"] == "read":
        _, _, page, row = _where(st, st["starts"], st["n"])
        return tuple(_read(st, st["n"], page, row, dtype))

    B, nq, nkv, d, page, T, L = st["B"], case["nq"], case["nkv"], case["d"], case["page"], st["max_context"], st["max_new"]
    dev = st["q"].device
    key = torch.arange(T, device=dev)
    pages = st["table"][:, :-(-T // page)].long()
    kv = []
    for t in ("k", "v"):  # padded [B, nkv, T, d] in float32
        p, s = st[t + "_pages"], st[t + "_scales"]
        x = _codes(p)[pages].view(p.dtype).float()
        x = x if s is None else x * s[pages][..., None]
        kv.append(x.transpose(1, 2).reshape(B, nkv, -1, d)[:, :, :T])
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


def exact(case, seed):
    """The definition in float64, sequence by sequence."""
    st = prepare(case, seed)
    lens, new = _lengths(case)
    page, d, nkv = case["page"], case["d"], case["nkv"]

    def dequantised(t, b, first, count):
        p, s = st[t + "_pages"], st[t + "_scales"]
        tok = range(first, first + count)
        pg = torch.tensor([int(x) for x in st["table"][b].tolist()], device=p.device)[[x // page for x in tok]]
        r = torch.tensor([x % page for x in tok], device=p.device)
        x = p.view(torch.int8)[pg, :, r].view(p.dtype).to(torch.float64) if p.element_size() == 1 else p[pg, :, r].double()
        return x if s is None else x * s[pg, :, r].double().unsqueeze(-1)

    if case["op"] == "read":
        parts = [[dequantised(t, b, 0, a) for b, a in enumerate(lens) if a] for t in ("k", "v")]
        return tuple(torch.cat(p) for p in parts)
    if case["op"] == "write":
        out = []
        for t in ("k", "v"):
            x = st[t].double()
            if case["fmt"] == "bf16":
                x = st[t].to(torch.bfloat16).double()
            top = x.abs().amax(-1, keepdim=True)
            if case["fmt"] == "int8":
                step = torch.where(top > 0, top / 127, torch.ones_like(top))
                x = torch.round(x / step).clamp(-127, 127) * step
            if case["fmt"] == "e4m3":
                e = torch.ceil(torch.log2(top / 448)).clamp(min=-126)
                e = torch.where(torch.exp2(e - 1) * 448 >= top, e - 1, e)  # log2 may be off by its last bit at a power of two
                e = torch.where(torch.exp2(e) * 448 < top, e + 1, e)
                unit = torch.where(top > 0, torch.exp2(e), torch.ones_like(top))
                y = x / unit
                step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
                x = torch.round(y / step) * step * unit
            out.append(x)
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
