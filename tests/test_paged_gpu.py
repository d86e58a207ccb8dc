"""The paged-cache operators against float64 references: appending (plain and quantised), reading back, attention of new tokens."""
import itertools
import math

import pytest
import torch

import paper_2502_20727_b200 as spd
from paged_util import DTYPES, Batch, check_attention, quantise

pytestmark = pytest.mark.gpu


def attend(bt, d=None, **kw):
    d = d or bt.device()
    out = torch.full((bt.n, bt.nq, bt.d), 77.0, dtype=bt.dtype, device="cuda")
    got = spd.paged_attention(d["q"], d["k_pages"], d["v_pages"], d["cu"], d["lens"], d["table"], max_new=kw.pop("max_new", bt.max_new()),
                              max_context=kw.pop("max_context", bt.max_context()), window=bt.window, sinks=bt.sinks, err=d["err"],
                              k_scales=d["k_scales"], v_scales=d["v_scales"], out=out, **kw)
    assert got is out
    return out, int(d["err"].item())


def run_and_check(bt, **kw):
    out, err = attend(bt, **kw)
    assert err == 0
    live = check_attention(bt, out)
    assert (out.cpu()[~live] == 77.0).all(), "rows of nobody were written"
    return out


# ---- appending and reading back ----------------------------------------------------------------------------------
WRITE_SHAPES = [  # (nkv, d, page, lens, new)
    (8, 128, 16, [0, 5, 15, 16, 100], [1, 1, 1, 1, 1]),
    (2, 64, 16, [3, 0, 30], [40, 0, 17]),
    (5, 32, 8, [7], [33]),
    (1, 128, 48, [0, 47, 48], [1, 2, 95]),
    (40, 128, 16, [9, 1], [3, 21]),
]


@pytest.mark.parametrize("dtype,fmt", [("bf16", "bf16"), ("bf16", "e4m3"), ("bf16", "int8"), ("f32", "f32"), ("f32", "e4m3"), ("f32", "int8"),
                                       ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("shape", range(len(WRITE_SHAPES)))
def test_write_then_read(dtype, fmt, shape):
    nkv, d, page, lens, new = WRITE_SHAPES[shape]
    bt = Batch(dtype=dtype, fmt="bf16" if fmt == "bf16" else "f32" if fmt == "f32" else fmt, nq=nkv, nkv=nkv, d=d, page=page, lens=lens, new=new,
               lead=2, behind=3, seed=shape)
    g = torch.Generator().manual_seed(100 + shape)
    fused = (torch.randn((bt.n, 3 * nkv, d), generator=g) * torch.exp(2 * torch.randn((bt.n, 3 * nkv, 1), generator=g))).to(DTYPES[dtype])
    fused[bt.cu[0] + 1 if bt.n > bt.cu[0] + 1 else bt.cu[0], nkv] = 0  # a row of zeros
    dev = bt.device()
    x = fused.cuda()
    k, v = x[:, nkv:2 * nkv], x[:, 2 * nkv:]  # strided slices of one projection output
    before = {n: dev[n + "_pages"].clone() for n in "kv"}
    before_s = {n: None if dev[n + "_scales"] is None else dev[n + "_scales"].clone() for n in "kv"}
    spd.kv_write(k, v, dev["k_pages"], dev["v_pages"], dev["cu"], dev["lens"], dev["table"], err=dev["err"], k_scales=dev["k_scales"],
                 v_scales=dev["v_scales"])
    assert int(dev["err"].item()) == 0
    touched = torch.zeros((bt.n_pages, page), dtype=torch.bool)
    for name, src in (("k", fused[:, nkv:2 * nkv]), ("v", fused[:, 2 * nkv:])):
        pages = dev[name + "_pages"].cpu()
        for b in range(bt.B):
            for i in range(new[b]):
                p, s = bt.row_of(b, lens[b] + i)
                touched[p, s] = True
                row = src[bt.cu[b] + i].double()
                got = pages[p, :, s]
                if fmt in ("bf16", "f32"):
                    assert torch.equal(got, src[bt.cu[b] + i].to(DTYPES[fmt]))
                    continue
                codes, scale = quantise(row, fmt)
                gs = dev[name + "_scales"].cpu()[p, :, s]
                top = row.abs().amax(-1)
                if fmt == "e4m3":
                    assert torch.equal(gs, scale)
                    assert torch.equal(got.view(torch.uint8), codes.view(torch.uint8))
                else:  # one rounding of the scale; codes of values a rounding of the product away from a tie may go either way
                    assert ((gs.double() - torch.where(top > 0, top / 127, torch.ones_like(top))).abs() <= 2.0 ** -24 * top / 127 + 1e-45).all()
                    exact = torch.where(top[:, None] > 0, row * 127 / top[:, None].clamp(min=1e-300), row)
                    assert ((got.double() - exact).abs() <= 0.5 + 127 * 2.0 ** -22).all()
    # every other slot keeps its bits
    for name in "kv":
        same = (dev[name + "_pages"].cpu().view(torch.uint8) == before[name].cpu().view(torch.uint8)).view(bt.n_pages, nkv, page, -1).all(-1).all(1)
        assert same[~touched].all()
        if before_s[name] is not None:
            a, b_ = dev[name + "_scales"].cpu().view(torch.int32), before_s[name].cpu().view(torch.int32)
            assert (a == b_).all(1)[~touched].all()
    # reading back gives code * scale, rounded once; rows of nobody stay
    out_dtype = torch.float32 if dtype == "f32" else torch.bfloat16
    ko, vo = (torch.full((bt.n, nkv, d), 55.0, dtype=out_dtype, device="cuda") for _ in range(2))
    spd.kv_read(dev["k_pages"], dev["v_pages"], dev["cu"], dev["lens"], dev["table"], err=dev["err"], k_scales=dev["k_scales"],
                v_scales=dev["v_scales"], out=(ko, vo))
    assert int(dev["err"].item()) == 0
    for name, o in (("k", ko.cpu()), ("v", vo.cpu())):
        pages, sc = dev[name + "_pages"].cpu(), dev[name + "_scales"]
        for b in range(bt.B):
            for i in range(new[b]):
                p, s = bt.row_of(b, lens[b] + i)
                val = pages[p, :, s].float()
                if sc is not None:
                    val = val * sc.cpu()[p, :, s][:, None]
                assert torch.equal(o[bt.cu[b] + i], val.to(out_dtype))
        assert (o[:bt.cu[0]] == 55.0).all() and (o[bt.cu[-1]:] == 55.0).all()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_quantise_special_rows(fmt):
    """Largest and smallest floats, NaN and infinity: the row concerned only."""
    d, nkv = 64, 1
    rows = torch.zeros((7, nkv, d))
    rows[0, 0, 3] = 3.4e38
    rows[1, 0, :] = 1e-38
    rows[2, 0, 5] = 1e-45
    rows[3, 0, 0] = math.nan
    rows[4, 0, 0] = -math.inf
    rows[5, 0, :] = torch.linspace(-448, 448, d)
    rows[6, 0, :] = -2.0 ** torch.linspace(-30, 5, d)
    bt = Batch(dtype="f32", fmt=fmt, nq=1, nkv=1, d=d, page=16, lens=[0], new=[7])
    dev = bt.device()
    x = rows.cuda()
    a = dict(err=dev["err"], k_scales=dev["k_scales"], v_scales=dev["v_scales"])
    spd.kv_write(x, x, dev["k_pages"], dev["v_pages"], dev["cu"], dev["lens"], dev["table"], **a)
    k, v = spd.kv_read(dev["k_pages"], dev["v_pages"], dev["cu"], dev["lens"], dev["table"], n_tokens=7, dtype=torch.float32, **a)
    assert torch.equal(k.nan_to_num(1.5), v.nan_to_num(1.5)) and int(dev["err"].item()) == 0
    k = k.cpu()
    assert torch.isnan(k[3]).all() and torch.isnan(k[4]).all()
    for r in (0, 1, 2, 5, 6):
        top = rows[r].abs().max().double()
        # e4m3: half a step of the value, or of the smallest normal code (2^-9 s / 2, s < top / 224); int8: half a step of s
        tol = torch.maximum(rows[r].double().abs() * 2.0 ** -4, top / 224 * 2.0 ** -10) if fmt == "e4m3" else (top / 127 * 0.5001).expand_as(rows[r])
        assert ((k[r].double() - rows[r].double()).abs() <= tol + 2.0 ** -126).all(), r  # scales stop at 2^-126


def test_write_and_read_flag_what_does_not_fit():
    bt = Batch(dtype="bf16", fmt="bf16", nq=2, nkv=2, d=64, page=16, lens=[0, 10], new=[4, 4])
    dev = bt.device()
    x = torch.ones((8, 2, 64), dtype=torch.bfloat16, device="cuda")
    call = lambda t, l: spd.kv_write(x, x, dev["k_pages"], dev["v_pages"], dev["cu"], l, t, err=dev["err"])  # noqa: E731
    before = dev["k_pages"].clone()
    for entry, lens, bit in ((bt.n_pages, dev["lens"], 1), (-1, dev["lens"], 1), (0, torch.tensor([-3, 16 * bt.width], dtype=torch.int32, device="cuda"), 2)):
        t = torch.full_like(dev["table"], entry)
        dev["err"].zero_()
        call(t, lens)
        assert int(dev["err"].item()) == bit
        if bit == 1:
            assert torch.equal(before.view(torch.int16), dev["k_pages"].view(torch.int16))
            k, v = (torch.full((8, 2, 64), 5.0, device="cuda") for _ in range(2))
            dev["err"].zero_()
            spd.kv_read(dev["k_pages"], dev["v_pages"], dev["cu"], lens, t, err=dev["err"], out=(k, v))
            assert int(dev["err"].item()) == bit and (k == 5).all() and (v == 5).all()


# ---- attention ---------------------------------------------------------------------------------------------------
HEADS = [(8, 8), (8, 2), (16, 2), (10, 2), (1, 1), (24, 8)]
BATCHES = [  # (lens, new): single tokens, an empty cache, an empty chunk, tile edges, long chunks
    ([0, 1, 15, 16, 17, 200], [1, 1, 1, 1, 1, 1]),
    ([0, 127, 128, 300], [5, 1, 3, 2]),
    ([40, 0, 7], [0, 130, 65]),
    ([513], [257]),
    ([0], [1]),
]
TYPES = [("bf16", "bf16"), ("bf16", "e4m3"), ("bf16", "int8"), ("f32", "f32"), ("f32", "e4m3"), ("f32", "int8")]


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("batch", range(len(BATCHES)))
@pytest.mark.parametrize("d", [128, 64])
def test_attention(types, batch, d):
    lens, new = BATCHES[batch]
    nq, nkv = HEADS[(batch + (d == 64)) % len(HEADS)]
    run_and_check(Batch(dtype=types[0], fmt=types[1], nq=nq, nkv=nkv, d=d, page=16, lens=lens, new=new, lead=1, behind=2, seed=batch))


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("heads", HEADS)
def test_attention_head_layouts(types, heads):
    run_and_check(Batch(dtype=types[0], fmt=types[1], nq=heads[0], nkv=heads[1], d=64, page=16, lens=[37, 90], new=[9, 30], seed=3))


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("page", [1, 8, 24, 32, 64, 256])
def test_attention_page_sizes(types, page):
    run_and_check(Batch(dtype=types[0], fmt=types[1], nq=8, nkv=2, d=128, page=page, lens=[70, 0, 129], new=[1, 40, 33], seed=page))
    run_and_check(Batch(dtype=types[0], fmt=types[1], nq=8, nkv=2, d=64, page=page, lens=[70, 255], new=[1, 1], seed=page))


@pytest.mark.parametrize("types", TYPES)
def test_attention_head_dim_32(types):
    run_and_check(Batch(dtype=types[0], fmt=types[1], nq=4, nkv=2, d=32, page=16, lens=[70, 0], new=[1, 40], window=20, sinks=2, seed=2))


WINDOWS = [(1, 0), (1, 1), (16, 4), (17, 16), (100, 3), (128, 130), (1000, 5), (64, 1)]


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("window", WINDOWS)
def test_attention_window_and_sinks(types, window):
    for d, lens, new in ((128, [300, 0, 64, 1], [1, 1, 1, 1]), (128, [400, 0, 131], [37, 150, 1]), (64, [700], [260])):
        run_and_check(Batch(dtype=types[0], fmt=types[1], nq=8, nkv=4, d=d, page=16, lens=lens, new=new, window=window[0], sinks=window[1], seed=5))


@pytest.mark.parametrize("types", TYPES)
def test_attention_long_context_single_tokens(types):
    run_and_check(Batch(dtype=types[0], fmt=types[1], nq=8, nkv=1, d=128, page=16, lens=[5000, 3, 2049], new=[1, 1, 1], seed=6))
    run_and_check(Batch(dtype=types[0], fmt=types[1], nq=4, nkv=1, d=128, page=16, lens=[4000, 90], new=[5, 20], window=1500, sinks=4, seed=7))


@pytest.mark.parametrize("types", TYPES)
def test_attention_sharp_softmax(types):
    """Scores of very unequal size: the running maximum moves late and far."""
    for new in (1, 3, 140):
        run_and_check(Batch(dtype=types[0], fmt=types[1], nq=4, nkv=2, d=64, page=16, lens=[400], new=[new], seed=8, spread=4.0))


def test_attention_strided_and_scaled():
    bt = Batch(dtype="bf16", fmt="bf16", nq=8, nkv=2, d=64, page=16, lens=[20, 3], new=[1, 70], seed=9)
    dev = bt.device()
    wide = torch.zeros((bt.n, 12, 64), dtype=torch.bfloat16, device="cuda")
    wide[:, :8] = dev["q"]
    out_wide = torch.full((bt.n, 11, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    spd.paged_attention(wide[:, :8], dev["k_pages"], dev["v_pages"], dev["cu"], dev["lens"], dev["table"], max_new=bt.max_new() + 50,
                        max_context=bt.width * 16, err=dev["err"], out=out_wide[:, 2:10], scale=0.03)
    assert int(dev["err"].item()) == 0
    check_attention(bt, out_wide[:, 2:10], scale=0.03)
    assert (out_wide[:, :2] == 3).all() and (out_wide[:, 10:] == 3).all()


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("new", [1, 6, 150])
def test_a_key_that_is_not_seen_has_no_influence(types, new):
    """NaN and infinities in the last cached row: the queries before it are as if it were not there."""
    for bad in (math.nan, math.inf):
        bt = Batch(dtype=types[0], fmt=types[1], nq=8, nkv=4, d=128, page=16, lens=[90], new=[new], seed=11)
        dev = bt.device()
        p, s = bt.row_of(0, 90 + new - 1)
        for n in "kv":
            if dev[n + "_scales"] is None:
                dev[n + "_pages"][p, :, s, 7] = bad
            else:
                dev[n + "_scales"][p, :, s] = bad
        out, err = attend(bt, dev)
        assert err == 0
        last = bt.cu[-1] - 1
        ref, tol = bt.reference()
        got = out.double().cpu()
        assert ((got - ref).abs()[:last] <= tol[:last]).all()
        assert not torch.isfinite(got[last]).all()


def test_a_visible_infinity_in_v_reaches_the_queries_that_see_it():
    for new, at in ((150, 100), (150, 20), (4, 91), (1, 90)):
        bt = Batch(dtype="bf16", fmt="bf16", nq=4, nkv=2, d=128, page=16, lens=[90], new=[new], seed=12)
        dev = bt.device()
        p, s = bt.row_of(0, at)
        dev["v_pages"][p, 1, s, 9] = math.inf
        out, err = attend(bt, dev)
        got = out.double().cpu()
        ref, tol = bt.reference()
        hit = torch.zeros_like(ref, dtype=torch.bool)
        first = max(0, at - 90)
        hit[first:, 2:, 9] = True
        assert err == 0 and (torch.isinf(got[hit]) | torch.isnan(got[hit])).all()
        assert ((got - ref).abs()[~hit] <= tol[~hit]).all()


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("new", [1, 20, 200])
def test_bad_batches_are_flagged_and_skipped(types, new):
    bt = Batch(dtype=types[0], fmt=types[1], nq=4, nkv=2, d=64, page=16, lens=[50, 60], new=[new, new], seed=13)
    # more new tokens than the call's bound, a length beyond it, a negative length, rows outside the tensor
    for what in ("new", "context", "negative", "rows"):
        dev = bt.device()
        kw = {}
        if what == "new":
            if new == 1:
                continue
            kw["max_new"] = new - 1
        elif what == "context":
            kw["max_context"] = 50 + new
        elif what == "negative":
            dev["lens"][1] = -1
        else:
            dev["cu"][2] = bt.n + 1
        out, err = attend(bt, dev, **kw)
        assert err == 2, what
        if what != "new":
            assert (out[bt.cu[1]:] == 77).all()
            ref, tol = bt.reference()
            assert ((out.double().cpu() - ref).abs() <= tol)[:bt.cu[1]].all()
        else:
            assert (out == 77).all()
    for entry in (-1, bt.n_pages):
        dev = bt.device()
        dev["table"][0, 1] = entry
        out, err = attend(bt, dev)
        assert err == 1
        ref, tol = bt.reference()
        assert ((out.double().cpu() - ref).abs() <= tol)[bt.cu[1]:].all()


@pytest.mark.parametrize("types", TYPES)
def test_attention_is_deterministic_and_replays(types):
    for lens, new in (([700, 30, 1], [1, 1, 1]), ([300, 20], [30, 200])):
        bt = Batch(dtype=types[0], fmt=types[1], nq=8, nkv=2, d=128, page=16, lens=lens, new=new, seed=14)
        dev = bt.device()
        first = run_and_check(bt)
        second, _ = attend(bt, dev)
        assert torch.equal(first, second)
        static = torch.zeros_like(first)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        graphs = []
        with torch.cuda.stream(side):
            for _ in range(2):  # two captured calls, replayed in turn
                g = torch.cuda.CUDAGraph()
                with torch.cuda.graph(g, stream=side):
                    spd.paged_attention(dev["q"], dev["k_pages"], dev["v_pages"], dev["cu"], dev["lens"], dev["table"], max_new=bt.max_new(),
                                        max_context=bt.max_context(), err=dev["err"], k_scales=dev["k_scales"], v_scales=dev["v_scales"], out=static)
                graphs.append(g)
            for g in graphs * 2:
                static.zero_()
                g.replay()
        side.synchronize()
        assert torch.equal(static, first) and int(dev["err"].item()) == 0


def test_two_streams_at_once():
    a = Batch(dtype="bf16", fmt="bf16", nq=8, nkv=2, d=128, page=16, lens=[3000, 20], new=[1, 1], seed=15)
    b = Batch(dtype="bf16", fmt="int8", nq=8, nkv=1, d=128, page=16, lens=[100, 2000], new=[40, 3], seed=16)
    da, db = a.device(), b.device()
    torch.cuda.synchronize()
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    oa, ob = [], []
    for _ in range(5):
        with torch.cuda.stream(sa):
            oa.append(attend_no_sync(a, da))
        with torch.cuda.stream(sb):
            ob.append(attend_no_sync(b, db))
    torch.cuda.synchronize()
    for o in oa:
        check_attention(a, o)
    for o in ob:
        check_attention(b, o)


def attend_no_sync(bt, d):
    return spd.paged_attention(d["q"], d["k_pages"], d["v_pages"], d["cu"], d["lens"], d["table"], max_new=bt.max_new(), max_context=bt.max_context(),
                               window=bt.window, sinks=bt.sinks, err=d["err"], k_scales=d["k_scales"], v_scales=d["v_scales"])


@pytest.mark.parametrize("types", [t for t in TYPES if t[0] == "bf16"])
def test_write_then_attend_step_by_step(types):
    """As it is used: a prompt is written and attended, then single tokens one by one, then a chunk - against one attention over
    everything, on the same cached codes."""
    nq, nkv, d, page, lens = 8, 2, 128, 16, [0, 0]
    total, steps = [70, 33], [(50, 20), (1, 1), (1, 1), (18, 11)]
    bt = Batch(dtype=types[0], fmt=types[1], nq=nq, nkv=nkv, d=d, page=page, lens=[0, 0], new=total, seed=17)
    dev = bt.device()
    for n in "kv":  # the cache starts empty
        dev[n + "_pages"] = torch.zeros_like(dev[n + "_pages"].view(torch.uint8)).view(dev[n + "_pages"].dtype)
    kv = {n: torch.randn((sum(total), nkv, d), generator=torch.Generator().manual_seed(ord(n))).to(bt.dtype).cuda() for n in "kv"}
    a = dict(err=dev["err"], k_scales=dev["k_scales"], v_scales=dev["v_scales"])
    outs = [[], []]
    at = [0, 0]
    for step in steps:
        rows = torch.cat([torch.arange(at[b], at[b] + step[b]) + bt.cu[b] for b in range(2)]).cuda()
        cu = torch.tensor([0, step[0], step[0] + step[1]], dtype=torch.int32, device="cuda")
        ls = torch.tensor(at, dtype=torch.int32, device="cuda")
        spd.kv_write(kv["k"][rows], kv["v"][rows], dev["k_pages"], dev["v_pages"], cu, ls, dev["table"], **a)
        o = spd.paged_attention(dev["q"][rows], dev["k_pages"], dev["v_pages"], cu, ls, dev["table"], max_new=max(step),
                                max_context=max(x + y for x, y in zip(at, step)), **a)
        outs[0].append(o[:step[0]])
        outs[1].append(o[step[0]:])
        at = [x + y for x, y in zip(at, step)]
    assert at == total and int(dev["err"].item()) == 0
    k, v = spd.kv_read(dev["k_pages"], dev["v_pages"], dev["cu"], torch.zeros_like(dev["lens"]), dev["table"], n_tokens=bt.n, dtype=torch.float32, **a)
    for name, x in (("k", k.double().cpu()), ("v", v.double().cpu())):
        for b in range(2):
            for t in range(total[b]):
                p, s = bt.row_of(b, t)
                bt.values[name][p, :, s] = x[bt.cu[b] + t]
    check_attention(bt, torch.cat([torch.cat(o) for o in outs]))
