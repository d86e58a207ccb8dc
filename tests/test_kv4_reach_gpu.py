"""Attention over a 4-bit cache at the far ends: batches whose keys are dealt out over the whole GPU, rows of any finite size that a query does not see,
caches beyond 32-bit offsets, calls that overlap."""
import math
import random
import threading

import pytest
import torch

import paper_2502_20727_b200 as spd
from kv4_util import Batch4, values4
from paged_util import check_attention
from test_paged_gpu import attend, run_and_check

pytestmark = pytest.mark.gpu
BOUND = 4096  # the host's bound of a sequence's length, by which such a batch is told from small ones


def many(B=70, top=260, new=1, nq=16, nkv=8, d=128, page=16, seed=0, **kw):
    """More (sequence, KV head, 32 keys) than 16 for each warp that 148 SMs hold, by the bound."""
    assert B * nkv * (BOUND // 32) >= 16 * 148 * 12 and B <= 512
    rng = random.Random(seed)
    lens = [rng.choice([0, 1, 31, 32, 33, top, rng.randint(0, top)]) for _ in range(B)]
    bt = Batch4(dtype="bf16", nq=nq, nkv=nkv, d=d, page=page, lens=lens, new=[rng.randint(0, new) if new > 1 else 1 for _ in range(B)], lead=1, behind=2,
                seed=seed, offset=0.3, **kw)
    bt.table = torch.cat([bt.table, torch.full((B, -(-BOUND // page)), -7, dtype=torch.int32)], 1)
    return bt


def run(bt):
    out, err = attend(bt, max_context=BOUND)
    assert err == 0
    live = check_attention(bt, out)
    assert (out.cpu()[~live] == 77.0).all()
    return out


@pytest.mark.parametrize("nq,new", [(8, 1), (16, 1), (64, 1), (16, 4), (16, 8), (64, 2), (72, 1), (128, 1), (8, 16)])
@pytest.mark.parametrize("d", [128, 64])
def test_many_sequences(nq, new, d):
    run(many(nq=nq, new=new, d=d, seed=nq + new))


@pytest.mark.parametrize("page", [1, 8, 24, 32, 48, 64])
@pytest.mark.parametrize("new", [1, 6])
def test_many_sequences_page_sizes(page, new):
    run(many(nq=16, new=new, page=page, seed=page))


@pytest.mark.parametrize("window", [(1, 0), (17, 3), (100, 40), (64, 130)])
def test_many_sequences_with_a_window(window):
    for new in (1, 5):
        run(many(nq=16, new=new, top=400, window=window[0], sinks=window[1], seed=7 + new))


def test_many_sequences_several_steps_a_warp():
    run(many(B=64, top=2500, nq=8, seed=3))
    run(many(B=40, top=1500, new=2, nq=56, seed=4))


def test_many_sequences_replay_and_overlap():
    """The same bits every time; two streams at once, each call with a workspace of its own; a workspace that two captured graphs share in turn."""
    bt = many(seed=5)
    first = run(bt)
    d = bt.device()
    torch.cuda.synchronize()
    call = lambda **kw: spd.paged_attention(d["q"], d["k_pages"], d["v_pages"], d["cu"], d["lens"], d["table"], max_new=1, max_context=BOUND, err=d["err"],  # noqa: E731
                                            k_scales=d["k_scales"], v_scales=d["v_scales"], **kw)
    outs = []
    streams = [torch.cuda.Stream() for _ in range(3)]
    for _ in range(4):
        for s in streams:
            with torch.cuda.stream(s):
                outs.append(call())
    torch.cuda.synchronize()
    live = torch.arange(bt.cu[0], bt.cu[-1])
    assert all(torch.equal(o[live], first[live]) for o in outs)
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    static = [torch.zeros_like(first) for _ in range(2)]
    side = streams[0]
    graphs = []
    with torch.cuda.stream(side):
        for o in static:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                call(out=o, workspace=ws)
            graphs.append(g)
        ws.fill_(255)
        for g in graphs * 2:
            g.replay()
    side.synchronize()
    assert all(torch.equal(o[live], first[live]) for o in static) and int(d["err"]) == 0
    with pytest.raises(spd.SpdError):
        call(workspace=ws[:1024])


def test_many_sequences_what_does_not_fit():
    bt = many(seed=6)
    ref, tol = bt.reference()
    for what in ("negative", "context", "rows", "page"):
        dev = bt.device()
        b = max(range(bt.B), key=lambda i: bt.lens[i])
        if what == "negative":
            dev["lens"][b] = -1
        elif what == "context":
            dev["lens"][b] = BOUND
        elif what == "rows":
            b = bt.B - 1
            dev["cu"][bt.B] = bt.n + 1
        else:
            dev["table"][b, 0] = bt.n_pages
        out, err = attend(bt, dev, max_context=BOUND)
        assert err == (1 if what == "page" else 2), what
        row = bt.cu[b]
        keep = [i for i in range(bt.cu[0], bt.cu[-1]) if i != row]
        assert ((out.double().cpu() - ref).abs() <= tol)[keep].all(), what
        if what != "page":
            assert (out[row] == 77).all(), what


def test_many_sequences_rows_that_are_not_finite():
    """One sequence's row in one KV head, anywhere in its keys: that sequence's heads there are NaN, nothing else changes."""
    bt = many(seed=8)
    ref, tol = bt.reference()
    b = max(range(bt.B), key=lambda i: bt.lens[i])
    for t in (0, 31, bt.lens[b] // 2, bt.lens[b]):
        for what in ("k_scales", "v_scales"):
            dev = bt.device()
            p, s = bt.row_of(b, t)
            dev[what][p, 5, s, 1, 0] = math.nan
            out, err = attend(bt, dev, max_context=BOUND)
            assert err == 0
            got = out.double().cpu()
            hit = torch.zeros_like(ref, dtype=torch.bool)
            hit[bt.cu[b], 10:12] = True
            dead = torch.isnan(ref)
            assert torch.isnan(got[hit]).all()
            assert ((got - ref).abs() <= tol)[~hit & ~dead].all()


@pytest.mark.parametrize("size", [2.0 ** 12, 2.0 ** 29, 2.0 ** 60, 3.0e38])
@pytest.mark.parametrize("new", [2, 8, 150])
@pytest.mark.parametrize("nq", [4, 8])
def test_finite_rows_of_any_size_that_are_not_seen(size, new, nq):
    """The last cached row's values are huge: the queries before it are as if it were not there, to the last bit of what they are bounded by."""
    tried = 0
    for window, at in ((0, -1), (33, 8), (40, 10)):  # the newest row; rows that the window has passed for all but the first queries
        bt = Batch4(dtype="bf16", nq=nq, nkv=4, d=128, page=16, lens=[40], new=[new], window=window, seed=11)
        dev = bt.device()
        t = 40 + new - 1 if at < 0 else at
        p, s = bt.row_of(0, t)
        if int(bt.table[0, t // 16]) != p:
            continue
        for name in ("k_scales", "v_scales"):
            dev[name][p, :, s, :, 0] = size / 16
            dev[name][p, :, s, :, 1] = -size
        out, err = attend(bt, dev)
        assert err == 0
        ref, tol = bt.reference()
        pos = torch.arange(40, 40 + new)
        blind = (pos < t) | ((pos - window >= t) if window else torch.zeros_like(pos, dtype=torch.bool))
        got = out.double().cpu()
        assert ((got - ref).abs() <= tol)[blind].all()
        tried += int(blind.any())
    assert tried >= 2


@pytest.mark.parametrize("page", [16, 24])
def test_pages_beyond_32_bit_offsets(page):
    """The batch's pages are the last ones of a cache of more than 2^32 bytes (K and V share it, at different pages)."""
    bts = [Batch4(dtype="bf16", nq=4, nkv=2, d=128, page=page, lens=[70, 9], new=new, seed=3) for new in ([1, 1], [12, 3], [60, 1])]
    bts.append(Batch4(dtype="f32", nq=4, nkv=2, d=128, page=page, lens=[70, 9], new=[5, 1], seed=3))
    n_big = 2 ** 32 // (2 * page * 64) + 200
    pages = torch.empty((n_big, 2, page, 64), dtype=torch.uint8, device="cuda")
    scales = torch.empty((n_big, 2, page, 2, 2), dtype=torch.bfloat16, device="cuda")
    for bt in bts:
        d = bt.device()
        n = bt.n_pages
        assert n <= 100
        kp, ks, vp, vs = pages[100:], scales[100:], pages[:n_big - 100], scales[:n_big - 100]
        for t, key in ((kp, "k_pages"), (ks, "k_scales"), (vp, "v_pages"), (vs, "v_scales")):
            t[-n:].copy_(d[key])
        table = torch.where((d["table"] >= 0) & (d["table"] < n), d["table"] + (n_big - 100 - n), d["table"])
        out = torch.full((bt.n, 4, 128), 77.0, dtype=bt.dtype, device="cuda")
        kw = dict(k_scales=ks, v_scales=vs, err=d["err"])
        spd.paged_attention(d["q"], kp, vp, d["cu"], d["lens"], table, max_new=bt.max_new(), max_context=bt.max_context(), out=out, **kw)
        assert int(d["err"]) == 0
        check_attention(bt, out)
        cu, zero = torch.tensor([0, 50], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        k, v = spd.kv_read(kp, vp, cu, zero, table[:1], n_tokens=50, dtype=bt.dtype, **kw)
        k2, v2 = spd.kv_read(d["k_pages"], d["v_pages"], cu, zero, d["table"][:1], n_tokens=50, dtype=bt.dtype, err=d["err"], k_scales=d["k_scales"], v_scales=d["v_scales"])
        assert torch.equal(k, k2) and torch.equal(v, v2)
        # what was read, appended again: by slots at the far end of the cache
        t = torch.arange(50, device="cuda")
        slots = (table[0].long()[t // page] * page + t % page).to(torch.int32)
        spd.kv_write_slots(k, k, kp, vp, slots, **kw)
        k3, v3 = spd.kv_read(kp, vp, cu, zero, table[:1], n_tokens=50, dtype=torch.float32, **kw)
        assert torch.equal(k3, v3) and int(d["err"]) == 0
        # values of a 4-bit row, quantised again: m is m again, s within its two roundings
        assert (k3 - k.float()).abs().max() <= 2.0 ** -7 * 16 * k.float().abs().max()
    del pages, scales, kp, ks, vp, vs
    torch.cuda.empty_cache()


@pytest.mark.parametrize("new", [1, 40])
def test_sequences_that_share_pages(new):
    """The same pages under two sequences of a batch (a shared prefix): both see what one alone sees."""
    bt = Batch4(dtype="bf16", nq=8, nkv=2, d=128, page=16, lens=[100], new=[new], seed=5)
    d = bt.device()
    kw = dict(max_new=new, max_context=100 + new, err=d["err"], k_scales=d["k_scales"], v_scales=d["v_scales"])
    one = spd.paged_attention(d["q"], d["k_pages"], d["v_pages"], d["cu"], d["lens"], d["table"], **kw)
    two = spd.paged_attention(torch.cat([d["q"], d["q"]]), d["k_pages"], d["v_pages"], torch.tensor([0, new, 2 * new], dtype=torch.int32, device="cuda"),
                              d["lens"].repeat(2), d["table"].repeat(2, 1), **kw)
    check_attention(bt, one)
    assert torch.equal(two[:new], two[new:]) and int(d["err"]) == 0
    check_attention(bt, two[:new])


@pytest.mark.parametrize("nq,nkv", [(32, 1), (71, 1), (128, 1), (400, 2)])
def test_many_query_heads_per_kv_head(nq, nkv):
    run_and_check(Batch4(dtype="bf16", nq=nq, nkv=nkv, d=64, page=16, lens=[150, 0, 40], new=[1, 1, 1], seed=31))
    run_and_check(Batch4(dtype="bf16", nq=nq, nkv=nkv, d=64, page=16, lens=[97], new=[4], window=50, sinks=3, seed=32))


def test_threads_that_call_at_once():
    """First calls of several variants from several threads, each on a stream of its own."""
    bts = [Batch4(dtype=t, nq=8, nkv=2, d=d, page=page, lens=[200, 30], new=[new, 1], seed=34) for t in ("bf16", "f32") for d, page, new in ((128, 16, 1), (64, 24, 40), (64, 16, 5))]
    bts.append(many(seed=35))
    ds = [bt.device() for bt in bts]
    outs, bad = [None] * len(bts), []
    torch.cuda.synchronize()
    start = threading.Barrier(len(bts))

    def work(i):
        try:
            bt, d = bts[i], ds[i]
            with torch.cuda.stream(torch.cuda.Stream()):
                start.wait()
                for _ in range(3):
                    outs[i] = spd.paged_attention(d["q"], d["k_pages"], d["v_pages"], d["cu"], d["lens"], d["table"], max_new=bt.max_new(),
                                                  max_context=BOUND if bt.B > 3 else bt.max_context(), err=d["err"], k_scales=d["k_scales"], v_scales=d["v_scales"])
                torch.cuda.current_stream().synchronize()
        except Exception as e:  # noqa: BLE001
            bad.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(bts))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad, bad
    for bt, d, out in zip(bts, ds, outs):
        assert int(d["err"]) == 0
        check_attention(bt, out)


def test_tensors_of_another_stream_and_strides():
    """Rows that are slices of one projection output, made on the stream that then attends; refusals of what does not fit the pages."""
    bt = Batch4(dtype="bf16", nq=8, nkv=2, d=128, page=16, lens=[20, 3], new=[1, 7], seed=9)
    d = bt.device()
    kw = dict(max_new=7, max_context=27, err=d["err"], k_scales=d["k_scales"], v_scales=d["v_scales"])
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        fused = torch.cat([d["q"] * 0, d["q"], d["q"] * 0], 1)
        out = spd.paged_attention(fused[:, 8:16], d["k_pages"], d["v_pages"], d["cu"], d["lens"], d["table"], **kw)
        torch.cuda.current_stream().synchronize()
    check_attention(bt, out)
    at = (d["cu"], d["lens"], d["table"])
    for q in (d["q"][:, :, ::2], d["q"].transpose(0, 1), d["q"].half(), d["q"][0], d["q"].cpu()):
        with pytest.raises(ValueError):
            spd.paged_attention(q, d["k_pages"], d["v_pages"], *at, **kw)
    for bad in (dict(k_scales=None), dict(v_scales=d["v_scales"].float()), dict(k_scales=d["k_scales"][..., :1]), dict(v_scales=d["v_scales"][:-1])):
        with pytest.raises(ValueError):
            spd.paged_attention(d["q"], d["k_pages"], d["v_pages"], *at, **{**kw, **bad})
    with pytest.raises(ValueError):
        spd.paged_attention(d["q"], d["k_pages"][..., :32], d["v_pages"], *at, **kw)
    with pytest.raises(spd.SpdError):
        spd.paged_attention(d["q"], d["k_pages"], d["v_pages"], *at, **{**kw, "max_new": 0})
    with pytest.raises(TypeError):
        spd.paged_attention([1.0], d["k_pages"], d["v_pages"], *at, **kw)


@pytest.mark.parametrize("nq,new,bound", [(64, 4, 40000), (64, 3, 4000), (8, 1, 40000), (16, 8, 70000)])
def test_key_ranges_by_the_host_bound(nq, new, bound):
    """Calls cut into key ranges for a far longer context than the sequences have: ranges without keys, rows beyond 16, tiles without rows."""
    bt = Batch4(dtype="bf16", nq=nq, nkv=8, d=128, page=16, lens=[0, 700, 31, 1, 300], new=[new, 1, new, 0, new], seed=41, behind=1)
    bt.table = torch.cat([bt.table, torch.full((bt.B, -(-bound // 16)), -7, dtype=torch.int32)], 1)
    out, err = attend(bt, max_context=bound)
    assert err == 0
    check_attention(bt, out)
    f32 = Batch4(dtype="f32", nq=16, nkv=2, d=128, page=16, lens=[0, 700, 31, 1, 300], new=[new, 1, 2, 0, 9], seed=42, behind=1)
    f32.table = torch.cat([f32.table, torch.full((f32.B, -(-bound // 16)), -7, dtype=torch.int32)], 1)
    out, err = attend(f32, max_context=bound)
    assert err == 0
    check_attention(f32, out)


@pytest.mark.parametrize("dtype,new", [("bf16", 1), ("bf16", 20), ("f32", 3)])
def test_scales_of_either_sign(dtype, new):
    """The caller's own parameters: negative scales, scales of zero."""
    bt = Batch4(dtype=dtype, nq=8, nkv=2, d=64, page=16, lens=[90, 5], new=[new, 1], seed=43)
    g = torch.Generator().manual_seed(1)
    for n in "kv":
        p = bt.scales[n]
        sign = torch.randint(-1, 2, p.shape[:-1], generator=g).to(p.dtype)
        p[..., 0] *= sign
        bt.values[n] = values4(bt.codes[n], p.nan_to_num(0.0))
    run_and_check(bt)


@pytest.mark.parametrize("power", [33, 45, 90])
@pytest.mark.parametrize("name", ["k", "v"])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("new", [1, 40])
def test_float32_calls_over_very_large_values(power, name, d, new):
    """K is brought back by the softmax scale.  V: three roundings at a size below 128 (half a step, 2^-18) of a score with its V row's exponent, in a
    weight and in the weights' sum: 6 ln 2 2^-18, under 2^-15.9 of the largest value that takes part."""
    bt = Batch4(dtype="f32", nq=8, nkv=2, d=d, page=16, lens=[120, 9], new=[new, 1], seed=44, rows=lambda n, x: x * 2.0 ** power if n == name else x)
    scale = d ** -0.5 * (2.0 ** -power if name == "k" else 1.0)
    out, err = attend(bt, scale=scale)
    assert err == 0
    ref, tol = bt.reference(scale)
    live = ~torch.isnan(ref[:, 0, 0])
    if name == "v":
        tol = tol + 2.0 ** -15.9 * bt.values["v"].nan_to_num(0.0).abs().max()
    assert ((out.double().cpu() - ref).abs() <= tol)[live].all()


def by_length(B, new, dtype="bf16", nq=64, d=128, seed=50):
    """One tile of rows per sequence and KV head, 19 to 128 sequences of 8 heads: more thread blocks than SMs, at most eight times as many."""
    rng = random.Random(seed)
    lens = [rng.choice([0, 0, 7, 31, 64, 64, rng.randint(0, 330)]) for _ in range(B)]
    return Batch4(dtype=dtype, nq=nq, nkv=8, d=d, page=16, lens=lens, new=[rng.choice([0, 1, new, new]) for _ in range(B)], lead=1, behind=2, seed=seed)


@pytest.mark.parametrize("dtype,nq,new,d", [("bf16", 64, 1, 128), ("bf16", 64, 1, 64), ("bf16", 16, 6, 128), ("bf16", 64, 5, 128), ("bf16", 64, 16, 64), ("f32", 8, 8, 64),
                                            ("f32", 64, 1, 128)])
@pytest.mark.parametrize("B", [19, 33, 127, 128, 129])
def test_sequences_by_length(dtype, nq, new, d, B):
    bt = by_length(B, new, dtype, nq, d, seed=B)
    run_and_check(bt)


@pytest.mark.parametrize("new", [1, 5])
def test_sequences_by_length_that_do_not_fit(new):
    bt = by_length(40, new)
    ref, tol = bt.reference()
    live = ~torch.isnan(ref[:, 0, 0])
    b = max((i for i in range(bt.B) if bt.new[i]), key=lambda i: bt.lens[i])
    for bad in (-1, -2 ** 31, 2 ** 31 - 1, bt.max_context()):
        dev = bt.device()
        dev["lens"][b] = bad
        out, err = attend(bt, dev)
        assert err == 2, bad
        keep = live.clone()
        keep[bt.cu[b]:bt.cu[b + 1]] = False
        assert ((out.double().cpu() - ref).abs() <= tol)[keep].all(), bad
        assert (out[bt.cu[b]:bt.cu[b + 1]] == 77).all(), bad
    dev = bt.device()  # offsets that run backwards: a sequence of a negative number of rows, and one that would have too many
    at = next(i for i in range(1, bt.B) if bt.new[i - 1] and bt.new[i])
    dev["cu"][at] = bt.n
    out, err = attend(bt, dev)
    assert err == 2
    keep = live.clone()
    keep[bt.cu[at - 1]:bt.cu[at + 1]] = False
    assert ((out.double().cpu() - ref).abs() <= tol)[keep].all()


def test_sequences_by_length_give_the_same_bits_in_any_order():
    bt = by_length(60, 1)
    first, _ = attend(bt)
    live = ~torch.isnan(bt.reference()[0][:, 0, 0]).cuda()
    dev = bt.device()
    order = torch.randperm(bt.B, generator=torch.Generator().manual_seed(1))
    new = torch.tensor(bt.new)[order]
    start = torch.cat([torch.zeros(1, dtype=torch.long), new.cumsum(0)])
    rows = torch.cat([torch.arange(bt.cu[b], bt.cu[b] + bt.new[b]) for b in order.tolist()]).cuda()
    dev["q"] = dev["q"][rows].contiguous()
    dev["cu"], dev["lens"], dev["table"] = start.int().cuda(), dev["lens"][order.cuda()].contiguous(), dev["table"][order.cuda()].contiguous()
    out = spd.paged_attention(dev["q"], dev["k_pages"], dev["v_pages"], dev["cu"], dev["lens"], dev["table"], max_new=bt.max_new(), max_context=bt.max_context(),
                              err=dev["err"], k_scales=dev["k_scales"], v_scales=dev["v_scales"])
    assert int(dev["err"]) == 0 and live[rows].all()
    assert torch.equal(out, first[rows])


@pytest.mark.parametrize("window,sinks", [(2500, 40), (2048, 0), (2100, 1000)])
def test_many_sequences_with_a_long_window(window, sinks):
    """Windows of as many keys as batches that are dealt out have."""
    run(many(top=3700, window=window, sinks=sinks, seed=60))
    run(many(B=64, top=3500, new=3, nq=32, window=window, sinks=sinks, seed=61))


@pytest.mark.parametrize("B,nq,nkv,new", [(1, 64, 8, 5), (1, 64, 8, 36), (2, 64, 8, 9), (1, 8, 1, 140), (1, 32, 32, 64), (1, 8, 8, 287), (3, 16, 2, 100), (4, 64, 8, 6), (1, 12, 4, 300),
                                          (2, 20, 4, 71), (6, 64, 8, 1), (2, 64, 8, 1), (3, 64, 8, 2), (11, 64, 8, 1), (1, 108, 108, 1)])
@pytest.mark.parametrize("d,window", [(128, 0), (64, 0), (128, 150)])
def test_many_rows_of_small_calls(B, nq, nkv, new, d, window):
    """Rows in tiles of 16 with an SM each, beside calls that just pass that bound; ranges as clusters that fill the GPU."""
    rng = random.Random(B + new)
    run_and_check(Batch4(dtype="bf16", nq=nq, nkv=nkv, d=d, page=16, lens=[rng.choice([0, 40, 700, 1300]) for _ in range(B)], new=[new] + [rng.randint(0, new) for _ in range(B - 1)],
                         window=window, sinks=9 if window else 0, lead=1, behind=2, seed=70))
