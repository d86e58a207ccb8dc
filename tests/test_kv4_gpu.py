"""The 4-bit paged cache against float64 references: appending (by block table and by slots), reading back, attention of new tokens."""
import math

import pytest
import torch

import paper_2502_20727_b200 as spd
from kv4_util import MIN_SCALE, Batch4, quantise4, values4
from paged_util import DTYPES, check_attention
from test_paged_gpu import BATCHES, HEADS, WINDOWS, WRITE_SHAPES, attend, run_and_check

pytestmark = pytest.mark.gpu
TYPES = ["bf16", "f32"]


def pages4(n_pages, nkv, page, d):
    """An empty cache: (k_pages, v_pages, k_scales, v_scales), codes 255 under NaN."""
    return [torch.full((n_pages, nkv, page, d // 2), 255, dtype=torch.uint8, device="cuda") for _ in "kv"] + \
        [torch.full((n_pages, nkv, page, 2, 2), math.nan, dtype=torch.bfloat16, device="cuda") for _ in "kv"]


def same_bits(a, b):
    return torch.equal(a.contiguous().view(torch.uint8).cpu(), b.contiguous().view(torch.uint8).cpu())


# ---- appending and reading back ----------------------------------------------------------------------------------
@pytest.mark.parametrize("by", ["table", "slots"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", range(len(WRITE_SHAPES)))
def test_write_then_read(dtype, shape, by):
    nkv, d, page, lens, new = WRITE_SHAPES[shape]
    bt = Batch4(dtype=dtype, nq=nkv, nkv=nkv, d=d, page=page, lens=lens, new=new, lead=2, behind=3, seed=shape)
    g = torch.Generator().manual_seed(100 + shape)
    fused = torch.randn((bt.n, 3 * nkv, d), generator=g) * torch.exp(2 * torch.randn((bt.n, 3 * nkv, 1), generator=g)) + torch.randn(d, generator=g)
    fused = fused.to(DTYPES[dtype])
    fused[bt.cu[0], nkv] = 0             # a row of zeros
    fused[bt.cu[0], 2 * nkv, :d // 2] = -3.25  # a constant half
    dev = bt.device()
    x = fused.cuda()
    k, v = x[:, nkv:2 * nkv], x[:, 2 * nkv:]  # strided slices of one projection output
    before = {n: dev[n].clone() for n in ("k_pages", "v_pages", "k_scales", "v_scales")}
    kv = dict(err=dev["err"], k_scales=dev["k_scales"], v_scales=dev["v_scales"])
    slots = torch.full((bt.n,), -1, dtype=torch.int32)
    for b in range(bt.B):
        for i in range(new[b]):
            p, s = bt.row_of(b, lens[b] + i)
            slots[bt.cu[b] + i] = p * page + s
    if by == "slots":
        spd.kv_write_slots(k, v, dev["k_pages"], dev["v_pages"], slots.cuda(), **kv)
    else:
        spd.kv_write(k, v, dev["k_pages"], dev["v_pages"], dev["cu"], dev["lens"], dev["table"], **kv)
    assert int(dev["err"].item()) == 0
    live = slots >= 0
    pg, row = (slots[live] // page).long(), (slots[live] % page).long()
    touched = torch.zeros((bt.n_pages, page), dtype=torch.bool)
    touched[pg, row] = True
    out_dtype = DTYPES[dtype]
    ko, vo = (torch.full((bt.n, nkv, d), 55.0, dtype=out_dtype, device="cuda") for _ in range(2))
    spd.kv_read(dev["k_pages"], dev["v_pages"], dev["cu"], dev["lens"], dev["table"], out=(ko, vo), **kv)
    assert int(dev["err"].item()) == 0
    for name, src, o in (("k", fused[:, nkv:2 * nkv], ko.cpu()), ("v", fused[:, 2 * nkv:], vo.cpu())):
        codes, p = dev[name + "_pages"].cpu(), dev[name + "_scales"].cpu()
        want_c, want_p = quantise4(src[live].float())
        got_c, got_p = codes[pg, :, row], p[pg, :, row]
        if dtype == "bf16":  # x - m is exact often enough that the definition's codes come out bit by bit
            assert same_bits(got_p, want_p) and torch.equal(got_c, want_c)
        else:  # float32 rows: (x - m), (max - m) / 15 and their rounding to bfloat16 may differ by float32's rounding at a tie
            assert torch.equal(got_p[..., 1], want_p[..., 1])
            assert ((got_p[..., 0].double() - want_p[..., 0].double()).abs() <= 2.0 ** -7 * want_p[..., 0].double()).all()
        # what reading gives is off by half a step (m <= x; 15 s may fall 2^-8 of 15 s short of the largest)
        step = got_p[..., 0].double().repeat_interleave(d // 2, -1)
        m = got_p[..., 1].double().abs().repeat_interleave(d // 2, -1)
        val = values4(got_c, got_p)
        assert ((val - src[live].double()).abs() <= 0.5 * step * (1 + 2.0 ** -20) + 2.0 ** -22 * (m + 15 * step)).all()
        got = o[live]
        assert torch.equal(got, val.float().to(out_dtype))
        assert (o[~live] == 55.0).all()
        # every other slot keeps its bits
        for key, now in ((name + "_pages", codes), (name + "_scales", p)):
            a, b_ = now.view(torch.uint8).view(bt.n_pages, nkv, page, -1), before[key].cpu().view(torch.uint8).view(bt.n_pages, nkv, page, -1)
            assert (a == b_).all(-1).all(1)[~touched].all()


def test_quantise_special_rows():
    """Ties, largest and smallest floats, far offsets, NaN and infinity: the row concerned only."""
    d = 64
    rows = torch.zeros((12, 1, d))
    rows[0, 0, 3] = 3.0e38
    rows[1, 0, :] = 1e-38
    rows[2, 0, 5] = 1e-45
    rows[3, 0, 0] = math.nan
    rows[4, 0, 40] = -math.inf
    rows[5, 0, :] = torch.linspace(-7.5, 7.5, d)
    rows[6, 0, :32] = 1000.0 + torch.linspace(-1, 1, 32)     # a smallest value that bfloat16 rounds by more than a step
    rows[7, 0, :] = torch.arange(d) % 31 * 0.5               # (x - m) / s = 0.5, 1.5, ...: ties to even
    rows[8, 0, 0], rows[8, 0, 1] = 3.0e38, -3.0e38           # a spread that is no float32
    rows[9, 0, :] = -2.0 ** torch.linspace(-30, 5, d)
    rows[10, 0, :] = -3.4028e38                              # rounds down to minus infinity
    rows[11, 0, :32] = 2.0 ** -70 * torch.arange(32)         # below the smallest scale
    kp, vp, ks, vs = pages4(1, 1, 16, d)
    i = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    err, cu, lens, table = i(0), i(0, 12), i(0), i(0).view(1, 1)
    kv = dict(err=err, k_scales=ks, v_scales=vs)
    spd.kv_write(rows.cuda(), rows.cuda(), kp, vp, cu, lens, table, **kv)
    k, v = spd.kv_read(kp, vp, cu, lens, table, n_tokens=12, dtype=torch.float32, **kv)
    assert torch.equal(k.nan_to_num(1.5), v.nan_to_num(1.5)) and int(err.item()) == 0
    k = k.cpu()
    for r in (3, 4, 8, 10):
        assert torch.isnan(k[r]).all() and (kp[0, 0, r] == 0).all() and torch.isnan(ks[0, 0, r].float()).all()
    for r in (0, 1, 2, 5, 6, 7, 9, 11):
        assert torch.equal(kp[0, 0, r].cpu(), quantise4(rows[r, 0])[0]), r
        assert torch.equal(ks[0, 0, r].cpu(), quantise4(rows[r, 0])[1]), r
        half = rows[r, 0].double().view(2, -1)
        low = half.amin(-1, keepdim=True)
        step = torch.maximum((half.amax(-1, keepdim=True) - low + 2.0 ** -7 * low.abs()) / 15 * (1 + 2.0 ** -8), torch.tensor(MIN_SCALE, dtype=torch.float64))
        assert ((k[r, 0].double().view(2, -1) - half).abs() <= 0.5 * step + 2.0 ** -22 * half.abs().amax()).all(), r
    assert torch.equal(kp[0, 0, 7, :4].cpu() & 15, torch.tensor([0, 0, 1, 2], dtype=torch.uint8))  # 0, 0.5, 1, 1.5
    assert (kp[0, 0, 12:] == 255).all()


def test_write_and_read_flag_what_does_not_fit():
    kp, vp, ks, vs = pages4(3, 2, 16, 64)
    i = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    x = torch.ones((4, 2, 64), dtype=torch.bfloat16, device="cuda")
    err = i(0)
    kv = dict(err=err, k_scales=ks, v_scales=vs)
    for table, lens, bit in ((i(3, 3).view(1, 2), i(0), 1), (i(-1, 0).view(1, 2), i(0), 1), (i(0, 1).view(1, 2), i(-4), 2), (i(0, 1).view(1, 2), i(32), 2)):
        err.zero_()
        spd.kv_write(x, x, kp, vp, i(0, 4), lens, table, **kv)
        assert int(err.item()) == bit
        err.zero_()
        k, v = (torch.full((4, 2, 64), 5.0, device="cuda") for _ in "kv")
        spd.kv_read(kp, vp, i(0, 4), lens, table, out=(k, v), **kv)
        assert int(err.item()) == bit and (k == 5).all() and (v == 5).all()
    err.zero_()
    spd.kv_write_slots(x, x, kp, vp, i(48, -1, 2 ** 31 - 1, -2 ** 31), **kv)
    assert int(err.item()) == 1
    assert (kp == 255).all() and (vp == 255).all() and torch.isnan(ks.float()).all() and torch.isnan(vs.float()).all()
    err.zero_()
    spd.kv_write_slots(x, x, kp, vp, i(-1, 47, -1, 0), **kv)
    assert int(err.item()) == 0
    assert (kp[2, :, 15] == 0).all() and (kp[0, :, 0] == 0).all() and int((kp != 255).sum()) == 2 * 2 * 32


@pytest.mark.parametrize("fmt", ["f32", "bf16", "e4m3", "int8"])
def test_slots_serve_every_format(fmt):
    """The same bits as by the block table."""
    bt = Batch4(dtype="bf16", nq=4, nkv=4, d=64, page=8, lens=[3, 11], new=[14, 2])
    slots = torch.tensor([bt.row_of(b, bt.lens[b] + i)[0] * 8 + bt.row_of(b, bt.lens[b] + i)[1] for b in range(2) for i in range(bt.new[b])], dtype=torch.int32)
    x = torch.randn((16, 8, 64), generator=torch.Generator().manual_seed(5)).to(torch.bfloat16).cuda()
    d = bt.device()
    got = []
    for by in "ts":
        k, v = (torch.zeros((bt.n_pages, 4, 8, 64), device="cuda").to(DTYPES[fmt]) for _ in "kv")
        s = [torch.zeros((bt.n_pages, 4, 8), device="cuda") for _ in "kv"] if fmt in ("e4m3", "int8") else [None, None]
        kv = dict(err=d["err"], k_scales=s[0], v_scales=s[1])
        if by == "t":
            spd.kv_write(x[:, :4], x[:, 4:], k, v, d["cu"], d["lens"], d["table"], **kv)
        else:
            spd.kv_write_slots(x[:, :4], x[:, 4:], k, v, slots.cuda(), **kv)
        got.append([k, v] + [t for t in s if t is not None])
    assert int(d["err"]) == 0 and all(same_bits(a, b) for a, b in zip(*got))
    assert got[0][0].float().abs().sum() > 0


# ---- attention ---------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("batch", range(len(BATCHES)))
@pytest.mark.parametrize("d", [128, 64])
def test_attention(dtype, batch, d):
    lens, new = BATCHES[batch]
    nq, nkv = HEADS[(batch + (d == 64)) % len(HEADS)]
    run_and_check(Batch4(dtype=dtype, nq=nq, nkv=nkv, d=d, page=16, lens=lens, new=new, lead=1, behind=2, seed=batch, offset=0.5))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("heads", HEADS)
def test_attention_head_layouts(dtype, heads):
    run_and_check(Batch4(dtype=dtype, nq=heads[0], nkv=heads[1], d=64, page=16, lens=[37, 90], new=[9, 30], seed=3))
    run_and_check(Batch4(dtype=dtype, nq=heads[0], nkv=heads[1], d=128, page=16, lens=[37, 90], new=[1, 1], seed=3))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("page", [1, 8, 24, 32, 64, 256])
def test_attention_page_sizes(dtype, page):
    run_and_check(Batch4(dtype=dtype, nq=8, nkv=2, d=128, page=page, lens=[70, 0, 129], new=[1, 40, 33], seed=page))
    for d in (64, 128):
        run_and_check(Batch4(dtype=dtype, nq=8, nkv=2, d=d, page=page, lens=[70, 255], new=[1, 1], seed=page))
        run_and_check(Batch4(dtype=dtype, nq=8, nkv=2, d=d, page=page, lens=[70, 255], new=[3, 4], seed=page))


@pytest.mark.parametrize("dtype", TYPES)
def test_attention_head_dim_32(dtype):
    run_and_check(Batch4(dtype=dtype, nq=4, nkv=2, d=32, page=16, lens=[70, 0], new=[1, 40], window=20, sinks=2, seed=2))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("window", WINDOWS)
def test_attention_window_and_sinks(dtype, window):
    for d, lens, new in ((128, [300, 0, 64, 1], [1, 1, 1, 1]), (128, [400, 0, 131], [37, 150, 1]), (64, [700], [260])):
        run_and_check(Batch4(dtype=dtype, nq=8, nkv=4, d=d, page=16, lens=lens, new=new, window=window[0], sinks=window[1], seed=5))


@pytest.mark.parametrize("dtype", TYPES)
def test_attention_long_context_single_tokens(dtype):
    run_and_check(Batch4(dtype=dtype, nq=8, nkv=1, d=128, page=16, lens=[5000, 3, 2049], new=[1, 1, 1], seed=6))
    run_and_check(Batch4(dtype=dtype, nq=4, nkv=1, d=128, page=16, lens=[4000, 90], new=[5, 20], window=1500, sinks=4, seed=7))


@pytest.mark.parametrize("dtype", TYPES)
def test_attention_sharp_softmax(dtype):
    """Scores of very unequal size: the running maximum moves late and far."""
    for new in (1, 3, 140):
        run_and_check(Batch4(dtype=dtype, nq=4, nkv=2, d=64, page=16, lens=[400], new=[new], seed=8, spread=4.0))


def stretch(kind):
    """Rows of V (and K) of very unequal size, far offsets, constant rows, halves of unequal size."""
    def rows(name, x):
        n = x.shape[0] * x.shape[2]
        i = torch.arange(n).view(x.shape[0], 1, x.shape[2], 1)
        if kind == "sizes" and name == "v":
            return x * 2.0 ** ((i % 7 - 3) * 5).double()       # 2^-15 .. 2^15
        if kind == "offset":
            return x + (30.0 if name == "v" else 4.0)
        if kind == "constant":
            return torch.where(i % 3 == 0, x[..., :1].expand_as(x), x)
        if kind == "halves" and name == "v":
            return x * torch.cat([torch.full((x.shape[-1] // 2,), 2.0 ** -9), torch.ones(x.shape[-1] // 2)]).double()
        if kind == "tiny" and name == "v":
            return x * 2.0 ** -40
        if kind == "large" and name == "v":
            return x * 2.0 ** 25
        return x
    return rows


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["sizes", "offset", "constant", "halves", "tiny", "large"])
@pytest.mark.parametrize("new", [1, 4, 150])
def test_attention_over_rows_of_unequal_size(dtype, kind, new):
    for d in (64, 128):
        run_and_check(Batch4(dtype=dtype, nq=4, nkv=2, d=d, page=16, lens=[300, 17], new=[new, 1], seed=18, rows=stretch(kind)))


def test_attention_strided_and_scaled():
    bt = Batch4(dtype="bf16", nq=8, nkv=2, d=64, page=16, lens=[20, 3], new=[1, 70], seed=9)
    dev = bt.device()
    wide = torch.zeros((bt.n, 12, 64), dtype=torch.bfloat16, device="cuda")
    wide[:, :8] = dev["q"]
    out_wide = torch.full((bt.n, 11, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    spd.paged_attention(wide[:, :8], dev["k_pages"], dev["v_pages"], dev["cu"], dev["lens"], dev["table"], max_new=bt.max_new() + 50,
                        max_context=bt.width * 16, err=dev["err"], out=out_wide[:, 2:10], scale=0.03, k_scales=dev["k_scales"], v_scales=dev["v_scales"])
    assert int(dev["err"].item()) == 0
    check_attention(bt, out_wide[:, 2:10], scale=0.03)
    assert (out_wide[:, :2] == 3).all() and (out_wide[:, 10:] == 3).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("new", [1, 6, 150])
@pytest.mark.parametrize("what", ["k_scales", "v_scales"])
@pytest.mark.parametrize("place", range(4))
def test_a_row_that_is_not_finite_is_nan_for_those_who_see_it(dtype, new, what, place):
    """NaN or an infinity in any one parameter of the last cached row, whose other parameters are anything: the queries before it are as if it
    were not there, the one that sees it (of that KV head) is NaN everywhere."""
    for bad in (math.nan, math.inf, -math.inf):
        bt = Batch4(dtype=dtype, nq=8, nkv=4, d=128, page=16, lens=[90], new=[new], seed=11)
        dev = bt.device()
        p, s = bt.row_of(0, 90 + new - 1)
        dev[what][p, 2, s, place // 2, place % 2] = bad
        out, err = attend(bt, dev)
        assert err == 0
        last = bt.cu[-1] - 1
        ref, tol = bt.reference()
        got = out.double().cpu()
        assert ((got - ref).abs()[:last] <= tol[:last]).all()
        assert torch.isnan(got[last, 4:6]).all()
        rest = [0, 1, 2, 3, 6, 7]
        assert ((got - ref).abs()[last, rest] <= tol[last, rest]).all()
        kv = dict(err=dev["err"], k_scales=dev["k_scales"], v_scales=dev["v_scales"])
        k, v = spd.kv_read(dev["k_pages"], dev["v_pages"], torch.tensor([0, 1], dtype=torch.int32, device="cuda"),
                           torch.tensor([90 + new - 1], dtype=torch.int32, device="cuda"), dev["table"], n_tokens=1, **kv)
        hit, other = (k, v) if what == "k_scales" else (v, k)
        assert torch.isnan(hit[0, 2]).all() and torch.isfinite(hit[0, [0, 1, 3]]).all() and torch.isfinite(other).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("new", [1, 20, 200])
def test_bad_batches_are_flagged_and_skipped(dtype, new):
    bt = Batch4(dtype=dtype, nq=4, nkv=2, d=64, page=16, lens=[50, 60], new=[new, new], seed=13)
    for what in ("context", "negative", "rows"):
        dev = bt.device()
        kw = {}
        if what == "context":
            kw["max_context"] = 50 + new
        elif what == "negative":
            dev["lens"][1] = -1
        else:
            dev["cu"][2] = bt.n + 1
        out, err = attend(bt, dev, **kw)
        assert err == 2, what
        assert (out[bt.cu[1]:] == 77).all()
        ref, tol = bt.reference()
        assert ((out.double().cpu() - ref).abs() <= tol)[:bt.cu[1]].all()
    for entry in (-1, bt.n_pages):
        dev = bt.device()
        dev["table"][0, 1] = entry
        out, err = attend(bt, dev)
        assert err == 1
        ref, tol = bt.reference()
        assert ((out.double().cpu() - ref).abs() <= tol)[bt.cu[1]:].all()


@pytest.mark.parametrize("dtype", TYPES)
def test_attention_is_deterministic_and_replays(dtype):
    for lens, new in (([700, 30, 1], [1, 1, 1]), ([300, 20], [30, 200])):
        bt = Batch4(dtype=dtype, nq=8, nkv=2, d=128, page=16, lens=lens, new=new, seed=14)
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


@pytest.mark.parametrize("B", [0, 3])
def test_calls_without_sequences_or_tokens(B):
    bt = Batch4(dtype="bf16", nq=4, nkv=2, d=64, page=16, lens=[20], new=[3])
    d = bt.device()
    i = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    kw = dict(err=d["err"], k_scales=d["k_scales"], v_scales=d["v_scales"])
    before = d["k_pages"].clone()
    where = i(B + 1), i(B), i(B, 4)
    rows = torch.full((5, 4, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    out = rows.clone()
    spd.paged_attention(rows, d["k_pages"], d["v_pages"], *where, max_new=1, max_context=10, out=out, **kw)
    spd.kv_write(rows[:, :2], rows[:, 2:], d["k_pages"], d["v_pages"], *where, **kw)
    spd.kv_write_slots(rows[:0, :2], rows[:0, 2:], d["k_pages"], d["v_pages"], i(0), **kw)
    k, v = spd.kv_read(d["k_pages"], d["v_pages"], *where, n_tokens=0, **kw)
    assert k.shape == v.shape == (0, 2, 64) and torch.equal(out, rows) and torch.equal(before, d["k_pages"]) and int(d["err"]) == 0
