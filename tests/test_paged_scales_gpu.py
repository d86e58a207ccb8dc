"""Attention over 8-bit caches whose V scales differ wildly, and how exact the weights of int8 caches are."""
import pytest
import torch

from paged_util import Batch
from test_paged_gpu import attend

pytestmark = pytest.mark.gpu

SHAPES = [dict(nq=8, nkv=2, lens=[300, 0, 40], new=[1, 1, 1]),       # single tokens
          dict(nq=16, nkv=1, lens=[0, 1000], new=[1, 1]),
          dict(nq=8, nkv=1, lens=[130, 5], new=[70, 3]),             # more than 16 rows
          dict(nq=4, nkv=2, lens=[513], new=[200], window=100, sinks=5)]


def tolerance(bt):
    """bf16, e4m3: as for every bf16 call.  int8: a weight is two bf16s, the second off by 2^-8 of at most 2^-8 of it, so 2^-16; plus
    2^-17 for exponentials by a polynomial of relative error 2.6e-6 (weight and sum); the output's rounding 2^-8 of its value;
    float32 arithmetic as for float32 queries; second parts below 2^-126 vanish: 127 * 2^-126 per key."""
    ref, wide = bt.reference()
    if bt.fmt != "int8":
        return ref, wide
    kind, bt.dtype = bt.dtype, torch.float32
    _, narrow = bt.reference()
    bt.dtype = kind
    aw = (wide - narrow) / (1.01 * 2.0 ** -8) - ref.abs()  # sum of weight * |v|
    keys = max(a + n for a, n in zip(bt.lens, bt.new))
    return ref, narrow + 1.01 * 2.0 ** -8 * ref.abs() + (1.01 * 2.0 ** -16 + 2.0 ** -17) * aw + keys * 2.0 ** -119


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
@pytest.mark.parametrize("shift", [(0, 0), (-60, 60), (-90, -90), (90, 90), (-8, 8)])
@pytest.mark.parametrize("d", [64, 128])
def test_v_scales_of_any_size(fmt, shape, shift, d):
    kw = dict(SHAPES[shape])
    bt = Batch(dtype="bf16", fmt=fmt, d=d, page=16, seed=shape, **kw)
    g = torch.Generator().manual_seed(99)
    by = torch.exp2(torch.randint(shift[0], shift[1] + 1, bt.scales["v"].shape, generator=g).float())
    bt.scales["v"] = bt.scales["v"] * by
    bt.values["v"] = bt.values["v"] * by.double()[..., None]
    out, err = attend(bt)
    assert err == 0
    ref, tol = tolerance(bt)
    live = ~torch.isnan(ref[:, 0, 0])
    off = (out.double().cpu()[live] - ref[live]).abs() / tol[live]
    assert torch.isfinite(off).all() and off.max() <= 1, off.max()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("new", [1, 40, 200])
@pytest.mark.parametrize("scale", [3.3e38, 2.0 ** 120, -3.3e38, -1.0, float("inf"), -float("inf"), float("nan"), 0.0])
def test_unseen_rows_with_any_scale(fmt, new, scale):
    """Slots of nobody in the pages, and the new tokens' keys for the queries before them: any scale, the largest codes."""
    bt = Batch(dtype="bf16", fmt=fmt, nq=4, nkv=2, d=128, page=32, lens=[37], new=[new], window=50, sinks=2, seed=4)
    d = bt.device()
    for n in "kv":
        owned = ~torch.isnan(d[n + "_scales"])
        d[n + "_scales"] = torch.where(owned, d[n + "_scales"], torch.full_like(d[n + "_scales"], scale))
        codes = d[n + "_pages"].view(torch.uint8)
        codes[~owned] = 0x7E if fmt == "e4m3" else 0x7F
    out, err = attend(bt, d)
    assert err == 0
    ref, tol = tolerance(bt)
    live = ~torch.isnan(ref[:, 0, 0])
    off = (out.double().cpu()[live] - ref[live]).abs() / tol[live]
    assert torch.isfinite(off).all() and off.max() <= 1, off.max()


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("new", [1, 12, 150])
@pytest.mark.parametrize("name", ["k", "v"])
@pytest.mark.parametrize("behind", range(4))
def test_a_visible_row_of_nans_is_nan_where_it_is_seen(fmt, new, name, behind):
    """A cached row of NaNs (8-bit: scale NaN): queries that see it get NaNs, the others nothing."""
    bt = Batch(dtype="bf16", fmt=fmt, nq=4, nkv=1, d=64, page=16, lens=[140], new=[new], window=60, sinks=1, seed=6)
    t = 140 + (new // 2 + 2 * behind) % new  # some of the new tokens come before it
    page, slot = bt.row_of(0, t)
    if fmt == "bf16":
        bt.codes[name][page, :, slot] = float("nan")
    else:
        bt.scales[name][page, :, slot] = float("nan")
    bt.values[name][page, :, slot] = 0.0  # of no account to queries that do not see it
    out, _ = attend(bt)
    out = out.double().cpu()
    p = torch.arange(140, 140 + new)
    sees = (p >= t) & (t > p - 60)
    ref, tol = tolerance(bt)
    assert torch.isnan(out[sees]).all()
    off = (out[~sees] - ref[~sees]).abs() / tol[~sees]
    assert torch.isfinite(off).all() and (off <= 1).all()
