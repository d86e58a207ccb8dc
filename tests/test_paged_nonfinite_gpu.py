"""Attention over a cache whose K rows give infinite scores, with finite V: what softmax makes of them, in every kernel."""
import math

import pytest
import torch

from paged_util import Batch
from test_paged_gpu import TYPES, attend

pytestmark = pytest.mark.gpu

HEAD, DIM = 1, 7  # the KV head whose K rows are poisoned, and the head dim


def batch(types, **kw):
    bt = Batch(dtype=types[0], fmt=types[1], seed=21, **{**dict(nq=4, nkv=2, d=64, page=16), **kw})
    bt.q = bt.q.abs() + 0.125  # the sign of a poisoned score is that of the infinity
    return bt


def poison(bt, dev, t, sign):
    """Every score of key t (sequence 0) becomes sign * inf.  8-bit: codes of +-1 under an infinite scale, so that every term of the
    score is the same infinity (a code of 0 would stand for 0 * inf)."""
    p, s = bt.row_of(0, t)
    k = dev["k_pages"][p, HEAD, s]
    if dev["k_scales"] is None:
        k[DIM] = sign * math.inf
    else:
        k.view(torch.uint8).fill_((0x38 if sign > 0 else 0xB8) if bt.fmt == "e4m3" else (1 if sign > 0 else 255))
        dev["k_scales"][p, HEAD, s] = math.inf


def reference(bt, gone):
    """Sequence 0 as if the keys `gone` of the poisoned head did not exist; the tolerance is Batch.reference's.  NaN where no key is left."""
    a, n, group = bt.lens[0], bt.new[0], bt.nq // bt.nkv
    idx = torch.tensor([bt.row_of(0, t) for t in range(a + n)])
    k, v = (bt.values[x][idx[:, 0], :, idx[:, 1]] for x in "kv")
    t, p = torch.arange(a + n), torch.arange(a, a + n)[:, None]
    see = t <= p
    if bt.window:
        see &= (t > p - bt.window) | (t < bt.sinks)
    out = torch.full((n, bt.nq, bt.d), math.nan, dtype=torch.float64)
    tol = torch.zeros_like(out)
    q = bt.q.double()
    for h in range(bt.nq):
        left = see.clone()
        if h // group == HEAD:
            left[:, list(gone)] = False
        kh, vh, scale = k[:, h // group], v[:, h // group], bt.d ** -0.5
        w = torch.softmax((q[:, h] @ kh.t() * scale).masked_fill(~left, -math.inf), -1)
        mag = (q[:, h].abs() @ kh.abs().t() * scale).masked_fill(~left, 0).amax(-1, keepdim=True)
        aw = w @ vh.abs()
        out[:, h] = w @ vh
        tol[:, h] = (2 * (bt.d + 8) * 2.0 ** -24 * mag + 2.0 ** -18 + 2 * (a + n) * 2.0 ** -24) * aw
        if bt.dtype == torch.bfloat16:
            tol[:, h] += 1.01 * 2.0 ** -8 * (aw + out[:, h].abs())
    return out, tol


def check(got, ref, tol):
    got, want = got.double().cpu(), ~torch.isnan(ref)
    assert torch.isnan(got[~want]).all(), "a row without a softmax has to be NaN"
    bad = ~((got - ref).abs()[want] <= tol[want])  # an only key whose value is 0 leaves no room at all
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} values off"


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("new,page", [(1, 16), (3, 16), (40, 16), (40, 24), (1, 24)])
@pytest.mark.parametrize("at", list(range(8)) + list(range(64, 72)))
def test_a_score_of_infinity_is_nan_wherever_the_key_lies(types, new, page, at):
    """Queries that see the key: inf - inf in every weight's sum.  The others, and the other KV head: nothing."""
    lens = 128 + at - (new + 1) // 2  # some of the new tokens come before key 128 + at, where there are any
    bt = batch(types, lens=[lens], new=[new], page=page)
    dev = bt.device()
    t = 128 + at if new > 1 else at
    poison(bt, dev, t, 1)
    out, err = attend(bt, dev)
    assert err == 0
    ref, tol = reference(bt, ())
    p = torch.arange(lens, lens + new)
    ref[p >= t, 2:] = math.nan
    check(out, ref, tol)


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("new", [2, 5, 100])
def test_scores_of_minus_infinity_have_no_weight(types, new):
    """Keys with such scores among others: as if they did not exist."""
    bt = batch(types, lens=[150], new=[new])
    dev = bt.device()
    gone = list(range(3, 150, 7)) + [150]
    for t in gone:
        poison(bt, dev, t, -1)
    out, err = attend(bt, dev)
    assert err == 0
    check(out, *reference(bt, gone))


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("new", [1, 4, 100])
def test_rows_whose_scores_are_all_minus_infinity_are_nan(types, new):
    """Softmax has no value there.  A window's queries that still see another key are as if those keys did not exist."""
    bt = batch(types, lens=[300], new=[new], window=50, sinks=0)
    dev = bt.device()
    gone = range(240, 300 + (new + 1) // 2)
    for t in gone:
        poison(bt, dev, t, -1)
    out, err = attend(bt, dev)
    assert err == 0
    ref, tol = reference(bt, gone)
    assert torch.isnan(ref[0, 2:]).all() and not torch.isnan(ref[:, :2]).any()
    check(out, ref, tol)


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("nq,lens,new", [(8, 5000, 1), (4, 3000, 12), (2, 900, 1)])
def test_key_ranges_of_minus_infinity(types, nq, lens, new):
    """One sequence whose keys are cut into ranges: a range without a finite score adds nothing, a row without one is NaN."""
    for gone in (range(0, lens // 2), range(0, lens + new)):
        bt = batch(types, lens=[lens], new=[new], nq=nq)
        dev = bt.device()
        for t in gone:
            poison(bt, dev, t, -1)
        out, err = attend(bt, dev)
        assert err == 0
        check(out, *reference(bt, gone))


@pytest.mark.parametrize("page", [16, 24])
@pytest.mark.parametrize("nq,nkv,lens,new", [(4, 2, 90, 45), (6, 2, 130, 43), (4, 1, 3000, 5), (2, 2, 0, 129), (8, 2, 200, 33)])
def test_infinite_values_in_tiles_that_rows_do_not_fill(page, nq, nkv, lens, new):
    """Row tiles with rows left over, whose warps' lanes differ in what they see of several infinities in V."""
    bt = Batch(dtype="bf16", fmt="bf16", nq=nq, nkv=nkv, d=128, page=page, lens=[lens], new=[new], seed=22)
    dev = bt.device()
    ref, tol = bt.reference()
    group, head = nq // nkv, nkv - 1
    for i, dim in ((0, 3), (1, 40), (new // 2, 100), (new - 1, 17)):  # the i-th new token's value, in one dim
        p, s = bt.row_of(0, lens + i)
        dev["v_pages"][p, head, s, dim] = math.inf
        ref[i:, head * group:, dim] = math.nan
    out, err = attend(bt, dev)
    assert err == 0
    got, hit = out.double().cpu(), torch.isnan(ref)
    assert (~torch.isfinite(got[hit])).all()
    assert ((got - ref).abs()[~hit] <= tol[~hit]).all()
