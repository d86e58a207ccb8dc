"""Calls of the paged-cache operators that the documentation allows: no sequences, no tokens, many query heads per KV head, windows
that never end, several threads at once."""
import threading

import pytest
import torch

import paper_2502_20727_b200 as spd
from paged_util import Batch, check_attention
from test_paged_gpu import TYPES, attend, run_and_check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("B", [0, 3])
def test_calls_without_sequences_or_tokens(fmt, B):
    """An empty batch, and sequences none of which has a token: nothing happens."""
    bt = Batch(dtype="bf16", fmt=fmt, nq=4, nkv=2, d=64, page=16, lens=[20], new=[3])
    d = bt.device()
    i = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    kw = dict(err=d["err"], k_scales=d["k_scales"], v_scales=d["v_scales"])
    before = {n: d[n + "_pages"].view(torch.uint8).clone() for n in "kv"}
    x = torch.empty((0, 2, 64), dtype=torch.bfloat16, device="cuda")
    where = i(B + 1), i(B), i(B, 4)
    spd.kv_write(x, x, d["k_pages"], d["v_pages"], *where, **kw)
    k, v = spd.kv_read(d["k_pages"], d["v_pages"], *where, n_tokens=0, **kw)
    assert k.shape == v.shape == (0, 2, 64)
    q = torch.empty((0, 4, 64), dtype=torch.bfloat16, device="cuda")
    assert spd.paged_attention(q, d["k_pages"], d["v_pages"], *where, max_new=1, max_context=10, **kw).shape == (0, 4, 64)
    # rows of nobody stay what they are
    rows = torch.full((5, 4, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    out = rows.clone()
    spd.paged_attention(rows, d["k_pages"], d["v_pages"], *where, max_new=1, max_context=10, out=out, **kw)
    spd.kv_write(rows[:, :2], rows[:, 2:], d["k_pages"], d["v_pages"], *where, **kw)
    ko, vo = rows[:, :2].clone(), rows[:, 2:].clone()
    spd.kv_read(d["k_pages"], d["v_pages"], *where, out=(ko, vo), **kw)
    assert torch.equal(out, rows) and torch.equal(ko, rows[:, :2]) and torch.equal(vo, rows[:, 2:]) and int(d["err"]) == 0
    assert all(torch.equal(before[n], d[n + "_pages"].view(torch.uint8)) for n in "kv")


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("nq,nkv", [(32, 1), (71, 1), (128, 1), (400, 2)])
def test_many_query_heads_per_kv_head(types, nq, nkv):
    """Groups of heads that fill part of a row tile, one, or several."""
    run_and_check(Batch(dtype=types[0], fmt=types[1], nq=nq, nkv=nkv, d=64, page=16, lens=[150, 0, 40], new=[1, 1, 1], seed=31))
    run_and_check(Batch(dtype=types[0], fmt=types[1], nq=nq, nkv=nkv, d=64, page=16, lens=[97], new=[4], window=50, sinks=3, seed=32))


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("new", [1, 5, 150])
def test_windows_and_sinks_up_to_the_largest_number(types, new):
    """As good as none."""
    top = 2 ** 31 - 1
    bt = Batch(dtype=types[0], fmt=types[1], nq=8, nkv=2, d=128, page=16, lens=[140, 0], new=[new, 1], seed=33)
    want = run_and_check(bt)
    for window, sinks in ((top, 0), (top, top), (1, top), (2 ** 30 + 1, 7)):
        bt.window, bt.sinks = window, sinks
        out, err = attend(bt)
        assert err == 0
        check_attention(bt, out)
        if window != 1:
            assert torch.equal(out, want)


def test_threads_that_call_at_once():
    """First calls of several variants from several threads, each on a stream of its own."""
    bts = [Batch(dtype=a, fmt=f, nq=8, nkv=2, d=d, page=page, lens=[200, 30], new=[new, 1], seed=34)
           for a, f in TYPES for d, page, new in ((128, 16, 1), (64, 24, 40))]
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
                                                  max_context=bt.max_context(), err=d["err"], k_scales=d["k_scales"], v_scales=d["v_scales"])
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
