"""Extending cached sequences and attending through a sliding window: the stack against the CPU oracle and against a float64
reference with a window.  Bound: max|gpu-ref| / max|ref| as for the other stack calls (1e-4 float32, 2e-2 bfloat16 per block)."""
import numpy as np
import pytest
import torch

import paper_2502_20727_b200 as spd
import spd_inputs as si
from parity_util import Pair, rel_err, stack_tol, to_np
from window_ref import stack_forward

pytestmark = pytest.mark.gpu

FP32 = si.Workload("small", "fp32", 2, 256, 4, 2, 64, 688, 2, (0, 1), 3, 16, 4)
BF16 = si.Workload("small", "bf16", 2, 512, 8, 4, 64, 1376, 4, (0, 1), 3, 16, 4)
WIDE = si.Workload("wide", "bf16", 1, 1024, 16, 2, 128, 2048, 2, (0,), 2, 16, 4)
BIAS = si.Workload("bias", "bf16", 1, 512, 4, 4, 128, 1024, 2, (0,), 2, 16, 4, block="opt")


def extend(p, S, stream, lens=None):
    """S new tokens per sequence at p.pos on both sides."""
    x = si.make_hidden(p.w, (p.B, S, p.w.hidden), "cpu", 3, stream)
    ref, _ = p._oracle(to_np(x))
    seq = torch.from_numpy(p.pos.copy()).to(p.device)
    got = p.stack.extend(x.to(p.device), seq, p.block_table, int(p.pos.max()) + S)
    torch.cuda.synchronize()
    p.pos = p.pos + S
    return to_np(got), ref


CASES = [(FP32, 4096, (1, 5, 40)), (FP32, 16, (3, 40)), (BF16, 4096, (1, 2, 17, 50)), (BF16, 16, (21, 5)), (WIDE, 4096, (1, 4, 37)),
         (WIDE.with_(mask=(1,), kv_block=24), 64, (2, 130)), (BIAS, 4096, (1, 6, 33))]


@pytest.mark.parametrize("w,chunk,steps", CASES, ids=lambda v: str(getattr(v, "name", v)))
def test_extend_matches_oracle(w, chunk, steps):
    """Ragged cached lengths (one of them zero), then extensions of different widths, then a decode step."""
    for B in (w.batch, 64):  # many sequences allowed: few tokens take the decode step's projections
        lens = [29, 0, 47][:w.batch]
        p = Pair(w, B=w.batch, max_len=64 + sum(steps), max_prefill_tokens=chunk)
        if B == 64:
            p.stack.close()
            p.stack = spd.stack_from_workload(w, p.layers_gpu, sync_mask=p.mask, max_batch=64, max_seq_len=p.max_len, n_pages=p.n_pages,
                                              max_prefill_tokens=chunk, device=p.device)
        p.fill_cache(lens)
        tol = stack_tol(w.dtype, w.n_layers)
        for i, S in enumerate(steps):
            got, ref = extend(p, S, i)
            assert rel_err(got, ref) <= tol, (B, S)
        got, ref = p.decode(9)
        assert rel_err(got, ref) <= tol
        for b in range(w.batch):
            n = int(p.pos[b])
            for which in ("k", "v"):
                assert rel_err(p.gpu_cache(w.n_layers - 1, which, b, n), getattr(p.cache, which)[w.n_layers - 1, b, :n]) <= tol
        assert p.stack.device_error() == 0
        p.stack.close()


WINDOWS = [(FP32, 4096, 8, 0), (FP32, 16, 20, 3), (BF16, 4096, 1, 0), (BF16, 16, 33, 4), (WIDE, 4096, 48, 4), (WIDE.with_(mask=(1,), kv_block=24), 64, 100, 30),
           (BF16, 4096, 500, 2)]


@pytest.mark.parametrize("w,chunk,window,sinks", WINDOWS, ids=lambda v: str(getattr(v, "name", v)))
def test_window_in_every_call(w, chunk, window, sinks):
    """Prefill, extension and decode steps (captured and replayed) with a window; pages behind it are given back before decoding."""
    S0, S1 = 70, 9
    p = Pair(w, B=w.batch, max_len=S0 + S1 + 4, max_prefill_tokens=chunk)
    p.stack.set_window(window, sinks)
    kc = np.zeros((w.n_layers, p.B, p.max_len, w.n_kv_heads, w.head_dim))
    vc = np.zeros_like(kc)
    tol = stack_tol(w.dtype, w.n_layers)

    def both(call, S, stream):
        x = si.make_hidden(w, (p.B, S, w.hidden), "cpu", 5, stream)
        ref = stack_forward(w, p.mask, p.layers_np, to_np(x), p.pos, kc, vc, window, sinks)
        got = call(x.to(p.device), torch.from_numpy(p.pos.copy()).to(p.device))
        torch.cuda.synchronize()
        assert rel_err(to_np(got).reshape(ref.shape), ref) <= tol, (stream, rel_err(to_np(got).reshape(ref.shape), ref))
        p.pos = p.pos + S

    both(lambda x, seq: p.stack.prefill(x, p.block_table), S0, 0)
    both(lambda x, seq: p.stack.extend(x, seq, p.block_table, S0 + S1), S1, 1)
    first = S0 + S1 + 1 - window
    for j in range(p.block_table.shape[1]):
        if j * w.kv_block >= sinks and (j + 1) * w.kv_block <= first:
            p.block_table[:, j] = 1 << 20
    xb = torch.empty((p.B, w.hidden), dtype=w.torch_dtype, device=p.device)
    sb, out = torch.empty(p.B, dtype=torch.int32, device=p.device), torch.empty((p.B, w.hidden), dtype=w.torch_dtype, device=p.device)

    def step(x, seq):
        xb.copy_(x[:, 0])
        sb.copy_(seq)
        return p.stack.decode_step(xb, sb, p.block_table, int(p.pos.max()) + 1, out)

    for t in range(4):
        both(step, 1, 2 + t)
    assert p.stack.device_error() == 0
    p.stack.close()


def test_window_in_rank_mode():
    """The rank mode's prompt and decode calls see the same window."""
    S, window, sinks = 40, 12, 2
    p = Pair(WIDE, B=2, max_len=48, max_prefill_tokens=256)
    p.stack.tp_attach_local()
    p.stack.set_window(window, sinks)
    kc = np.zeros((1, 2, 48, WIDE.n_kv_heads, WIDE.head_dim))
    vc = np.zeros_like(kc)
    x = si.make_hidden(WIDE, (2, S, WIDE.hidden), "cpu", 0, 0)
    ref = stack_forward(WIDE, p.mask, p.layers_np, to_np(x), p.pos, kc, vc, window, sinks)
    got = to_np(p.stack.tp_prefill(x.to(p.device), p.block_table))
    assert max(rel_err(got[r].reshape(ref.shape), ref) for r in range(WIDE.T)) <= stack_tol("bf16", 1)
    for t in range(3):
        xd = si.make_hidden(WIDE, (2, WIDE.hidden), "cpu", 0, 1 + t)
        ref = stack_forward(WIDE, p.mask, p.layers_np, to_np(xd)[:, None], np.full(2, S + t), kc, vc, window, sinks)[:, 0]
        got = to_np(p.stack.tp_decode_step(xd.to(p.device), torch.full((2,), S + t, dtype=torch.int32, device=p.device), p.block_table, S + t + 1))
        assert max(rel_err(got[r], ref) for r in range(WIDE.T)) <= stack_tol("bf16", 1)
    assert p.stack.device_error() == 0
    p.stack.close()


def test_window_off_again_is_the_old_result():
    """Without a window every call runs as it did before one was set: the same bits."""
    p = Pair(BF16, B=3, max_len=64)
    x = si.make_hidden(BF16, (3, 40, 512), "cpu", 0, 0).to(p.device)
    xd = si.make_hidden(BF16, (3, 512), "cpu", 0, 1).to(p.device)
    seq = torch.full((3,), 40, dtype=torch.int32, device=p.device)
    a = p.stack.prefill(x, p.block_table).clone()
    b = p.stack.decode_step(xd, seq, p.block_table, 41).clone()
    p.stack.set_window(7, 1)
    c = p.stack.prefill(x, p.block_table).clone()
    d = p.stack.decode_step(xd, seq, p.block_table, 41).clone()
    p.stack.set_window(0)
    e = p.stack.prefill(x, p.block_table).clone()
    f = p.stack.decode_step(xd, seq, p.block_table, 41).clone()
    torch.cuda.synchronize()
    assert torch.equal(a, e) and torch.equal(b, f) and not torch.equal(a, c) and not torch.equal(b, d)
    p.stack.close()


def test_prefix_moved_to_another_sequence():
    """Cached rows read out of one sequence's pages and written into another's continue to the same bits."""
    for w in (FP32, BF16, WIDE):
        p = Pair(w, B=2, max_len=80)
        st, n = p.stack, 37
        x = si.make_hidden(w, (2, n, w.hidden), "cpu", 1, 0).to(p.device)
        st.prefill(x, p.block_table)
        err = torch.zeros(1, dtype=torch.int32, device=p.device)
        cu = torch.tensor([0, n], dtype=torch.int32, device=p.device)
        at = torch.zeros(1, dtype=torch.int32, device=p.device)
        for l in range(w.n_layers):
            k, v = st.read_cache(l, cu, at, p.block_table[:1], n_tokens=n, err=err)
            st.write_cache(l, k, v, cu, at, p.block_table[1:2], err=err)
        y = si.make_hidden(w, (1, 6, w.hidden), "cpu", 1, 1).to(p.device).expand(2, 6, w.hidden).contiguous()
        out = st.extend(y, torch.full((2,), n, dtype=torch.int32, device=p.device), p.block_table, n + 6)
        torch.cuda.synchronize()
        assert torch.equal(out[0], out[1]) and int(err) == 0 and st.device_error() == 0
        st.close()


def test_extend_refusals_and_bounds():
    p = Pair(BF16, B=2, max_len=64, max_prefill_tokens=64)
    st, dev = p.stack, p.device
    lib, ctx, bt = st.lib, st._ctx, p.block_table
    x = si.make_hidden(BF16, (2, 4, 512), "cpu", 0, 0).to(dev)
    out = torch.full_like(x, 3.0)
    seq = torch.tensor([5, 9], dtype=torch.int32, device=dev)
    good = [x.data_ptr(), 2, 4, seq.data_ptr(), bt.data_ptr(), bt.shape[1], 20, out.data_ptr()]

    def call(**kw):
        a = dict(zip(("x", "B", "S", "seq", "bt", "mp", "mc", "out"), good))
        a.update(kw)
        return lib.spd_extend(ctx, *a.values(), torch.cuda.current_stream().cuda_stream)

    for n in ("x", "seq", "bt", "out"):
        assert call(**{n: None}) == -2
    for kw, rc in ((dict(B=0), -1), (dict(B=3), -1), (dict(S=0), -1), (dict(mc=3), -1), (dict(out=x.data_ptr()), -1), (dict(mc=65), -4),
                   (dict(mp=1), -4)):
        assert call(**kw) == rc, kw
    assert lib.spd_set_window(ctx, -1, 0) == -1 and lib.spd_set_window(ctx, 4, -1) == -1
    torch.cuda.synchronize()
    assert bool((out == 3.0).all()) and st.device_error() == 0
    # one sequence beyond the bound: reported, the other one right
    assert call() == 0
    one = out.clone()
    assert st.device_error() == 0
    seq.copy_(torch.tensor([5, 30], dtype=torch.int32))
    assert call() == 0
    torch.cuda.synchronize()
    assert torch.equal(out[0], one[0]) and st.device_error() == 2
    with pytest.raises(ValueError):
        st.extend(x, seq[:1], bt, 20)
    st.close()
