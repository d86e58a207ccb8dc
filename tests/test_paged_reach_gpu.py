"""The paged-cache operators at the far ends of what their arguments allow: caches beyond 2^32 bytes and elements, shared prefixes,
an extension captured into the caller's graph."""
import pytest
import torch

import paper_2502_20727_b200 as spd
import spd_inputs as si
from paged_util import Batch, check_attention
from parity_util import Pair

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("types", [("bf16", "bf16"), ("bf16", "e4m3"), ("bf16", "int8"), ("f32", "f32")])
@pytest.mark.parametrize("page", [16, 24])
def test_pages_beyond_32_bit_offsets(types, page):
    """The batch's pages are the last ones of a cache of more than 2^32 elements (K and V share it, at different pages)."""
    bts = [Batch(dtype=types[0], fmt=types[1], nq=4, nkv=2, d=128, page=page, lens=[70, 9], new=new, seed=3) for new in ([1, 1], [12, 3], [60, 1])]
    per_page = 2 * page * 128
    n_big = (2 ** 32) // per_page + 200
    big = {}
    for bt in bts:
        d = bt.device()
        if not big:
            big = {n: torch.empty((n_big, 2, page, 128), dtype=d["k_pages"].dtype, device="cuda") for n in ("k_pages",)}
            big["v_pages"] = big["k_pages"]
            if d["k_scales"] is not None:
                big["k_scales"] = torch.empty((n_big, 2, page), device="cuda")
                big["v_scales"] = big["k_scales"]
        # K pages at the end; V pages have to be the same page numbers of another tensor: a view that starts 100 pages earlier
        n = bt.n_pages
        views = {}
        for key, t in big.items():
            v = t[100:] if key[0] == "k" else t[:n_big - 100]
            v[-n:].view(torch.uint8).copy_(d[key].view(torch.uint8)) if key.endswith("pages") else v[-n:].copy_(d[key])
            views[key] = v
        table = torch.where((d["table"] >= 0) & (d["table"] < n), d["table"] + (n_big - 100 - n), d["table"])
        assert n <= 100
        out = torch.full((bt.n, 4, 128), 77.0, dtype=bt.dtype, device="cuda")
        err = torch.zeros(1, dtype=torch.int32, device="cuda")
        kw = dict(k_scales=views.get("k_scales"), v_scales=views.get("v_scales"), err=err)
        spd.paged_attention(d["q"], views["k_pages"], views["v_pages"], d["cu"], d["lens"], table, max_new=bt.max_new(), max_context=bt.max_context(), out=out, **kw)
        assert int(err) == 0
        check_attention(bt, out)
        # rows of sequence 0 read back and appended behind themselves
        cu = torch.tensor([0, 50], dtype=torch.int32, device="cuda")
        zero = torch.zeros(1, dtype=torch.int32, device="cuda")
        k, v = spd.kv_read(views["k_pages"], views["v_pages"], cu, zero, table[:1], n_tokens=50, dtype=bt.dtype, **kw)
        k2, v2 = spd.kv_read(d["k_pages"], d["v_pages"], cu, zero, d["table"][:1], n_tokens=50, dtype=bt.dtype, err=err, k_scales=d["k_scales"],
                             v_scales=d["v_scales"])
        assert torch.equal(k, k2) and torch.equal(v, v2)
        spd.kv_write(k, v, views["k_pages"], views["v_pages"], cu, zero, table[:1], **kw)
        k3, v3 = spd.kv_read(views["k_pages"], views["v_pages"], cu, zero, table[:1], n_tokens=50, dtype=bt.dtype, **kw)
        step = 2.0 ** -6 if types[1] == "int8" else 0.0  # int8 codes of code values: the largest is 127 again up to a rounding
        assert int(err) == 0 and (k3.float() - k.float()).abs().max() <= step * k.float().abs().max()
    del big, views
    torch.cuda.empty_cache()


@pytest.mark.parametrize("fmt", ["bf16", "int8"])
@pytest.mark.parametrize("new", [1, 40])
def test_sequences_that_share_pages(fmt, new):
    """The same pages under two sequences of a batch (a shared prefix): both see what one alone sees."""
    bt = Batch(dtype="bf16", fmt=fmt, nq=8, nkv=2, d=128, page=16, lens=[100], new=[new], seed=5)
    d = bt.device()
    kw = dict(max_new=new, max_context=100 + new, err=d["err"], k_scales=d["k_scales"], v_scales=d["v_scales"])
    one = spd.paged_attention(d["q"], d["k_pages"], d["v_pages"], d["cu"], d["lens"], d["table"], **kw)
    two = spd.paged_attention(torch.cat([d["q"], d["q"]]), d["k_pages"], d["v_pages"], torch.tensor([0, new, 2 * new], dtype=torch.int32, device="cuda"),
                              d["lens"].repeat(2), d["table"].repeat(2, 1), **kw)
    check_attention(bt, one)
    check_attention(bt, two[:new])
    assert torch.equal(two[:new], two[new:]) and int(d["err"]) == 0


def test_extend_captured_and_replayed():
    """spd_extend inside the caller's graph: replayed at another length, with other tokens, it is the direct call."""
    w = si.Workload("small", "bf16", 2, 512, 8, 4, 64, 1376, 4, (0, 1), 2, 16, 4)
    p = Pair(w, B=2, max_len=128)
    st = p.stack
    for S in (3, 50):
        p.fill_cache([40, 17])
        x = [si.make_hidden(w, (2, S, 512), "cpu", 0, i).to(p.device) for i in range(2)]
        lens = [torch.tensor(v, dtype=torch.int32, device=p.device) for v in ([40, 17], [11, 40])]
        direct = [st.extend(x[i], lens[i], p.block_table, 100).clone() for i in range(2)]
        xs, ls, out = x[0].clone(), lens[0].clone(), torch.empty_like(x[0])
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=torch.cuda.current_stream()):
            st.extend(xs, ls, p.block_table, 100, out)
        for i in (0, 1, 0):
            p.fill_cache([40, 17])
            if i:
                st.extend(x[0], lens[0], p.block_table, 100)  # the cache as the direct calls left it
            xs.copy_(x[i])
            ls.copy_(lens[i])
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, direct[i]), (S, i)
        del g
    assert st.device_error() == 0
    st.close()


def test_timeline_and_profile_of_extensions_and_windows():
    """The launch timeline knows these attention launches too: one per layer, with time of their own within the call's span."""
    w = si.Workload("wide", "bf16", 3, 1024, 16, 2, 128, 2048, 2, (0, 1, 0), 2, 16, 4)
    p = Pair(w, B=2, max_len=1024)
    st = p.stack
    p.fill_cache([900, 700])
    seq = torch.tensor([900, 700], dtype=torch.int32, device=p.device)
    for S, window in ((4, 0), (60, 0), (60, 100), (1, 300)):
        st.set_window(window, 4)
        x = si.make_hidden(w, (2, S, w.hidden), "cpu", 0, S).to(p.device)
        run = (lambda: st.extend(x, seq, p.block_table, 1000)) if S > 1 else (lambda: st.decode_step(x[:, 0].contiguous(), seq, p.block_table, 1000))
        plain = run().clone()
        st.timeline_begin()
        for _ in range(3):
            out = run()
        launches, span, calls = st.timeline_read()
        st.timeline_end()
        own = [t for kind, t in launches if kind == "attention"]
        assert calls == 3 and len(own) == 3 and all(t > 0 for t in own) and sum(t for _, t in launches) <= span
        assert torch.equal(out, plain)
        st.profile_begin()
        run()
        prof = st.profile_end()
        assert prof["attention"]["launches"] >= 3 and prof["attention"]["ms"] > 0
    assert st.device_error() == 0
    st.close()
