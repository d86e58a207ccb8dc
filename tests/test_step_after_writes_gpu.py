"""A decode step right behind calls that write cached rows: its attention asks for pages of earlier tokens early, and has to find them
as those calls leave them.  Launched directly and from the caller's graph, in every form of the step."""
import pytest
import torch

import spd_inputs as si
from parity_util import Pair

pytestmark = pytest.mark.gpu

STACKS = [si.Workload("wide", "bf16", 1, 1024, 16, 2, 128, 2048, 2, (0,), 8, 16, 4),          # tensor-core decode attention
          si.Workload("narrow", "bf16", 1, 512, 8, 8, 64, 1376, 4, (1,), 8, 16, 4),            # the page ring
          si.Workload("small", "fp32", 1, 256, 4, 2, 64, 688, 2, (0,), 8, 16, 4),
          si.Workload("bias", "bf16", 1, 512, 4, 4, 128, 1024, 2, (0,), 8, 16, 4, block="opt"),
          si.Workload("norope", "fp32", 1, 256, 4, 2, 64, 688, 2, (0,), 8, 16, 4, rope_base=0.0)]


@pytest.mark.parametrize("w", STACKS, ids=lambda w: w.name)
@pytest.mark.parametrize("captured", [False, True])
def test_step_behind_an_append_sees_it(w, captured):
    B, L = 8, 1500
    p = Pair(w, B=B, max_len=L + 8)
    st, dev = p.stack, p.device
    st.set_graphs(False)
    kv_heads = w.n_kv_heads
    cu = torch.arange(0, (B + 1) * L, L, dtype=torch.int32, device=dev)
    zero, lens = (torch.full((B,), n, dtype=torch.int32, device=dev) for n in (0, L))
    err = torch.zeros(1, dtype=torch.int32, device=dev)
    x = si.make_hidden(w, (B, w.hidden), "cpu", 0, 1).to(dev)
    g = torch.Generator(device=dev)
    rows = []
    for seed in range(2):
        g.manual_seed(seed)
        rows.append([torch.randn((B * L, kv_heads, w.head_dim), generator=g, device=dev).to(w.torch_dtype) for _ in "kv"])
    out = torch.empty_like(x)

    def write(i):
        st.write_cache(0, *rows[i], cu, zero, p.block_table, err=err)

    def step():
        st.decode_step(x, lens, p.block_table, L + 1, out)

    want = []
    for i in range(2):
        write(i)
        torch.cuda.synchronize()
        step()
        torch.cuda.synchronize()
        want.append(out.clone())
    assert not torch.equal(*want)
    torch.cuda.synchronize()
    graphs = []
    if captured:
        for i in range(2):
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[i], stream=torch.cuda.current_stream()):
                write(i)
                step()
    for turn in range(20):
        if captured:
            graphs[turn % 2].replay()
        else:
            write(turn % 2)
            step()
        got = out.clone()
        torch.cuda.synchronize()
        assert torch.equal(got, want[turn % 2]), turn
    assert int(err) == 0 and st.device_error() == 0
    del graphs
    st.close()
