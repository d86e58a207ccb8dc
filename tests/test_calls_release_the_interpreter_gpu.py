"""The operators' calls do not hold the interpreter's lock while the driver makes them wait, as it does when a stream's queue is full."""
import threading
import time

import pytest
import torch

import paper_2502_20727_b200 as spd
from kv4_util import Batch4

pytestmark = pytest.mark.gpu


def calls():
    bt = Batch4(dtype="bf16", nq=8, nkv=2, d=64, page=16, lens=[20, 3], new=[1, 1], seed=1)
    d = bt.device()
    i = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    kv = dict(err=d["err"], k_scales=d["k_scales"], v_scales=d["v_scales"])
    k = torch.zeros((bt.n, 2, 64), dtype=torch.bfloat16, device="cuda")
    out, kr, vr = torch.empty_like(d["q"]), torch.empty_like(k), torch.empty_like(k)
    slots, free, table = i(-1, -1), torch.zeros(bt.n_pages, dtype=torch.int32, device="cuda"), d["table"].clone()
    plan = spd.plan_batch(d["lens"], i(0, 0), table, free, i(0), page=16, n_pages=bt.n_pages, n_tokens=2, err=d["err"])
    at, zero = (d["cu"], d["lens"], d["table"]), i(0, 0)
    return {"kv_write": lambda: spd.kv_write(k, k, d["k_pages"], d["v_pages"], *at, **kv),
            "kv_write_slots": lambda: spd.kv_write_slots(k, k, d["k_pages"], d["v_pages"], slots, **kv),
            "kv_read": lambda: spd.kv_read(d["k_pages"], d["v_pages"], *at, out=(kr, vr), **kv),
            "paged_attention": lambda: spd.paged_attention(d["q"], d["k_pages"], d["v_pages"], *at, max_new=1, max_context=21, out=out, **kv),
            "plan_batch": lambda: spd.plan_batch(d["lens"], zero, table, free, plan.n_free, page=16, n_pages=bt.n_pages, n_tokens=2, err=d["err"], out=plan)}


@pytest.mark.parametrize("name", ["kv_write", "kv_write_slots", "kv_read", "paged_attention", "plan_batch"])
def test_other_threads_run_meanwhile(name):
    call = calls()[name]
    call()
    torch.cuda.synchronize()
    took = []

    def fill():  # more launches than a stream's queue holds, behind a kernel of about 0.7 s
        with torch.cuda.stream(torch.cuda.Stream()):
            torch.cuda._sleep(1_300_000_000)
            start = time.perf_counter()
            for _ in range(3000):
                call()
            took.append(time.perf_counter() - start)
            torch.cuda.current_stream().synchronize()

    t = threading.Thread(target=fill)
    t.start()
    gap, last = 0.0, time.perf_counter()
    while t.is_alive():
        now = time.perf_counter()
        gap, last = max(gap, now - last), now
    t.join()
    assert took and took[0] > 0.4, f"the queue was not full ({took})"
    assert gap < 0.25, f"this thread stood still for {gap:.2f} s"
