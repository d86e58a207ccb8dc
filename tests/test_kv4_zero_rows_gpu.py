"""Attention over 4-bit pages where queries, keys or both are zeros or as good as: padding, a zero-filled cache, a warm-up on zeros.  Equal scores: the
mean of the visible rows of V."""
import pytest
import torch

from kv4_util import Batch4
from paged_util import check_attention
from test_paged_gpu import attend, run_and_check

pytestmark = pytest.mark.gpu


def batch(new, k_size=0.0, q_size=0.0, dtype="bf16", d=128, **kw):
    """32 heads on 8, four sequences: from 6 new tokens on more tiles of 16 rows than SMs."""
    bt = Batch4(dtype=dtype, nq=32, nkv=8, d=d, page=16, lens=[0, 129, 300, 17], new=[new, new, 1, new], lead=1, behind=2, seed=new,
                rows=lambda name, x: x * k_size if name == "k" else x, **kw)
    bt.q = (bt.q.double() * q_size).to(bt.dtype)
    return bt


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [1, 40, 150])
@pytest.mark.parametrize("window", [(0, 0), (50, 3)])
def test_zero_queries_over_zero_keys(dtype, d, new, window):
    run_and_check(batch(new, dtype=dtype, d=d, window=window[0], sinks=window[1]))


@pytest.mark.parametrize("new", [1, 40, 150])
def test_zero_queries_over_zero_filled_pages(new):
    """Parameters of 0 as well, as in memory that was filled with zeros and never appended to."""
    bt = batch(new)
    dev = bt.device()
    dev["k_pages"].zero_()
    dev["k_scales"].zero_()
    out, err = attend(bt, dev)
    assert err == 0
    check_attention(bt, out)


@pytest.mark.parametrize("new", [1, 40, 150])
@pytest.mark.parametrize("sizes", [(0, 1.0), (1.0, 0), (2.0 ** -90, 2.0 ** -55), (2.0 ** -55, 2.0 ** -90), (2.0 ** -120, 1.0), (2.0 ** -100, 2.0 ** -30)])
def test_products_next_to_nothing(new, sizes):
    run_and_check(batch(new, q_size=sizes[0], k_size=sizes[1]))


@pytest.mark.parametrize("new", [40, 150])
def test_some_rows_are_padding(new):
    """Every third query zero, the keys of every second sequence zeros."""
    bt = batch(new, q_size=1.0, k_size=1.0)
    bt.q[::3] = 0
    for b in (0, 2):
        for t in range(bt.lens[b] + bt.new[b]):
            p, s = bt.row_of(b, t)
            bt.values["k"][p, :, s] = 0
            bt.codes["k"][p, :, s] = 0
            bt.scales["k"][p, :, s] = 0
    run_and_check(bt)
