"""Calls whose host bounds are far beyond what the batch holds, up to the documented limit of 2^30 tokens: the launch follows the rows that there are."""
import pytest
import torch

from kv4_util import Batch4
from paged_util import Batch, check_attention
from test_paged_gpu import attend

pytestmark = pytest.mark.gpu
PAGE = 1024


def batch(dtype, fmt, **kw):
    return Batch4(dtype=dtype, **kw) if fmt == "int4" else Batch(dtype=dtype, fmt=fmt, **kw)


@pytest.mark.parametrize("dtype,fmt,d", [("f32", "int4", 128), ("f32", "int4", 64), ("f32", "int4", 32), ("f32", "f32", 64), ("f32", "int8", 128), ("bf16", "int4", 128), ("bf16", "int4", 64),
                                         ("bf16", "int4", 32), ("bf16", "bf16", 128), ("bf16", "e4m3", 64), ("bf16", "int8", 128), ("bf16", "bf16", 32)])
@pytest.mark.parametrize("nq,nkv", [(4, 1), (64, 1), (8, 8)])
@pytest.mark.parametrize("bound", [2 ** 30, 2 ** 29 + 1, 2 ** 24])
def test_bounds_far_beyond_the_batch(dtype, fmt, d, nq, nkv, bound):
    bt = batch(dtype, fmt, nq=nq, nkv=nkv, d=d, page=PAGE, lens=[40, 3, 0, 700], new=[9, 1, 0, 150], lead=1, behind=2, seed=nq)
    bt.table = torch.cat([bt.table, torch.full((bt.B, 2 ** 30 // PAGE), -7, dtype=torch.int32)], 1)
    out, err = attend(bt, max_new=bound, max_context=bound)
    assert err == 0
    live = check_attention(bt, out)
    assert (out.cpu()[~live] == 77.0).all()


@pytest.mark.parametrize("dtype,fmt", [("f32", "int4"), ("bf16", "int4"), ("bf16", "bf16"), ("f32", "f32")])
def test_a_sequence_beyond_the_tensor_is_still_skipped(dtype, fmt):
    bt = batch(dtype, fmt, nq=8, nkv=2, d=64, page=PAGE, lens=[40, 3], new=[9, 40], seed=3)
    bt.table = torch.cat([bt.table, torch.full((bt.B, 2 ** 30 // PAGE), -7, dtype=torch.int32)], 1)
    ref, tol = bt.reference()
    for end in (bt.n + 1, 2 ** 31 - 1):
        dev = bt.device()
        dev["cu"][2] = end
        out, err = attend(bt, dev, max_new=2 ** 30, max_context=2 ** 30)
        assert err == 2
        assert ((out.double().cpu() - ref).abs() <= tol)[:9].all() and (out[9:] == 77).all()
