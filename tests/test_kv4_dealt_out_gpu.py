"""Single and drafted tokens over 4-bit pages whose keys are dealt out evenly to the warps that fit the GPU, under windows and sinks.  The workspace that such a call
asks for says that it is one."""
import ctypes
import random

import pytest
import torch

import paper_2502_20727_b200 as spd
from kv4_util import Batch4
from paged_util import check_attention
from test_paged_gpu import attend

pytestmark = pytest.mark.gpu


def is_dealt_out(bt, new, bound):
    lib, n = spd.load_library(), ctypes.c_size_t(0)
    c = spd.spd_kv_cache(None, None, None, None, bt.n_pages, bt.nkv, bt.page, bt.d, 5)
    assert lib.spd_paged_attention_workspace_bytes(c, bt.B, bt.n, 1, bt.nq, new, bound, bt.window, bt.sinks, n) == 0
    few = new * (bt.nq // bt.nkv) <= 8
    warps = torch.cuda.get_device_properties(0).multi_processor_count * (3 if few else 2) * 4
    return n.value == warps * 2 * (8 if few else 16) * (bt.d + 2) * 4 + 513 * 4


@pytest.mark.parametrize("B,nq,new,window,sinks", [(92, 16, 1, 2500, 40), (92, 64, 1, 2500, 0), (114, 16, 4, 2048, 0), (78, 8, 8, 2100, 1000), (64, 32, 4, 2500, 40), (64, 16, 8, 2200, 130),
                                                   (60, 72, 1, 2300, 7), (60, 16, 1, 0, 0), (60, 16, 8, 0, 0)])
@pytest.mark.parametrize("d,page", [(64, 16), (128, 24)])
def test_windows(B, nq, new, window, sinks, d, page):
    bound = 4096
    rng = random.Random(B + nq)
    lens = [rng.choice([0, 1, 31, 32, 33, 200, window + 40, rng.randint(0, 3900)]) for _ in range(B)]
    bt = Batch4(dtype="bf16", nq=nq, nkv=8, d=d, page=page, lens=lens, new=[rng.randint(0, new) if new > 1 else 1 for _ in range(B)], window=window, sinks=sinks, lead=1, behind=2,
                seed=B, offset=0.3)
    bt.table = torch.cat([bt.table, torch.full((B, bound // page + 1), -7, dtype=torch.int32)], 1)
    assert is_dealt_out(bt, new, bound)
    out, err = attend(bt, max_new=new, max_context=bound)
    assert err == 0
    live = check_attention(bt, out)
    assert (out.cpu()[~live] == 77.0).all()
    again, _ = attend(bt, max_new=new, max_context=bound)
    assert torch.equal(out, again)
