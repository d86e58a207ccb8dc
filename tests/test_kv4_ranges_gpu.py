"""Calls over 4-bit pages of very many sequences under long host bounds: they launch, and no ranges of the keys are made that the launch has no room for."""
import pytest
import torch

from kv4_util import Batch4
from paged_util import check_attention
from test_paged_gpu import attend

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,new,nq,bound", [(9486, 5, 8, 131072), (1187, 3, 8, 1 << 20), (8291, 3, 8, 131072), (40000, 2, 20, 8192)])
@pytest.mark.parametrize("d", [64, 128])
def test_many_sequences_under_a_long_bound(B, new, nq, bound, d):
    lens, news = [0] * B, [0] * B
    for i in range(0, B, 97):
        lens[i], news[i] = i % 200, 1 + i % new
    bt = Batch4(dtype="bf16", nq=nq, nkv=1, d=d, page=256, lens=lens, new=news, lead=1, behind=2, seed=7)
    bt.table = torch.cat([bt.table, torch.full((bt.B, bound // 256), -7, dtype=torch.int32)], 1)
    out, err = attend(bt, max_new=new, max_context=bound)
    assert err == 0
    check_attention(bt, out)
