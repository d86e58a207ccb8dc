"""Rows of a 4-bit cache that a query does not see may hold anything, the largest finite parameters of either sign and memory that nothing was written to among them."""
import pytest
import torch

from kv4_util import Batch4
from test_paged_gpu import attend

pytestmark = pytest.mark.gpu


def blind_rows(bt, t):
    """Queries of a single sequence that do not see key t."""
    pos = torch.arange(bt.lens[0], bt.lens[0] + bt.new[0])
    gone = (pos - bt.window >= t) if bt.window else torch.zeros_like(pos, dtype=torch.bool)
    return (pos < t) | gone


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("s,m", [(2.0 ** 12, -2.0 ** 16), (2.0 ** 60, 1.0), (2.0 ** 104, 2.0 ** 110), (2.0 ** 125, 0.0), (2.0 ** 126, -2.0 ** 127), (3.3e38, 3.3e38), (-3.3e38, 3.3e38),
                                 (-3.3e38, -3.3e38), (0.0, 3.3e38)])
@pytest.mark.parametrize("new", [2, 8, 150])
@pytest.mark.parametrize("d", [32, 64, 128])
def test_any_finite_parameters(dtype, s, m, new, d):
    tried = 0
    for window, at in ((0, -1), (33, 8), (40, 10)):  # the newest row; rows that the window has passed for all but the first queries
        bt = Batch4(dtype=dtype, nq=8, nkv=4, d=d, page=16, lens=[40], new=[new], window=window, seed=11)
        dev = bt.device()
        t = 40 + new - 1 if at < 0 else at
        p, row = bt.row_of(0, t)
        if int(bt.table[0, t // 16]) != p:
            continue
        for name in ("k", "v"):
            dev[name + "_pages"][p, :, row] = 255
            dev[name + "_scales"][p, :, row, :, 0] = s
            dev[name + "_scales"][p, :, row, :, 1] = m
        out, err = attend(bt, dev)
        assert err == 0
        ref, tol = bt.reference()
        blind = blind_rows(bt, t)
        assert ((out.double().cpu() - ref).abs() <= tol)[blind].all()
        tried += int(blind.any())
    assert tried >= 2


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("new", [1, 9, 70])
@pytest.mark.parametrize("d", [32, 64, 128])
def test_memory_that_nothing_was_written_to(dtype, new, d):
    """The slots behind a sequence's end hold every 16-bit pattern in turn."""
    for lens in ([33], [70]):
        bt = Batch4(dtype=dtype, nq=8, nkv=4, d=d, page=256, lens=lens, new=[new], seed=12)
        n = lens[0] + new
        ref, tol = bt.reference()
        g = torch.Generator().manual_seed(5)
        for _ in range(4):
            dev = bt.device()
            p = bt.row_of(0, 0)[0]
            for name in ("k_scales", "v_scales"):
                junk = torch.randint(-2 ** 15, 2 ** 15, dev[name][p, :, n:].shape, generator=g, dtype=torch.int16)
                dev[name][p, :, n:] = junk.view(torch.bfloat16).cuda()
            out, err = attend(bt, dev)
            assert err == 0
            live = torch.arange(bt.cu[0], bt.cu[1])
            assert ((out.double().cpu() - ref).abs() <= tol)[live].all()
