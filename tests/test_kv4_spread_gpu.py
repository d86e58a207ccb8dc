"""V rows of very unequal size under one query: rows within 2^100 of one another, a row of zeros counting as 2^-60."""
import pytest
import torch

from kv4_util import Batch4
from test_paged_gpu import attend

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,power", [("f32", 0), ("f32", 20), ("f32", 36), ("bf16", 0), ("bf16", 25)])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("new", [1, 3, 40, 150])
def test_zero_rows_beside_large_ones(dtype, power, d, new):
    """Rows of zeros take their share of the softmax whatever the others hold.  float32: three roundings at a size below 128 (half a step, 2^-18) of a score with its
    V row's exponent, in a weight and in the weights' sum: 6 ln 2 2^-18, under 2^-15.9."""
    def rows(name, x):
        if name == "k":
            return x * 0.25
        i = torch.arange(x.shape[0] * x.shape[2]).view(x.shape[0], 1, x.shape[2], 1)
        return torch.where(i % 3 == 0, 0.0, x * 2.0 ** power)
    bt = Batch4(dtype=dtype, nq=32, nkv=8, d=d, page=16, lens=[120, 9, 33, 0], new=[new, 1, new, new], seed=44, rows=rows)
    out, err = attend(bt)
    assert err == 0
    ref, tol = bt.reference()
    live = ~torch.isnan(ref[:, 0, 0])
    if dtype == "f32":
        tol = tol + 2.0 ** -15.9 * bt.values["v"].nan_to_num(0.0).abs().max()
    assert ((out.double().cpu() - ref).abs() <= tol)[live].all()
