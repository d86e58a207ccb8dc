"""What a plan refuses, it refuses before it allocates its outputs."""
import pytest
import torch

import paper_2502_20727_b200 as spd

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_tokens", [-1, 2 ** 30 + 1, 2 ** 31 - 1, 2 ** 40])
def test_more_rows_than_a_plan_has(n_tokens):
    i = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    lens, new, table, free, n_free, err = i(3, 0), i(1, 1), i(0, 1, 2, 3).view(2, 2), torch.zeros(8, dtype=torch.int32, device="cuda"), i(0), i(0)
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    with pytest.raises(spd.SpdError):
        spd.plan_batch(lens, new, table, free, n_free, page=16, n_pages=8, n_tokens=n_tokens, err=err)
    assert torch.cuda.max_memory_allocated() - before < 1 << 20
