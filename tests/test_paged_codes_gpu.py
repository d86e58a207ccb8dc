"""int8 codes of appended rows, bit for bit: code = x * (127 * (1 / max|x|)) with every step rounded to float32."""
import pytest
import torch

import paper_2502_20727_b200 as spd

pytestmark = pytest.mark.gpu


def write(x, page=16):
    """x: [n, nkv, d] appended as K and V of one sequence; the codes and scales that were stored, [n, nkv, d] and [n, nkv]."""
    n, nkv, d = x.shape
    pages = -(-n // page)
    i = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    codes = {k: torch.zeros((pages, nkv, page, d), dtype=torch.int8, device="cuda") for k in "kv"}
    scales = {k: torch.zeros((pages, nkv, page), device="cuda") for k in "kv"}
    err = i([0])
    spd.kv_write(x.cuda(), x.cuda(), codes["k"], codes["v"], i([0, n]), i([0]), i([list(range(pages))]), err=err, k_scales=scales["k"],
                 v_scales=scales["v"])
    assert int(err) == 0 and torch.equal(codes["k"], codes["v"]) and torch.equal(scales["k"], scales["v"])
    c = codes["k"].transpose(1, 2).reshape(pages * page, nkv, d)[:n]
    return c.cpu(), scales["k"].transpose(1, 2).reshape(pages * page, nkv)[:n].cpu()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d", [32, 64, 128])
def test_int8_codes_are_the_rounded_products(dtype, d):
    g = torch.Generator().manual_seed(d)
    n, nkv = 1500, 3
    top = torch.exp2(torch.rand((n, nkv, 1), generator=g) * 40 - 20)
    # values next to the borders between two codes: (j + 1/2) top / 127, up to four float32 steps to either side
    j = torch.randint(-127, 127, (n, nkv, d), generator=g).float() + 0.5
    x = (j.double() * top.double() / 127).float()
    x = (x.view(torch.int32) + torch.randint(-4, 5, x.shape, generator=g, dtype=torch.int32)).view(torch.float32)
    x[..., :1] = top
    x = x.to(dtype)
    f = x.float()
    top = f.abs().amax(-1, keepdim=True)
    codes, scales = write(x)
    assert torch.equal(codes, torch.round(f * (top.reciprocal() * 127)).to(torch.int8))
    assert torch.equal(scales, (top / 127)[..., 0])
