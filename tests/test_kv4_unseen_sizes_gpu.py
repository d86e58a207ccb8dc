"""Rows of a 4-bit cache that some queries do not see and that are a few times as large as the others: what a query gets is off by no more than the stated rounding of the rows that it sees, 2^-10
of the larger of 16 s and |m| of a row at most."""
import math

import pytest
import torch

import paper_2502_20727_b200 as spd
from kv4_util import values4

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("power", [1, 4, 7, 8, 9])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("which", ["newest", "window"])
def test_small_elements_beside_large_unseen_rows(power, d, which):
    """V: half of the dims hold m = 2^-6 (1 + 37/128) in every row (code 0), the others up to 1.  Queries of zeros: the mean of V.  A rounding of the output to bfloat16 (2^-8) and of a weight to
    float16 (2^-11), float32 sums; a value of V to float16 beside rows 2^8 times as large: half a step of 2^-24, once for m and once for the value, in units of 2^6 times the largest power of two: 2^-10 of
    16 s = 1."""
    B, new, nq, nkv, page, len0 = 8, 64, 32, 8, 16, 40
    n_all = len0 + new
    g = torch.Generator().manual_seed(power)
    pages = -(-n_all // page)
    n_pages = B * pages
    kp = torch.zeros((n_pages, nkv, page, d // 2), dtype=torch.uint8)
    ks = torch.ones((n_pages, nkv, page, 2, 2), dtype=torch.bfloat16)
    vp = torch.randint(0, 16, (n_pages, nkv, page, d // 2), generator=g, dtype=torch.uint8)
    vp[..., : d // 4] = 0
    vs = torch.empty((n_pages, nkv, page, 2, 2))
    vs[..., 0], vs[..., 1] = 1 / 16, 2.0 ** -6 * (1 + 37 / 128)
    window = 0 if which == "newest" else 30
    odd = n_all - 1 if which == "newest" else 12  # seen by the last query, or by the first two
    p, r = torch.arange(B) * pages + odd // page, odd % page
    vs[p, :, r] *= 2.0 ** power
    vs = vs.to(torch.bfloat16)
    rows = values4(vp, vs).view(B, pages, nkv, page, d).permute(0, 1, 3, 2, 4).reshape(B, pages * page, nkv, d)[:, :n_all]
    q = torch.zeros((B * new, nq, d), dtype=torch.bfloat16)
    i32 = lambda t: t.to(torch.int32).cuda()  # noqa: E731
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = spd.paged_attention(q.cuda(), kp.cuda(), vp.cuda(), i32(torch.arange(B + 1) * new), i32(torch.full((B,), len0)), i32(torch.arange(n_pages).view(B, pages)), max_new=new,
                              max_context=n_all, window=window, err=err, k_scales=ks.cuda(), v_scales=vs.cuda())
    assert int(err) == 0
    out = out.double().cpu().view(B, new, nq, d)
    tried = 0
    for i in range(new):
        pos = len0 + i
        lo = max(0, pos - window + 1) if window else 0
        if lo <= odd <= pos:
            continue
        ref = rows[:, lo:pos + 1].mean(1).repeat_interleave(nq // nkv, 1)
        tol = (1.01 * 2.0 ** -8 + 2.0 ** -11 + 2.0 ** -18 + math.ceil(n_all / 16) * 2.0 ** -23) * ref.abs() + 2.0 ** -10
        assert ((out[:, i] - ref).abs() <= tol).all(), (i, ((out[:, i] - ref).abs() / tol).max())
        tried += 1
    assert tried >= new // 2
