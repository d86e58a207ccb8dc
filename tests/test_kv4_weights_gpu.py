"""Softmax weights of very unequal size over 4-bit pages: one key takes nearly all of the softmax and has a small V row, tens of thousands of equal ones share the
rest and make a good part of the output.  Their weights are rounded to float16 alike, so that errors add up instead of cancelling."""
import math

import pytest
import torch

import paper_2502_20727_b200 as spd
from kv4_util import values4

pytestmark = pytest.mark.gpu


def long_context(N, B, new, nq, nkv, d, share, seed=0):
    """B sequences over the same pages: key 0 scores 15 times the scale, all others 0; V row 0 is 1/64 of the others, which are all alike.  share: a tail key's weight
    relative to key 0's."""
    page = 256
    g = torch.Generator().manual_seed(seed)
    n_pages = N // page
    kp = torch.zeros((n_pages, nkv, page, d // 2), dtype=torch.uint8, device="cuda")
    ks = torch.zeros((n_pages, nkv, page, 2, 2), dtype=torch.bfloat16, device="cuda")
    ks[..., 0] = 1
    kp[0, :, 0, 0] = 15
    vp = torch.randint(0, 256, (1, nkv, 1, d // 2), generator=g, dtype=torch.uint8).cuda().expand(n_pages, nkv, page, d // 2).contiguous()
    s = (1 + torch.rand((1, nkv, 1, 2), generator=g)).to(torch.bfloat16).cuda()
    vs = torch.zeros((n_pages, nkv, page, 2, 2), dtype=torch.bfloat16, device="cuda")
    vs[..., 0] = s
    vs[0, :, 0] /= 64
    n = B * new
    q = torch.zeros((n, nq, d), dtype=torch.bfloat16, device="cuda")
    q[:, :, 0] = 1
    cu = torch.arange(0, n + 1, new, dtype=torch.int32, device="cuda")
    lens = torch.full((B,), N - new, dtype=torch.int32, device="cuda")
    table = torch.arange(n_pages, dtype=torch.int32, device="cuda").repeat(B, 1)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    scale = -math.log(share) / 15
    out = spd.paged_attention(q, kp, vp, cu, lens, table, max_new=new, max_context=N, err=err, k_scales=ks, v_scales=vs, scale=scale)
    assert int(err) == 0
    # every query sees a few keys more or less of 2^15 and more: counted exactly
    v = values4(vp[0, :, :2].cpu(), vs[0, :, :2].cpu())  # [nkv, 2, d]
    tail = (N - new + torch.arange(new, dtype=torch.float64)).repeat(B)[:, None, None] * share
    v = v.repeat_interleave(nq // nkv, 0)
    ref = (v[None, :, 0] + tail * v[None, :, 1]) / (1 + tail)
    return out.double().cpu(), ref


def check(out, ref, subnormal):
    """A rounding of the output to bfloat16 (2^-8), of a weight and of a value to float16 (2^-11 each), of a score to float32 (2^-24 of up to 30, and twice that of a weight), and what
    is given as `subnormal`: the share of the output that is lost where a weight is below float16's normal numbers."""
    tol = (1.01 * 2.0 ** -8 + 2 * 2.0 ** -11 + 2 * 30 * 2.0 ** -24 + 2.0 ** -16 + subnormal) * ref.abs()
    worst = ((out - ref).abs() / tol.clamp(min=1e-30))[ref != 0].max()
    assert worst <= 1, f"{worst:.2f} of the tolerance"


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("units", [1.5, 2.5, 0.4])
def test_tail_of_a_chunk(d, units):
    """Rows in tiles of 128, one range: every tile follows the maximum of the first.  A weight relative to the largest is scaled by 2^7 and then off by 2^-25 at most: units
    2^-24 by a share of 2^-8 / units of the tail, of which the output has at most all."""
    N = 32768
    out, ref = long_context(N, 320, 5, 8, 1, d, units * 2.0 ** -24)
    check(out, ref, 2.0 ** -8 / units)


@pytest.mark.parametrize("d", [64, 128])
def test_tail_of_single_tokens(d):
    """Keys dealt out evenly: a warp has about 9000 of one sequence.  Weights are relative to the largest contribution to the output, so that a tail key's is 2.5 x 2^-18 here, times
    its row's scale in units of its power of two (1 to 2), and off by 2^-25 at most: 2^-8 / 2.5 of the 29 % of the tail that lie with key 0; the tail makes a
    quarter of the output."""
    N = 32768
    out, ref = long_context(N, 64, 1, 64, 8, d, 2.5 * 2.0 ** -24)
    check(out, ref, 2.0 ** -8 / 2.5 * 0.29 * 0.25)
