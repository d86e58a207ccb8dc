"""Into how many ranges the keys of calls over 4-bit pages are cut, by the workspace that holds their partial rows: within what a launch can have, and none
that a call of many row tiles does not need."""
import ctypes

import pytest

from test_kv4_cpu import cache4
from test_paged_cpu import lib  # noqa: F401

MAX_GRID_Z = 65535  # a launch has sequences times ranges there


def ranges(lib, B, n_tokens, nq, nkv, new, context, d=128, window=0):  # noqa: F811
    n = ctypes.c_size_t(0)
    c = cache4(n_kv_heads=nkv, head_dim=d, n_pages=4096)
    assert lib.spd_paged_attention_workspace_bytes(c, B, n_tokens, 1, nq, new, context, window, 0, n) == 0
    return max(1, n.value // (n_tokens * nq * (d + 2) * 4))


@pytest.mark.parametrize("B,n_tokens,nq,nkv,new,context", [(9486, 9486 * 5, 8, 1, 5, 131072), (9486, 9490, 8, 1, 5, 131072), (1187, 1187 * 3, 8, 1, 3, 1 << 20), (8291, 8291 * 3, 8, 1, 3, 131072),
                                                           (65535, 65535 * 3, 8, 1, 3, 8192), (65535, 65540, 8, 1, 700, 1 << 20), (40000, 1000, 20, 1, 2, 8192), (2000, 2000, 64, 2, 1, 1 << 30)])
@pytest.mark.parametrize("d", [64, 128])
def test_many_sequences_fit_a_launch(lib, B, n_tokens, nq, nkv, new, context, d):  # noqa: F811
    assert B * ranges(lib, B, n_tokens, nq, nkv, new, context, d) <= MAX_GRID_Z


@pytest.mark.parametrize("B,new,context,nq,nkv", [(1, 2048, 16384, 64, 8), (1, 1024, 16384, 64, 8), (1, 4096, 16384, 64, 8), (1, 8192, 1 << 20, 64, 8), (12, 700, 1700, 40, 40), (2, 2048, 4096, 32, 32),
                                                  (600, 5, 32768, 64, 8)])
def test_many_row_tiles_need_no_ranges(lib, B, new, context, nq, nkv):  # noqa: F811
    """More row tiles than twice the SMs keep them busy as they are."""
    assert (new * (nq // nkv) + 127) // 128 * nkv * B > 2 * 148
    assert ranges(lib, B, B * new, nq, nkv, new, context) == 1
