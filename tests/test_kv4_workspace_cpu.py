"""A workspace that is asked for once, with the bounds of a program's steps and its most tokens, serves every step of fewer tokens."""
import ctypes
import random

import pytest

from test_paged_cpu import cache, lib  # noqa: F401
from test_kv4_cpu import cache4

FORMATS = {"int4": lambda **kw: cache4(**kw), "bf16": lambda **kw: cache(format=1, **kw), "int8": lambda **kw: cache(format=3, k_scales=0x10000, v_scales=0x10000, **kw)}


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("seed", range(8))
def test_fewer_tokens_need_no_more(lib, fmt, seed):  # noqa: F811
    rng = random.Random(seed)
    spread = lambda lo, hi: int(lo * (hi / lo) ** rng.random())  # noqa: E731
    for _ in range(400):
        nkv, group, B, new, context = rng.choice([1, 2, 4, 8, 40]), rng.choice([1, 2, 4, 8, 16]), spread(1, 400), spread(1, 3000), spread(1, 200000)
        c = FORMATS[fmt](n_kv_heads=nkv, head_dim=rng.choice([32, 64, 128]), n_pages=4096)
        dtype, window, n, need = rng.choice([0, 1, 1]) if fmt != "bf16" else 1, rng.choice([0, 0, spread(1, 5000)]), ctypes.c_size_t(0), []
        for tokens in sorted({1, B, *(spread(1, B * new) for _ in range(6)), B * new}):
            assert lib.spd_paged_attention_workspace_bytes(c, B, tokens, dtype, nkv * group, new, context, window, 4, n) == 0
            need.append(n.value)
        assert need == sorted(need), (nkv, group, B, new, context, need)
