"""The windowed reference of the stack against the CPU oracle where they overlap, and refusals that need no device."""
import numpy as np
import pytest

import oracle
import paper_2502_20727_b200 as spd
import spd_inputs as si
from paper_2502_20727_b200 import build as spd_build
from parity_util import oracle_dims, to_np
from window_ref import stack_forward


@pytest.mark.parametrize("T,rope", [(1, 10000.0), (2, 10000.0), (2, 0.0)])
def test_reference_without_a_window_is_the_oracle(T, rope):
    w = si.Workload("tiny", "fp32", 2, 64, 4, 2, 32, 96, T, (0, 1), 2, 9, 3, rope_base=rope)
    layers = si.to_oracle_layers(si.make_stack(w, "cpu", 0))
    cache = oracle.Cache(oracle_dims(w), 2, 16)
    kc, vc = np.zeros((2, 2, 16, 2, 32)), np.zeros((2, 2, 16, 2, 32))
    pos = np.zeros(2, dtype=np.int32)
    for S in (5, 1, 7):
        x = to_np(si.make_hidden(w, (2, S, 64), "cpu", 0, S))
        ref, _, _ = oracle.stack_forward(oracle_dims(w), w.mask, layers, x, pos, cache)
        a = stack_forward(w, w.mask, layers, x, pos, kc.copy(), vc.copy(), window=64)  # wider than the context: the same
        b = stack_forward(w, w.mask, layers, x, pos, kc, vc)
        assert np.max(np.abs(b - ref)) <= 1e-12 * np.max(np.abs(ref)) and np.array_equal(a, b)
        pos = pos + S


def test_null_context_is_refused():
    spd_build.build()
    lib = spd.load_library()
    assert lib.spd_extend(None, 16, 1, 1, 16, 16, 1, 1, 32, None) == -2
    assert lib.spd_set_window(None, 4, 0) == -2


def test_attention_refuses_contexts_beyond_its_positions():
    spd_build.build()
    lib = spd.load_library()
    c = spd.spd_kv_cache(0x10000, 0x10000, None, None, 4, 2, 1 << 20, 64, 1)
    r = spd.spd_ragged(0x10000, 0x10000, 0x10000, 2, 4096, 0)  # no tokens: a call that is allowed does nothing
    for max_context, rc in ((1 << 30, 0), ((1 << 30) + 1, -1), (2 ** 31 - 1, -1)):
        assert lib.spd_paged_attention(c, r, 0x10000, 256, 0x20000, 256, 1, 4, 1, max_context, 0.1, 0, 0, None, 0, 0x10000, None) == rc
