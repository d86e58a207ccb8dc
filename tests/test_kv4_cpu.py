"""Host-side checks of the 4-bit cache and the slot append: every refusal comes before a device is touched."""
import ctypes

import pytest
import torch

import paper_2502_20727_b200 as spd
from test_paged_cpu import P, attend, cache, lib, ragged, write  # noqa: F401

INT4 = 5


def cache4(**kw):
    return cache(**{**dict(format=INT4, k_scales=P, v_scales=P), **kw})


@pytest.mark.parametrize("read", [False, True])
def test_cache_refusals(lib, read):  # noqa: F811
    for kw, rc in ((dict(k_scales=None), -2), (dict(v_scales=None), -2), (dict(k_scales=P + 4), -1), (dict(v_scales=P + 2), -1), (dict(head_dim=48), -1),
                   (dict(k_pages=P + 8), -1), (dict(v_pages=None), -2), (dict(format=6), -1), (dict(format=4), -1)):
        assert write(lib, c=cache4(**kw), read=read) == rc, kw
        assert attend(lib, c=cache4(**kw)) == rc, kw
    assert write(lib, c=cache4(), r=ragged(n_tokens=0), read=read) == 0 and attend(lib, c=cache4(), r=ragged(B=0)) == 0


def test_slot_append_refusals(lib):  # noqa: F811
    def call(c=None, **kw):
        a = {**dict(slots=P, n=3, k=P, v=P, ks=128, vs=128, dtype=1, err=P), **kw}
        return lib.spd_kv_write_slots(c or cache4(), *a.values(), None)
    for kw, rc in ((dict(slots=None), -2), (dict(k=None), -2), (dict(v=None), -2), (dict(err=None), -2), (dict(n=-1), -1), (dict(dtype=2), -1),
                   (dict(k=P + 4), -1), (dict(ks=120), -1), (dict(vs=132), -1)):
        assert call(**kw) == rc, kw
    assert lib.spd_kv_write_slots(None, P, 3, P, P, 128, 128, 1, P, None) == -2
    assert call(c=cache(format=2)) == -2
    assert call(n=0, slots=None, k=None, v=None) == 0


def test_workspace_is_asked_for_by_format(lib):  # noqa: F811
    n = ctypes.c_size_t(0)
    big = cache4(n_kv_heads=1, head_dim=128, n_pages=4096)
    assert lib.spd_paged_attention_workspace_bytes(big, 1, 1, 1, 8, 1, 65536, 0, 0, n) == 0 and n.value > 0
    assert attend(lib, c=big, r=ragged(B=1, n_tokens=1, max_pages=4096), nq=8, qs=1024, os=1024, max_new=1, max_context=65536) == -3
    assert lib.spd_paged_attention_workspace_bytes(cache4(format=4), 1, 1, 1, 8, 1, 65536, 0, 0, n) == -1


def test_binding_refuses_what_does_not_match():
    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    pages, scales = torch.zeros((4, 2, 16, 32), dtype=torch.uint8), torch.zeros((4, 2, 16, 2, 2), dtype=torch.bfloat16)
    x = torch.zeros((3, 2, 64))
    for kw in (dict(), dict(k_scales=scales, v_scales=scales)):  # no CPU tensors
        with pytest.raises(ValueError):
            spd.kv_write(x, x, pages, pages, i(3), i(2), i(2, 4), err=i(1), **kw)
        with pytest.raises(ValueError):
            spd.kv_write_slots(x, x, pages, pages, i(3), err=i(1), **kw)
