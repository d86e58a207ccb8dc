"""Host-side checks of the paged-cache operators: every refusal comes before a device is touched."""
import ctypes

import pytest
import torch

import paper_2502_20727_b200 as spd
from paper_2502_20727_b200 import build as spd_build

P = 0x10000  # stands for a 16-byte aligned device address; refused calls never use it


@pytest.fixture(scope="module")
def lib():
    spd_build.build()
    return spd.load_library()


def cache(**kw):
    base = dict(k_pages=P, v_pages=P, k_scales=None, v_scales=None, n_pages=4, n_kv_heads=2, kv_block_size=16, head_dim=64, format=1)
    base.update(kw)
    return spd.spd_kv_cache(*base.values())


def ragged(**kw):
    base = dict(cu_new=P, seq_lens=P, block_table=P, B=2, max_pages=4, n_tokens=3)
    base.update(kw)
    return spd.spd_ragged(*base.values())


def write(lib, c=None, r=None, read=False, **kw):
    a = dict(k=P, v=P, ks=128, vs=128, dtype=1, err=P)
    a.update(kw)
    return (lib.spd_kv_read if read else lib.spd_kv_write)(c or cache(), r or ragged(), a["k"], a["v"], a["ks"], a["vs"], a["dtype"], a["err"], None)


BAD_CACHE = [(dict(format=4), -1), (dict(format=-1), -1), (dict(head_dim=48), -1), (dict(head_dim=256), -1), (dict(n_pages=0), -1),
             (dict(n_kv_heads=0), -1), (dict(kv_block_size=0), -1), (dict(k_pages=None), -2), (dict(v_pages=None), -2), (dict(k_pages=P + 8), -1),
             (dict(format=2), -2), (dict(format=3, k_scales=P), -2), (dict(format=3, k_scales=P + 2, v_scales=P), -1)]
BAD_RAGGED = [(dict(cu_new=None), -2), (dict(seq_lens=None), -2), (dict(block_table=None), -2), (dict(B=-1), -1), (dict(max_pages=0), -1),
              (dict(n_tokens=-1), -1)]


@pytest.mark.parametrize("read", [False, True])
def test_cache_refusals(lib, read):
    for kw, rc in BAD_CACHE:
        assert write(lib, c=cache(**kw), read=read) == rc, kw
    for kw, rc in BAD_RAGGED:
        assert write(lib, r=ragged(**kw), read=read) == rc, kw
    for kw, rc in ((dict(k=None), -2), (dict(v=None), -2), (dict(err=None), -2), (dict(dtype=2), -1), (dict(k=P + 4), -1), (dict(ks=120), -1),
                   (dict(vs=132), -1)):
        assert write(lib, read=read, **kw) == rc, kw
    assert write(lib, r=ragged(B=0), read=read) == 0 and write(lib, r=ragged(n_tokens=0), read=read, k=None, v=None) == 0


def attend(lib, c=None, r=None, **kw):
    a = dict(q=P, qs=256, out=2 * P, os=256, dtype=1, nq=4, max_new=2, max_context=40, scale=0.1, window=0, sinks=0, ws=None, wsb=0, err=P)
    a.update(kw)
    return lib.spd_paged_attention(c or cache(), r or ragged(), *a.values(), None)


def test_attention_refusals(lib):
    for kw, rc in BAD_CACHE:
        assert attend(lib, c=cache(**kw)) == rc, kw
    for kw, rc in BAD_RAGGED:
        assert attend(lib, r=ragged(**kw)) == rc, kw
    nan = float("nan")
    for kw, rc in ((dict(q=None), -2), (dict(out=None), -2), (dict(err=None), -2), (dict(out=P), -1), (dict(dtype=3), -1), (dict(nq=3), -1),
                   (dict(nq=0), -1), (dict(max_new=0), -1), (dict(max_context=0), -1), (dict(scale=0.0), -1), (dict(scale=-1.0), -1),
                   (dict(scale=nan), -1), (dict(scale=float("inf")), -1), (dict(window=-1), -1), (dict(sinks=-1), -1), (dict(qs=255), -1),
                   (dict(os=252), -1), (dict(max_context=65), -4), (dict(q=P + 2), -1), (dict(dtype=0), -1)):
        assert attend(lib, **kw) == rc, kw
    assert attend(lib, c=cache(format=0)) == -1  # a bfloat16 query on a float32 cache
    assert attend(lib, r=ragged(B=0)) == 0 and attend(lib, r=ragged(n_tokens=0), q=None, out=None) == 0


def test_workspace_refusals(lib):
    n = ctypes.c_size_t(0)
    ask = lambda c=None, **kw: lib.spd_paged_attention_workspace_bytes(c or cache(), *{**dict(B=2, n=3, dtype=1, nq=4, mn=2, mc=40, w=0, s=0), **kw}.values(), n)  # noqa: E731
    assert ask() == 0
    for kw in (dict(B=-1), dict(n=-1), dict(nq=0), dict(nq=3), dict(mn=0), dict(mc=0), dict(w=-1), dict(s=-1), dict(dtype=2)):
        assert ask(**kw) == -1, kw
    assert lib.spd_paged_attention_workspace_bytes(None, 1, 1, 1, 1, 1, 1, 0, 0, n) == -2
    # a single token on a long context is split over thread blocks, and then needs its partial results kept
    big = cache(n_kv_heads=1, head_dim=128, n_pages=4096)
    assert ask(big, B=1, n=1, nq=8, mn=1, mc=65536) == 0 and n.value > 0
    need = n.value
    r = ragged(B=1, n_tokens=1, max_pages=4096)
    kw = dict(nq=8, qs=1024, os=1024, max_new=1, max_context=65536)
    assert attend(lib, c=big, r=r, **kw) == -3
    assert attend(lib, c=big, r=r, ws=P, wsb=need - 1, **kw) == -3
    assert attend(lib, c=big, r=r, ws=P + 16, wsb=need + 64, **kw) == -3


def test_binding_refuses_what_does_not_match():
    pages = torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16)
    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ValueError):  # no CPU tensors
        spd.paged_attention(torch.zeros((3, 4, 64), dtype=torch.bfloat16), pages, pages, i(3), i(2), i(2, 4), max_new=2, max_context=40, err=i(1))
    with pytest.raises(ValueError):
        spd.kv_write(torch.zeros((3, 2, 64)), torch.zeros((3, 2, 64)), pages, pages, i(3), i(2), i(2, 4), err=i(1))
    with pytest.raises(ValueError):
        spd.kv_read(pages, pages, i(3), i(2), i(2, 4), err=i(1), n_tokens=3)
