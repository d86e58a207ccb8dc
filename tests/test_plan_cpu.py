"""Host-side checks of the step's plan: every refusal comes before a device is touched."""
import pytest
import torch

import paper_2502_20727_b200 as spd
from test_paged_cpu import P, lib  # noqa: F401


def plan(lib, pool=None, **kw):  # noqa: F811
    a = {**dict(lens=P, new=2 * P, B=2, table=P, width=4, n=3, cu=P, pos=P, slots=P, nxt=3 * P, err=P), **kw}
    p = spd.spd_page_pool(*{**dict(free=P, n_free=P, nxt=P, n_pages=4, page=16), **(pool or {})}.values())
    return lib.spd_plan_batch(p, *a.values(), None)


def test_refusals(lib):  # noqa: F811
    for kw, rc in ((dict(lens=None), -2), (dict(new=None), -2), (dict(table=None), -2), (dict(cu=None), -2), (dict(pos=None), -2), (dict(slots=None), -2),
                   (dict(nxt=None), -2), (dict(err=None), -2), (dict(B=-1), -1), (dict(B=16385), -1), (dict(width=0), -1), (dict(width=2 ** 27), -1),
                   (dict(n=-1), -1), (dict(nxt=P), -1), (dict(nxt=2 * P), -1)):
        assert plan(lib, **kw) == rc, kw
    for kw, rc in ((dict(free=None), -2), (dict(n_free=None), -2), (dict(nxt=None), -2), (dict(n_pages=0), -1), (dict(page=0), -1),
                   (dict(n_pages=2 ** 27), -1)):
        assert plan(lib, pool=kw) == rc, kw
    assert lib.spd_plan_batch(None, P, P, 2, P, 4, 3, P, P, P, 2 * P, P, None) == -2


def test_binding_refuses_what_does_not_match():
    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ValueError):  # no CPU tensors
        spd.plan_batch(i(2), i(2), i(2, 4), i(8), i(1), page=16, n_pages=8, n_tokens=3, err=i(1))


def test_more_rows_than_row_numbers(lib):  # noqa: F811
    assert plan(lib, n=2 ** 30 + 1) == -1 and plan(lib, n=2 ** 31 - 1) == -1
