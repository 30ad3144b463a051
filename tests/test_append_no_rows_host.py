"""Steps without rows: a rotating append of none has no queries and no positions to point at (an empty tensor's pointer is
NULL), and is no error; what does not depend on the rows is still checked.  Host only: nothing is launched."""
import ctypes as C

import pytest

from test_paged_host import CACHE, L, fill  # noqa: F401
from test_rotary_host import QUERIES, ROT, ROWS

NONE = dict(n_rows=0, k=0, v=0, slots=0, row_seq=0, row_pos=0)


def call(L, bits, rows, fields):  # noqa: F811
    rows = {**CACHE, **ROWS, **rows}
    if bits == 8:
        a = fill(L.PagedAppendRotaryArgs(), {**{f"rows.{k}": v for k, v in rows.items()}, **ROT, **fields})
        return L.raw().lvspec_paged_append_rotary(C.byref(a), None)
    return L.raw().lvspec_paged_mx_append(C.byref(fill(L.PagedMxAppendArgs(), {**rows, **ROT, **fields})), None)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("fields", [
    dict(QUERIES, q=0, q_out=0), {"rot.n_axes": 3, "rot.pos": 0}, {"rot.n_axes": 3, "rot.pos": 0, **QUERIES, "q": 0, "q_out": 0},
    dict(QUERIES), {"rot.pos": 0, "Hq": 0}])
def test_no_rows_is_no_error(L, bits, fields):  # noqa: F811
    assert call(L, bits, NONE, fields) == L.OK


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("change,want", [({"Hq": -1}, -1), ({"Hq": 65536}, -2), ({"rot.dim": 24}, -2), ({"rot.transpose": 1}, -1),
                                         ({"rot.n_axes": 5}, -1), ({"rot.inv_freq": 0}, -1)])
def test_what_needs_no_rows_is_checked(L, bits, change, want):  # noqa: F811
    assert call(L, bits, NONE, {**QUERIES, **change}) == want


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("change", [dict(q=0), dict(q_out=0), {"rot.n_axes": 3, "rot.pos": 0}])
def test_one_row_needs_them(L, bits, change):  # noqa: F811
    assert call(L, bits, dict(n_rows=1), {**QUERIES, **change}) == L.EINVAL
