"""Whether rows are worked on together at the sizes that tests/kv_units_cases.py gives for it, seen by the workspace without a GPU."""
import ctypes as C

import pytest

import kv_units_cases as cases
from paper_2605_17415_amd import kv
from test_host_kv import cache, lib  # noqa: F401


def workspace(lib, rows, heads, group, batch, max_new, columns, count):  # noqa: F811
    """16 bits, 64 coordinates, pages so long that every list has tiles to share: room for parts is asked for where the workgroups are fewer than the
    chip holds, 1,024, so never by as many rows and heads that are worked on one by one."""
    c = cache(format=kv.BF16, d=64, page=1024, heads=heads, batch=batch, columns=columns, table_stride=columns)
    return lib.ivftq_kv_attend_pages_workspace(C.byref(c), rows, heads * group, max_new, count)


@pytest.mark.parametrize("case,group", cases.ALL)
def test_rows_are_worked_on_together(lib, case, group):  # noqa: F811
    rows, batch = sum(case.news), len(case.news)
    assert rows * case.heads >= 1024
    assert workspace(lib, rows, case.heads, group, batch, max(case.news), case.columns, case.count) > 0
    # one by one: heads that fill a product's columns alone, and one row a sequence at a time
    assert workspace(lib, rows, case.heads, 16, batch, max(case.news), case.columns, case.count) == 0
    assert workspace(lib, rows, case.heads, group, rows, 1, case.columns, case.count) == 0
