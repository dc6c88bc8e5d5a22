"""Row lengths whose loop counters would pass 31 bits on the device are refused before anything touches it (the pointers are never dereferenced)."""
import ctypes as C

import pytest

from paper_2401_06706_amd import binding as M


@pytest.mark.parametrize("field", ["S", "n_bias"])
@pytest.mark.parametrize("n", [2 ** 30 + 1, 2 ** 31 - 100, 2 ** 31 - 1])
def test_histories_and_bias_lists(field, n):
    sizes = dict(B=1, N=0, V=100, R=1, dtype=0, per_seq=0, begin=0, end=1, S=0, n_bias=0)
    ptrs = {name: 1 << 20 for name, _ in M.LogitsBufs._fields_[1:]}
    ptrs["row_map"] = None
    bufs = M.LogitsBufs(C.sizeof(M.LogitsBufs), *ptrs.values())
    call = lambda **kw: M.lib().mcsd_logits_rules(C.byref(M.LogitsDesc(C.sizeof(M.LogitsDesc), *{**sizes, **kw}.values())), C.byref(bufs), None)
    assert call(**{field: n}) == -3
    assert b"2^30" in M.lib().mcsd_last_error()
    assert call(**{field: 2 ** 30, "end": 0}) == 0             # (no rows, no launch)


@pytest.mark.parametrize("n", [2 ** 30 + 1, 2 ** 31 - 1])
def test_rows_of_a_block_table(n):
    bufs = M.PageBufs(C.sizeof(M.PageBufs), *[4096 for _ in M.PageBufs._fields_[1:]])
    desc = M.PageDesc(C.sizeof(M.PageDesc), 1, 1, 100, n, 8)
    assert M.lib().mcsd_page_assign(C.byref(desc), C.byref(bufs), None) == -3
    assert b"2^30" in M.lib().mcsd_last_error()
