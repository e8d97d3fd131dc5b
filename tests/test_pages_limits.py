"""Which limits the calls of the paged prompt cache have, on the host: every call is refused for its own and no other's."""
import ctypes as C

import pytest

from test_pages_abi import V, chunk_of, create, rows_of  # noqa: F401


def test_rows_in_and_out_have_no_limits_of_the_queries(V):
    """2^24 new rows of 8 query heads are more than an attention call takes; 2^24 rows of one KV head can be written and read.
    (An arena that was never cleared refuses the valid call, last of all checks: nothing is launched.)"""
    s, n, h, st = create(V, L=1, Hq=8, Hkv=1, d=64)
    assert st == V.VLC_OK
    r = C.byref(rows_of(V))
    many = C.byref(chunk_of(V, B=1, max_pages=1 << 21, max_new=1 << 24, max_len=1 << 25))
    assert V.lib.vlc_pages_attn(h, many, 0, 1, r, None, None, None, r, None, None, 0, None) == V.VLC_ERR_SHAPE
    for st in (V.lib.vlc_pages_write(h, many, 0, 1, r, r, None), V.lib.vlc_pages_read(h, many, 0, 1, 0, 10, r, r, None)):
        assert st == V.VLC_ERR_INVALID_ARG and "vlc_pages_clear" in V.vlc_last_error_string()
    V.lib.vlc_pages_destroy(h)


@pytest.mark.parametrize("Hkv,rows,refused", [(8, 1 << 23, False), (8, (1 << 23) + 1, True), (64, 1 << 21, True), (1, 1 << 25, False)])
def test_rows_of_all_heads_that_a_launch_takes(V, Hkv, rows, refused):
    s, n, h, st = create(V, L=1, Hq=8 * Hkv, Hkv=Hkv, d=64)
    assert st == V.VLC_OK
    r = C.byref(rows_of(V, head=1 << 33))
    writes = C.byref(chunk_of(V, B=1, max_pages=1 << 21, max_new=rows, max_len=1 << 25))
    reads = C.byref(chunk_of(V, B=1, max_pages=1 << 21, max_new=1, max_len=1 << 25))
    want = V.VLC_ERR_SHAPE if refused else V.VLC_ERR_INVALID_ARG
    assert V.lib.vlc_pages_write(h, writes, 0, 1, r, r, None) == want
    assert ("vlc_pages_clear" in V.vlc_last_error_string()) != refused
    assert V.lib.vlc_pages_read(h, reads, 0, 1, 0, rows, r, r, None) == want
    assert ("vlc_pages_clear" in V.vlc_last_error_string()) != refused
    V.lib.vlc_pages_destroy(h)
