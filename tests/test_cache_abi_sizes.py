"""mars_kv_attention at the most work that its deal counts in 32 bits: what is beyond is refused on the host (no call here reaches a kernel:
those that are not too large have too small a workspace)."""
import os

import pytest

ARG, WORKSPACE = -1, -3
P = 0x1000  # never dereferenced


@pytest.fixture(scope="module")
def C():
    from paper_2601_15498_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2601_15498_amd import build
        build.build()
    from paper_2601_15498_amd import cache
    return cache


@pytest.mark.parametrize("B,N,heads,mask,width,fits", [
    # 2^30 tokens, 8 388 608 units of 128, behind which 300 nodes are three blocks of 128 rows: two pairs of twice as many units
    (79, 300, 2, False, 1 << 22, False), (59, 300, 2, False, 1 << 22, True), (60, 300, 2, False, 1 << 22, False),
    # under a mask they are three blocks of a unit more each
    (79, 300, 2, True, 1 << 22, True), (80, 300, 2, True, 1 << 22, False),
    # 200 nodes are one block of 256 rows
    (238, 200, 2, False, 1 << 22, True), (239, 200, 2, False, 1 << 22, False),
    # one token
    (238, 1, 2, False, 1 << 22, True), (239, 1, 2, False, 1 << 22, False),
    # short sequences of one unit, counted as two: blocks of rows go out whole
    (4096, 1, 1 << 16, False, 1, True), (4096, 8 * 128, 1 << 16, True, 1, False),
])
def test_work_that_cannot_be_counted_is_refused(C, B, N, heads, mask, width, fits):
    cache = C.CacheStruct(P, P, P, P, P, 1, 4, heads, 64, 256 if width > 1 else 8, 3, width)
    rows = C.RowsStruct(P, 1 << 20, 1 << 12, 64)
    rc = C.lib().mars_kv_attention(cache, 0, None, rows, 1, heads, None, P if mask else None, 1.0, 0, rows, None, B, N, 0x100000, 1, None)
    assert rc == (WORKSPACE if fits else ARG)


@pytest.mark.parametrize("scale,ok", [(1e-45, True), (2.3e38, True), (2.4e38, False), (3.4e38, False)])
def test_a_scale_whose_powers_of_two_are_no_number_is_refused(C, scale, ok):
    """The kernels take exp2(scale * log2(e) * score): the factor has to be a number in 32 bits."""
    rows = C.RowsStruct(P, 1 << 20, 1 << 12, 64)
    rc = C.lib().mars_kv_attention(C.CacheStruct(P, P, P, P, P, 1, 4, 2, 64, 16, 3, 8), 0, None, rows, 1, 2, None, None, scale, 0, rows, None, 2, 3, 0x100000, 1,
                                   None)
    assert rc == (WORKSPACE if ok else ARG)
