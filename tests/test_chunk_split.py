"""How a call over chunks cuts contexts (chunk_split of csrc/cdb_internal.h): what the grid and the records are sized by.
CPU only: no call here reaches a launch."""
import ctypes as C

import pytest

from paper_2608_09444_amd import chunk

MOST_PAGES = (2 ** 31 - 1 - 64) // 16  # of a page table
MOST_SEGMENTS, RECORD_ROWS = 16, 4096


class Split(C.Structure):
    _fields_ = [("want", C.c_int), ("most", C.c_int)]


def split(heads, chunks, rows, pages):
    f = chunk.lib()._ZN3cdb11chunk_splitEiiii
    f.restype, f.argtypes = Split, [C.c_int] * 4
    s = f(heads, chunks, rows, pages)
    return s.want, s.most


CALLS = [(h, c, r) for h in (1, 4, 16, 55, 128) for c, r in ((1, 1), (1, 13), (64, 64), (256, 256), (1, 512), (2, 2048), (3, 2100),
                                                               (2, 4097), (256, 65536), (0, 0))]
FAR = [2 ** 26 - 1, 2 ** 26, 2 ** 26 + 1, 100_000_000, MOST_PAGES - 3, MOST_PAGES - 1, MOST_PAGES]


@pytest.mark.parametrize("heads,chunks,rows", CALLS)
def test_every_table_has_segments_that_records_hold(heads, chunks, rows):
    for pages in [*range(0, 700), *(2 ** k + d for k in range(10, 26) for d in (-1, 0, 1)), *FAR]:
        want, most = split(heads, chunks, rows, pages)
        assert 1 <= want and 1 <= most <= MOST_SEGMENTS, pages
        assert most == 1 or most * rows <= RECORD_ROWS, pages


@pytest.mark.parametrize("heads,chunks,rows", CALLS)
def test_a_wider_table_has_no_fewer_segments(heads, chunks, rows):
    """What a table could hold takes no segments from shorter contexts in it."""
    most = [split(heads, chunks, rows, pages)[1] for pages in (*range(1, 4000), *range(4000, 20000, 37), *FAR)]
    assert all(b >= a for a, b in zip(most, most[1:]))
