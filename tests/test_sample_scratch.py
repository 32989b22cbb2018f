"""Scratch of ann_sample for rows that are divided among workgroups: missing, short or misaligned, it is refused before any
work on the GPU (none is needed here)."""
import ctypes as C

import pytest

from paper_2305_04359_amd import binding as A
from test_mx_refusals import PTR, SAMPLE, refused


@pytest.mark.parametrize("rows,n", [(1, 4097), (3, 5000), (700, 70_003), (5000, 128_000)])
def test_refused(rows, n):
    L, need = A.lib(), C.c_uint64(0)
    assert L.ann_sample_scratch(rows, n, C.byref(need)) == 0 and need.value > 0
    good = {**SAMPLE, "rows": rows, "n": n, "ld": n, "bytes": need.value}
    for bad in (dict(scratch=None), dict(scratch=PTR + 8), dict(scratch=PTR + 4), dict(bytes=need.value - 1), dict(bytes=0)):
        refused("ann_sample", *{**good, **bad}.values())


def test_scratch_grows_with_the_rows_up_to_a_part():
    """Short rows need none; long ones are taken 4,096 at a time."""
    L, need = A.lib(), C.c_uint64(0)

    def of(rows, n):
        assert L.ann_sample_scratch(rows, n, C.byref(need)) == 0
        return need.value

    assert of(10 ** 6, 4096) == 0 and of(0, 5000) == 0
    assert 0 < of(1, 4097) < of(2, 4097) < of(4096, 4097) == of(4097, 4097) == of(10 ** 6, 4097)
