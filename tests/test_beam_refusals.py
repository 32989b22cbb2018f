"""What ann_beam_select and ann_beam_reorder refuse, before any work on the GPU (none is needed here), and the plain form by
hand."""
import ctypes as C

import numpy as np
import pytest

import beam_plain as P
from paper_2305_04359_amd import binding as A
from test_mx_refusals import PTR, refused

SELECT = dict(scores=PTR, groups=3, beams=4, n=100, dtype=2, ld=100, totals=PTR, finished=None, pad=0, k=8, parents=PTR, ids=PTR, out=PTR, scratch=PTR,
              bytes=1 << 30, stream=None)
FAR = PTR + (1 << 30)
REORDER = dict(x=PTR, out=FAR, parents=PTR, groups=3, beams=4, k=4, outer=2, outer_in=12 * 640, outer_out=12 * 640, row_in=640, row_out=640, mid=2, mid_in=320,
               mid_out=320, run=320, stream=None)


@pytest.mark.parametrize("name,good,bad", [
    *[("ann_beam_select", SELECT, b) for b in (dict(scores=None), dict(totals=None), dict(parents=None), dict(ids=None), dict(out=None), dict(scratch=None),
      dict(dtype=0), dict(dtype=5), dict(beams=0), dict(beams=65), dict(k=0), dict(k=129), dict(n=0), dict(n=1 << 24, ld=1 << 24), dict(groups=1 << 29),
      dict(ld=99), dict(bytes=100), dict(scratch=PTR + 8), dict(scores=PTR + 2), dict(totals=PTR + 1), dict(parents=PTR + 2), dict(ids=PTR + 2),
      dict(out=PTR + 2), dict(finished=PTR, pad=100))],
    *[("ann_beam_reorder", REORDER, b) for b in (dict(x=None), dict(out=None), dict(parents=None), dict(beams=0), dict(beams=65), dict(k=0), dict(k=65),
      dict(groups=1 << 25), dict(outer=1 << 31), dict(mid=1 << 31), dict(run=1 << 31), dict(parents=PTR + 2),
      dict(run=321), dict(row_in=639), dict(row_out=639), dict(mid_in=319), dict(outer_in=12 * 640 - 1), dict(outer_out=0), dict(row_in=0),  # overlaps
      dict(outer_in=1 << 62), dict(out=PTR + 640), dict(out=PTR + 2 * 12 * 640 - 1), dict(x=FAR + 640),
      dict(out=PTR, k=3), dict(out=PTR, outer_out=12 * 640 + 16), dict(out=PTR, row_out=656, outer_out=1 << 20, outer_in=1 << 20))],
])
def test_refused(name, good, bad):
    refused(name, *{**good, **bad}.values())


def test_totals_that_overlap_are_refused():
    # 12 totals of the beams; 3 x k of the continuations, whose groups' places are others than the beams' unless k = beams
    apart = dict(totals=PTR, out=FAR)
    for bad in (dict(out=PTR, k=8), dict(out=PTR, k=3), dict(out=PTR + 4, k=4), dict(out=PTR + 44, k=4), dict(out=PTR - 4 * 3 * 4 + 4, k=4), dict(out=PTR - 4 * 3 * 8 + 4, k=8)):
        refused("ann_beam_select", *{**SELECT, **apart, **bad}.values())


def test_nothing_to_do_reads_no_pointer():
    L = A.lib()
    assert L.ann_beam_select(*{**SELECT, "groups": 0, "scores": None, "totals": None, "parents": None, "ids": None, "out": None, "scratch": None}.values()) == 0
    for none in (dict(groups=0), dict(outer=0), dict(mid=0), dict(run=0)):
        assert L.ann_beam_reorder(*{**REORDER, **none, "x": None, "out": None, "parents": None}.values()) == 0


def test_scratch_sizes():
    L, b = A.lib(), C.c_uint64(7)
    assert L.ann_beam_select_scratch(0, 4, 100, 8, C.byref(b)) == 0 and b.value == 0
    assert L.ann_beam_select_scratch(1, 4, 100, 8, C.byref(b)) == 0 and b.value >= 4 * 8 * 8
    for args in ((1, 0, 100, 8), (1, 65, 100, 8), (1, 4, 0, 8), (1, 4, 1 << 24, 8), (1, 4, 100, 0), (1, 4, 100, 129), (1 << 31, 1, 100, 8)):
        refused("ann_beam_select_scratch", *args, C.byref(b))
    refused("ann_beam_select_scratch", 1, 4, 100, 8, None)


def test_binding_refuses_host_tensors():
    import torch
    with pytest.raises(ValueError):
        A.ann_beam_select(torch.zeros(4, 10), torch.zeros(4), 2, 3)
    with pytest.raises(ValueError):
        A.ann_beam_reorder(torch.zeros(4, 10), torch.zeros((2, 2), dtype=torch.int32), 2)


def test_dimensions_are_joined():
    # (size, stride, stride): a cache with room for more tokens, slices of it, and a dense side
    assert A._joined([(2, 600, 600), (3, 200, 200), (1, 7, 9), (200, 1, 1)]) == [(1200, 1, 1)]
    assert A._joined([(8, 2048, 1111), (1111, 1, 1)]) == [(8, 2048, 1111), (1111, 1, 1)]
    assert A._joined([(1, 3, 3)]) == []


def test_plain_form_by_hand():
    inf, nan = np.inf, np.nan
    z = np.log(np.array([[1.0, 2.0, 1.0], [6.0, 1.0, 1.0]]))
    p, i, v = P.select(z, [0.0, 0.0], 2, 3)
    assert p.tolist() == [[1, 0, 0]] and i.tolist() == [[0, 1, 0]] and np.allclose(v, np.log([[0.75, 0.5, 0.25]]))
    p, i, v = P.select(z, [0.0, -inf], 2, 4)
    assert p.tolist() == [[0, 0, 0, -1]] and i.tolist() == [[1, 0, 2, -1]] and v[0, 3] == -inf
    p, i, v = P.select(z, [0.0, -0.1], 2, 2, finished=[0, 1], pad=2)
    assert p.tolist() == [[1, 0]] and i.tolist() == [[2, 1]] and v[0, 0] == -0.1
    p, i, v = P.select(np.array([[inf, 0.0, inf, nan, -inf]]), [0.0], 1, 3)
    assert i.tolist() == [[0, 2, -1]] and np.allclose(v[0, :2], -np.log(2))
    assert P.select(np.array([[-inf, nan]]), [0.0], 1, 1)[1].tolist() == [[-1]]
