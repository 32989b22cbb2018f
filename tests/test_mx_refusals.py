"""What the calls on 4-bit rows and ann_sample refuse, before any work on the GPU (none is needed here)."""
import ctypes as C

import numpy as np
import pytest

import mx_plain as P
from paper_2305_04359_amd import binding as A

PTR = 1 << 20  # stands for an aligned device pointer; refused calls read nothing


def refused(name, *args):
    L = A.lib()
    assert getattr(L, name)(*args) == -1, args
    assert L.ann_last_error().decode()


QUANTIZE = dict(x=PTR, n=10, d=100, dtype=2, ldx=100, codes=PTR, scales=PTR, norms=None, stream=None)
DEQUANTIZE = dict(codes=PTR, scales=PTR, n=10, d=100, out=PTR, dtype=2, ldo=100, stream=None)
PRODUCT = dict(x=PTR, nx=3, xdtype=4, ldx=100, codes=PTR, scales=PTR, n=10, d=100, out=PTR, odtype=2, ldo=10, stream=None)
PRODUCT_MX = dict(xcodes=PTR, xscales=PTR, nx=3, codes=PTR, scales=PTR, n=10, d=100, out=PTR, odtype=2, ldo=10, stream=None)
SEARCH = dict(codes=PTR, scales=PTR, norms=PTR, n=1000, d=100, metric=0, qcodes=PTR, qscales=PTR, qnorms=PTR, nq=3, k=10, ids=PTR,
              dists=PTR, scratch=PTR, bytes=1 << 20, stream=None)
SAMPLE = dict(scores=PTR, rows=3, n=10, dtype=2, ld=10, opts=None, uniform=PTR, ids=PTR, logprobs=None, scratch=PTR, bytes=1 << 30, stream=None)


@pytest.mark.parametrize("name,good,bad", [
    *[("ann_mx_quantize", QUANTIZE, b) for b in (dict(x=None), dict(codes=None), dict(scales=None), dict(d=0), dict(d=65537), dict(n=1 << 31),
      dict(dtype=5), dict(dtype=-1), dict(ldx=99), dict(codes=PTR + 8), dict(scales=PTR + 2), dict(x=PTR + 2), dict(norms=PTR + 1))],
    *[("ann_mx_dequantize", DEQUANTIZE, b) for b in (dict(codes=None), dict(scales=None), dict(out=None), dict(d=0), dict(dtype=0), dict(dtype=1),
      dict(dtype=7), dict(ldo=99), dict(out=PTR + 2), dict(codes=PTR + 4))],
    *[("ann_mx_product", PRODUCT, b) for b in (dict(x=None), dict(codes=None), dict(scales=None), dict(out=None), dict(xdtype=0), dict(xdtype=9),
      dict(odtype=1), dict(ldx=99), dict(ldo=9), dict(nx=1 << 31), dict(n=1 << 31), dict(d=0), dict(x=PTR + 1), dict(out=PTR + 2),
      dict(codes=PTR + 8))],
    *[("ann_mx_product_mx", PRODUCT_MX, b) for b in (dict(xcodes=None), dict(xscales=None), dict(codes=None), dict(scales=None), dict(out=None),
      dict(odtype=0), dict(ldo=9), dict(nx=1 << 31), dict(xcodes=PTR + 8), dict(xscales=PTR + 1), dict(d=70000))],
    *[("ann_mx_search", SEARCH, b) for b in (dict(codes=None), dict(qcodes=None), dict(qscales=None), dict(norms=None), dict(qnorms=None),
      dict(ids=None), dict(dists=None), dict(scratch=None), dict(scratch=PTR + 8), dict(bytes=15), dict(k=0), dict(k=129), dict(metric=2),
      dict(n=1 << 31), dict(nq=1 << 31), dict(d=0), dict(norms=PTR + 2), dict(ids=PTR + 1))],
    *[("ann_sample", SAMPLE, b) for b in (dict(scores=None), dict(uniform=None), dict(ids=None), dict(dtype=0), dict(dtype=6), dict(n=0),
      dict(n=1 << 31), dict(rows=1 << 31), dict(ld=9), dict(scores=PTR + 2), dict(uniform=PTR + 2), dict(ids=PTR + 3), dict(logprobs=PTR + 1))],
])
def test_refused(name, good, bad):
    refused(name, *{**good, **bad}.values())


def test_sample_refuses_settings_that_are_not_aligned():
    for field in ("temperature_dev", "top_k_dev", "top_p_dev", "min_p_dev"):
        o = A.SampleOpts(temperature=1.0)
        setattr(o, field, PTR + 2)
        refused("ann_sample", *{**SAMPLE, "opts": C.byref(o)}.values())


def test_nothing_to_do_reads_no_pointer():
    L = A.lib()
    for name, args, none in (("ann_mx_quantize", QUANTIZE, dict(n=0, x=None, codes=None, scales=None)),
                             ("ann_mx_dequantize", DEQUANTIZE, dict(n=0, codes=None, scales=None, out=None)),
                             ("ann_mx_product", PRODUCT, dict(nx=0, x=None, out=None)),
                             ("ann_mx_product", PRODUCT, dict(n=0, codes=None, scales=None, out=None)),
                             ("ann_mx_product_mx", PRODUCT_MX, dict(nx=0, xcodes=None, xscales=None, out=None)),
                             ("ann_mx_search", SEARCH, dict(nq=0, qcodes=None, qscales=None, ids=None, dists=None)),
                             ("ann_sample", SAMPLE, dict(rows=0, scores=None, uniform=None, ids=None))):
        assert getattr(L, name)(*{**args, **none}.values()) == 0, (name, none)


def test_scratch_sizes():
    L, b = A.lib(), C.c_uint64(7)
    assert L.ann_mx_search_scratch(0, 100, 5, 10, C.byref(b)) == 0 and b.value == 0
    for args in ((1 << 31, 100, 5, 10), (10, 0, 5, 10), (10, 100, 1 << 31, 10), (10, 100, 5, 0), (10, 100, 5, 129)):
        refused("ann_mx_search_scratch", *args, C.byref(b))
    refused("ann_mx_search_scratch", 10, 100, 5, 10, None)
    refused("ann_sample_scratch", 10, 0, C.byref(b))
    refused("ann_sample_scratch", 10, 10, None)


def test_binding_refuses_host_tensors():
    import torch
    with pytest.raises(ValueError):
        A.ann_mx_quantize(torch.zeros(3, 4))
    with pytest.raises(ValueError):
        A.MxRows(torch.zeros((3, 64), dtype=torch.uint8), torch.zeros((3, 4), dtype=torch.uint8), 100)
    with pytest.raises(ValueError):
        A.ann_sample(torch.zeros(3, 4), torch.zeros(3))


def test_plain_form_of_the_levels():
    """The restatement that the GPU tests compare with, at values that the definition settles by hand."""
    x = np.array([[6.0, 5.0, 4.9, 5.1, 0.25, 0.75, 0.26, 1.25, 1.75, 2.5, 3.5, -2.5, -0.0, 7.9, 7.0]])
    codes, scales = P.quantize(x)
    assert scales.tolist() == [[127, 0, 0, 0]]
    want = [6.0, 4.0, 4.0, 6.0, 0.0, 1.0, 0.5, 1.0, 2.0, 2.0, 4.0, -2.0, 0.0, 6.0, 6.0]
    assert P.values(codes, scales, 15).tolist() == [want]
    assert codes[0, 6] & 15 == 8  # -0 keeps its sign
    assert P.quantize(np.array([[8.0]]))[1][0, 0] == 128 and P.quantize(np.array([[0.0]]))[1][0, 0] == 0
    assert P.quantize(np.array([[1.0, np.inf]]))[1][0, 0] == 255
    assert P.draw(np.array([0.0, 0.0, -np.inf, 0.0]), 0.5) == (1, pytest.approx(-np.log(3)))
    assert P.draw(np.array([-np.inf]), 0.5) == (-1, -np.inf)
    assert P.draw(np.array([1.0, 5.0, 5.0]), 0.9, temperature=0.0) == (1, 0.0)
