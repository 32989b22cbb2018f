"""What the calls on 8-bit rows refuse, before any work on the GPU (none is needed here), and the plain form by hand."""
import numpy as np
import pytest

import oct_plain as P
from paper_2305_04359_amd import binding as A
from test_mx_refusals import PTR, refused

QUANTIZE = dict(x=PTR, n=10, d=100, dtype=2, ldx=100, columns=0, codes=PTR, scales=PTR, stream=None)
DEQUANTIZE = dict(codes=PTR, scales=PTR, n=10, d=100, out=PTR, dtype=2, ldo=100, stream=None)
PRODUCT = dict(xcodes=PTR, xscales=PTR, nx=3, codes=PTR, scales=PTR, n=10, d=100, out=PTR, odtype=2, ldo=10, stream=None)


@pytest.mark.parametrize("name,good,bad", [
    *[("ann_oct_quantize", QUANTIZE, b) for b in (dict(x=None), dict(codes=None), dict(scales=None), dict(d=0), dict(d=(1 << 20) + 1), dict(n=1 << 31),
      dict(dtype=5), dict(dtype=-1), dict(ldx=99), dict(columns=1, ldx=9), dict(codes=PTR + 8), dict(scales=PTR + 2), dict(x=PTR + 2))],
    *[("ann_oct_dequantize", DEQUANTIZE, b) for b in (dict(codes=None), dict(scales=None), dict(out=None), dict(d=0), dict(dtype=0), dict(dtype=1),
      dict(dtype=7), dict(ldo=99), dict(out=PTR + 2), dict(codes=PTR + 4), dict(n=1 << 31))],
    *[("ann_oct_product", PRODUCT, b) for b in (dict(xcodes=None), dict(xscales=None), dict(codes=None), dict(scales=None), dict(out=None),
      dict(odtype=0), dict(odtype=5), dict(ldo=9), dict(nx=1 << 31), dict(n=1 << 31), dict(xcodes=PTR + 8), dict(xscales=PTR + 1), dict(codes=PTR + 1),
      dict(out=PTR + 2), dict(d=0), dict(d=(1 << 20) + 1))],
])
def test_refused(name, good, bad):
    refused(name, *{**good, **bad}.values())


def test_more_steps_than_32_bits_count_are_refused():
    big = dict(n=1 << 20, d=1 << 19)  # 2^32 steps
    for name, args in (("ann_oct_quantize", {**QUANTIZE, **big, "ldx": 1 << 20}), ("ann_oct_dequantize", {**DEQUANTIZE, **big, "ldo": 1 << 20}),
                       ("ann_oct_product", {**PRODUCT, **big, "ldo": 1 << 20}), ("ann_oct_product", {**PRODUCT, **big, "n": 10, "nx": 1 << 20})):
        refused(name, *args.values())


def test_nothing_to_do_reads_no_pointer():
    L = A.lib()
    for name, args, none in (("ann_oct_quantize", QUANTIZE, dict(n=0, x=None, codes=None, scales=None)),
                             ("ann_oct_quantize", QUANTIZE, dict(n=0, ldx=0, columns=1, x=None, codes=None, scales=None)),
                             ("ann_oct_dequantize", DEQUANTIZE, dict(n=0, codes=None, scales=None, out=None)),
                             ("ann_oct_product", PRODUCT, dict(nx=0, xcodes=None, xscales=None, out=None)),
                             ("ann_oct_product", PRODUCT, dict(n=0, codes=None, scales=None, out=None))):
        assert getattr(L, name)(*{**args, **none}.values()) == 0, (name, none)


def test_binding_refuses_host_tensors():
    import torch
    with pytest.raises(ValueError):
        A.ann_oct_quantize(torch.zeros(3, 4))
    with pytest.raises(ValueError):
        A.OctRows(torch.zeros((3, 128), dtype=torch.uint8), torch.zeros((3, 4), dtype=torch.uint8), 100)


def test_plain_form_by_hand():
    """The restatement that the GPU tests compare with, at values that the definition settles by hand."""
    x = np.array([[448.0, 433.0, 432.0, 431.0, 1.0, 1.0625, 1.1875, -1.0625, 2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -10, 2.0 ** -10 * 1.01, -0.0, 464.0 / 512]])
    codes, scales = P.quantize(x)
    assert scales.tolist() == [[127, 0, 0, 0]]
    want = [448.0, 448.0, 448.0, 416.0, 1.0, 1.0, 1.25, -1.0, 2.0 ** -9, 0.0, 2.0 ** -8, 2.0 ** -9, 0.0, 0.875]
    assert P.values(codes, scales, 14).tolist() == [want]
    assert codes[0, 12] == 128  # -0 keeps its sign
    for most, byte in ((448.0, 127), (np.nextafter(448.0, 500), 128), (896.0, 128), (897.0, 129), (0.0, 0), (2.0 ** -149, 0), (np.inf, 255), (np.nan, 255),
                       (1.75, 127 - 8), (1.76, 127 - 7)):
        assert P.quantize(np.array([[most, 0.0]]))[1][0, 0] == byte
