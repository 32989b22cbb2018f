"""What ann_distill and ann_distill_grad refuse, before any work on the GPU (none is needed here)."""
import ctypes as C

import pytest

from paper_2305_04359_amd import binding as A
from test_mx_refusals import PTR, refused

LOSS = dict(scores=PTR, rows=3, n=100, dtype=2, ld=100, ids=PTR, teacher=PTR, tdtype=2, k=5, t=1.0, losses=PTR, stats=PTR, scratch=PTR, bytes=1 << 30,
            stream=None)
GRAD = dict(scores=PTR, rows=3, n=100, dtype=2, ld=100, ids=PTR, teacher=PTR, tdtype=2, k=5, t=1.0, stats=PTR, grads=None, scale=1.0, out=PTR + (1 << 20), ldo=100,
            stream=None)
BOTH = (dict(scores=None), dict(ids=None), dict(teacher=None), dict(stats=None), dict(dtype=0), dict(dtype=5), dict(tdtype=1), dict(tdtype=-1), dict(n=0),
        dict(n=1 << 31, ld=1 << 31), dict(rows=1 << 31), dict(ld=99), dict(k=0), dict(k=1025), dict(t=0.0), dict(t=-1.0), dict(t=float("nan")),
        dict(t=float("inf")), dict(t=2.0 ** -61), dict(t=2.0 ** 61), dict(scores=PTR + 2), dict(ids=PTR + 2), dict(teacher=PTR + 1), dict(stats=PTR + 2))


@pytest.mark.parametrize("name,good,bad", [
    *[("ann_distill", LOSS, b) for b in (*BOTH, dict(losses=None), dict(losses=PTR + 1), dict(n=100_000, ld=100_000, scratch=None),
                                         dict(n=100_000, ld=100_000, bytes=8), dict(n=100_000, ld=100_000, scratch=PTR + 8))],
    *[("ann_distill_grad", GRAD, b) for b in (*BOTH, dict(out=None), dict(out=PTR + 2), dict(ldo=99), dict(grads=PTR + 2), dict(out=PTR, ldo=101), dict(out=PTR + 4),
                                               dict(out=PTR + 400, ld=150), dict(out=PTR + 800), dict(out=PTR - 4, ld=200, ldo=200), dict(out=PTR + 396, ld=200, ldo=200))],
])
def test_refused(name, good, bad):
    refused(name, *{**good, **bad}.values())


def test_nothing_to_do_reads_no_pointer():
    L = A.lib()
    none = dict(rows=0, scores=None, ids=None, teacher=None, stats=None)
    assert L.ann_distill(*{**LOSS, **none, "losses": None, "scratch": None}.values()) == 0
    assert L.ann_distill_grad(*{**GRAD, **none, "out": None}.values()) == 0


def test_scratch_sizes():
    L, b = A.lib(), C.c_uint64(7)
    assert L.ann_distill_scratch(0, 100, C.byref(b)) == 0 and b.value == 0
    assert L.ann_distill_scratch(1, 8192, C.byref(b)) == 0 and b.value == 0
    assert L.ann_distill_scratch(1, (1 << 31) - 1, C.byref(b)) == 0 and 0 < b.value < 1 << 20
    for args in ((1 << 31, 100), (10, 0), (10, 1 << 31)):
        refused("ann_distill_scratch", *args, C.byref(b))
    refused("ann_distill_scratch", 10, 100, None)


def test_binding_refuses_host_tensors():
    import torch
    z, i = torch.zeros(3, 4), torch.zeros((3, 2), dtype=torch.int32)
    with pytest.raises(ValueError):
        A.ann_distill(z, i, torch.zeros(3, 2))


def test_strides_beyond_memory_are_refused():
    # (4 * 2^62 and 4 * 3 * 2^60 leave 64 bits)
    for rows, big in ((1, 1 << 62), (3, 1 << 60), (2, 1 << 63)):
        refused("ann_distill", *{**LOSS, "rows": rows, "ld": big}.values())
        refused("ann_distill_grad", *{**GRAD, "rows": rows, "ld": big}.values())
        refused("ann_distill_grad", *{**GRAD, "rows": rows, "ldo": big}.values())
        refused("ann_distill_grad", *{**GRAD, "rows": rows, "ld": big, "ldo": big}.values())
