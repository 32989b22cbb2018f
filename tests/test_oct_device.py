"""The device that the calls on 8-bit rows, distillation and beam steps run on: that of their tensors, whichever is current (no
GPU needed: stand-ins as for the calls on 4-bit rows)."""
import pytest
import torch

from paper_2305_04359_amd import binding as A
from test_mx_device import Tensor, calls  # noqa: F401


def all_calls(device):
    x = Tensor((6, 200), device=device)
    rows = A.ann_oct_quantize(x)
    A.ann_oct_quantize(x, columns=True)
    A.ann_oct_dequantize(rows)
    A.ann_oct_product(rows, rows)
    ids, teacher = Tensor((6, 4), torch.int32, device), Tensor((6, 4), device=device)
    _, stats = A.ann_distill(x, ids, teacher)
    A.ann_distill_grad(x, ids, teacher, stats, grad_losses=Tensor(6, device=device))
    parents, _, _ = A.ann_beam_select(x, Tensor(6, device=device), 3, 3, finished=Tensor(6, torch.bool, device))
    A.ann_beam_reorder(x, parents, 3)


NAMES = ["ann_oct_quantize", "ann_oct_quantize", "ann_oct_dequantize", "ann_oct_product", "ann_distill", "ann_distill_grad", "ann_beam_select",
         "ann_beam_reorder"]


def test_calls_run_on_the_device_of_their_tensors(calls):  # noqa: F811
    for index in (1, 0):
        calls.clear()
        all_calls(f"cuda:{index}")
        assert calls == [(name, index, 1000 + index) for name in NAMES]


def test_tensors_of_other_devices_are_refused(calls):  # noqa: F811
    x, far = Tensor((6, 200)), Tensor((6, 4), device="cuda:0")
    rows, stats = A.ann_oct_quantize(x), Tensor((6, 2))
    ids, teacher, parents = Tensor((6, 4), torch.int32), Tensor((6, 4)), Tensor((2, 3), torch.int32)
    calls.clear()
    for call in (lambda: A.ann_oct_product(rows, A.ann_oct_quantize(Tensor((6, 200), device="cuda:0"))) or calls.pop(),
                 lambda: A.ann_oct_product(rows, rows, out=Tensor((6, 6), device="cuda:0")),
                 lambda: A.ann_distill(x, ids, far), lambda: A.ann_distill(x, Tensor((6, 4), torch.int32, "cuda:0"), teacher),
                 lambda: A.ann_distill_grad(x, ids, teacher, Tensor((6, 2), device="cuda:0")),
                 lambda: A.ann_distill_grad(x, ids, teacher, stats, grad_losses=Tensor(6, device="cuda:0")),
                 lambda: A.ann_beam_select(x, Tensor(6, device="cuda:0"), 3, 3),
                 lambda: A.ann_beam_select(x, Tensor(6), 3, 3, finished=Tensor(6, torch.bool, "cuda:0")),
                 lambda: A.ann_beam_reorder(x, Tensor((2, 3), torch.int32, "cuda:0"), 3),
                 lambda: A.ann_beam_reorder(x, parents, 3, out=Tensor((6, 200), device="cuda:0"))):
        with pytest.raises(ValueError):
            call()


def test_shapes_and_types_are_refused(calls):  # noqa: F811
    x, ids, teacher, stats = Tensor((6, 200)), Tensor((6, 4), torch.int32), Tensor((6, 4)), Tensor((6, 2))
    for call in (lambda: A.OctRows(Tensor((6, 256), torch.uint8), Tensor((6, 8), torch.uint8), 200),
                 lambda: A.OctRows(Tensor((6, 256), torch.int8), Tensor((6, 4), torch.uint8), 200),
                 lambda: A.OctRows(Tensor((6, 256), torch.uint8), Tensor((5, 4), torch.uint8), 200),
                 lambda: A.ann_oct_product(A.ann_oct_quantize(x), A.ann_oct_quantize(Tensor((6, 300)))),
                 lambda: A.ann_distill(x, Tensor((5, 4), torch.int32), Tensor((5, 4))), lambda: A.ann_distill(x, ids, Tensor((6, 5))),
                 lambda: A.ann_distill(x, Tensor((6, 4), torch.int64), teacher), lambda: A.ann_distill(x, ids, teacher, losses_out=Tensor(5)),
                 lambda: A.ann_distill(x, ids, teacher, stats_out=Tensor((6, 3))), lambda: A.ann_distill_grad(x, ids, teacher, Tensor((6,))),
                 lambda: A.ann_distill_grad(x, ids, teacher, stats, out=Tensor((6, 200), torch.bfloat16)),
                 lambda: A.ann_distill_grad(x, ids, teacher, stats, grad_losses=Tensor(6, torch.float64)),
                 lambda: A.ann_beam_select(x, Tensor(6), 4, 3), lambda: A.ann_beam_select(x, Tensor(6), 0, 3), lambda: A.ann_beam_select(x, Tensor(5), 3, 3),
                 lambda: A.ann_beam_select(x, Tensor(6), 3, 3, finished=Tensor(6, torch.int32)),
                 lambda: A.ann_beam_select(x, Tensor(6), 3, 3, finished=Tensor(6, torch.bool), pad_id=200),
                 lambda: A.ann_beam_select(x, Tensor(6), 3, 3, ids_out=Tensor((2, 3), torch.int64)),
                 lambda: A.ann_beam_reorder(x, Tensor((2, 3), torch.int64), 3), lambda: A.ann_beam_reorder(x, Tensor((3, 3), torch.int32), 3),
                 lambda: A.ann_beam_reorder(x, Tensor((2, 3), torch.int32), 3, dim=2),
                 lambda: A.ann_beam_reorder(x, Tensor((2, 3), torch.int32), 3, out=Tensor((5, 200)))):
        calls.clear()
        with pytest.raises((ValueError, TypeError)):
            call()


def test_totals_are_the_next_steps_as_they_are(calls):  # noqa: F811
    x = Tensor((6, 200))
    _, _, totals = A.ann_beam_select(x, Tensor(6), 3, 3)
    A.ann_beam_select(x, totals, 3, 3, finished=Tensor((2, 3), torch.bool))
    assert [c[0] for c in calls] == ["ann_beam_select"] * 2
    for shape in ((3, 2), (6, 1), (2, 4), (2, 3, 1)):
        with pytest.raises(ValueError):
            A.ann_beam_select(x, Tensor(shape), 3, 3)
        with pytest.raises(ValueError):
            A.ann_beam_select(x, totals, 3, 3, finished=Tensor(shape, torch.bool))
