"""The device that the calls on 4-bit rows and ann_sample run on: that of their tensors, whichever is current (no GPU
needed: tensors, the device and the library are stand-ins that record what the binding asks for)."""
import pytest
import torch

from paper_2305_04359_amd import binding as A


class Tensor:
    """What the binding looks at of a contiguous device tensor."""
    is_cuda = True

    def __init__(self, shape, dtype=torch.float32, device="cuda:1"):
        self.shape = torch.Size((shape,) if isinstance(shape, int) else shape)
        self.dtype, self.device = dtype, torch.device(device)

    def dim(self):
        return len(self.shape)

    def stride(self):
        return tuple(self.shape[i + 1:].numel() for i in range(self.dim()))

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 20

    def numel(self):
        return self.shape.numel()

    def element_size(self):
        return self.dtype.itemsize


class Calls(list):
    """(name, current device, stream) of the calls into the library, which return `rc`."""
    rc = 0


@pytest.fixture
def calls(monkeypatch):
    """Device 0 is current outside of the calls."""
    made, now = Calls(), [0]

    class Device:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            self.before, now[0] = now[0], self.index

        def __exit__(self, *exc):
            now[0] = self.before

    class Library:
        def __getattr__(self, name):
            def call(*args):
                if name.endswith("_scratch"):
                    args[-1]._obj.value = 64
                else:
                    made.append((name, now[0], args[-1]))
                    return made.rc
                return 0
            return call

    monkeypatch.setattr(A, "lib", Library)
    monkeypatch.setattr(A, "_raw_stream", lambda index: 1000 + index)
    monkeypatch.setattr(A, "_current_device", lambda: now[0], raising=False)
    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(torch, "empty", lambda shape, dtype, device: Tensor(shape, dtype, device))
    yield made
    assert now == [0]


def all_calls(device):
    x = Tensor((5, 200), device=device)
    rows = A.ann_mx_quantize(x, norms=True)
    A.ann_mx_dequantize(rows)
    A.ann_mx_product(x, rows)
    A.ann_mx_product(rows, rows)
    A.ann_mx_search(rows, rows, 3)
    A.ann_sample(x, Tensor(5, device=device))


NAMES = ["ann_mx_quantize", "ann_mx_dequantize", "ann_mx_product", "ann_mx_product_mx", "ann_mx_search", "ann_sample"]


def test_calls_run_on_the_device_of_their_tensors(calls):
    for index in (1, 0):
        calls.clear()
        all_calls(f"cuda:{index}")
        assert calls == [(name, index, 1000 + index) for name in NAMES]


def test_the_device_comes_back_after_a_refusal(monkeypatch, calls):
    def refuse(rc):
        raise A.AnnError(rc, "refused")

    monkeypatch.setattr(A, "_check", refuse)
    calls.rc = -1
    with pytest.raises(A.AnnError):
        A.ann_mx_quantize(Tensor((5, 200)))
    assert [c[1] for c in calls] == [1]
