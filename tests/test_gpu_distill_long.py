"""Sums of ann_distill over very long rows."""
import math

import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24  # half a step of fp32


@pytest.mark.parametrize("rows", (520, 500))  # rows by a workgroup each; rows in two parts
def test_sums_of_thousands_of_equal_weights(env, rows):
    """A thread adds 8,192 and 16,384 weights that are all alike, so that roundings of a running fp32 sum would all go one
    way.  A weight: its argument a <= 2 is rounded three times (3 U a), exp2 is off by a step (2 U), all of it times its ln 2 and
    less: 10 U.  Thirty-two of them one after another 31 U, the sums of these added so that what is lost is kept 3 U,
    14 joins with an exp2 and a product each 70 U: 114 U of the sum.  The loss of an only entry, one of the row's largest, is its
    logarithm, rounded once."""
    torch, A, _ = env
    n = 1 << 22
    below = [0.25, 0.5, 0.75, 1.0, 1.25, 1.5, 2.0]
    z = torch.empty((rows, n), dtype=torch.float16, device="cuda")
    for r in range(rows):
        z[r] = -below[r % len(below)]
    z[:, :8192] = 0.0  # every thread's largest score, at its beginning
    z[:, n // 2:n // 2 + 8192] = 0.0
    ids = torch.full((rows, 1), 8000, dtype=torch.int32, device="cuda")
    losses, stats = A.ann_distill(z, ids, torch.zeros((rows, 1), device="cuda"))
    want = torch.tensor([16_384 + (n - 16_384) * math.exp(-below[r % len(below)]) for r in range(rows)], dtype=torch.float64)
    assert (stats[:, 0] == 0).all()
    assert ((stats[:, 1].double().cpu() - want).abs() <= 114 * U * want).all(), ((stats[:, 1].double().cpu() - want).abs() / want).max()
    assert ((losses.double().cpu() - want.log()).abs() <= 115 * U + U * want.log()).all()
