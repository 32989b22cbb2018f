"""Draws from so many long rows that a workgroup takes several of a row's chunks of 4,096 entries (some eight thousand
workgroups serve a call, so that from 8,192 / chunks rows on each has more than one)."""
import numpy as np
import pytest

from helpers import dev
from test_gpu_sample import check, scores_of, uniform

pytestmark = pytest.mark.gpu

SIZES = [(700, 70_003, "float32"),   # 18 chunks, two a workgroup
         (500, 128_000, "float16"),  # 32 chunks, two a workgroup
         (3000, 40_001, "bfloat16")]  # 10 chunks, four a workgroup
SPECIAL = 12  # rows of a kind of their own, at the front


def batch(torch, rows, n, dtype):
    rng = np.random.default_rng(rows + n)
    g = torch.Generator(device="cuda:0").manual_seed(n)
    z = 3.0 * torch.randn((rows, n), device="cuda:0", generator=g)
    z[0] = z[0].sort().values
    z[1] = z[1].sort(descending=True).values
    z[2] = 1.5
    z[3] = -float("inf")
    z[4, 5000:] = -float("inf")
    z[5, 30:] = -float("inf")
    z[6, ::2] = float("nan")
    z[7, n - 1] = float("inf")
    z[8] = torch.round(z[8])
    z[9, n // 2:n // 2 + 900] += 30.0  # good scores side by side, in two chunks
    z[10] = torch.round(4 * z[10].sort().values)
    z[11, 8190:8194] = 40.0  # on both sides of a chunk's end
    return z.to(getattr(torch, dtype)), uniform(torch, rng, rows), rng


def compare(torch, A, z, u, rng, **settings):
    """The rows of a kind of their own and some others: as the definition says, and bit for bit as in calls of fewer rows."""
    ids, logprobs = A.ann_sample(z, u, **settings)
    rows = len(z)

    def part(lo, hi):
        return {k: v[lo:hi].contiguous() if isinstance(v, torch.Tensor) else v for k, v in settings.items()}

    for lo, hi in [(i, i + 1) for i in range(SPECIAL)] + [(int(i), int(i) + 2) for i in rng.integers(SPECIAL, rows - 2, 3)] + [(rows - 1, rows)]:
        s = part(lo, hi)
        i, lp = A.ann_sample(z[lo:hi], u[lo:hi].contiguous(), **s)
        assert torch.equal(i, ids[lo:hi]) and torch.equal(lp, logprobs[lo:hi]), (lo, settings)
        assert torch.equal(check(torch, A, z[lo:hi], u[lo:hi].contiguous(), **s), i)


@pytest.mark.parametrize("rows,n,dtype", SIZES)
@pytest.mark.parametrize("rule", [dict(top_k=30), dict(top_k=200, min_p=0.002), dict(top_k=600, temperature=0.7), dict(top_k=30, top_p=0.8, min_p=0.01),
                                  dict(top_k=600, top_p=0.9), dict(top_k=2000), dict(top_p=0.9), dict(top_p=0.6, min_p=0.01, temperature=1.4),
                                  dict(min_p=0.05), {}], ids=str)
def test_rules(env, rows, n, dtype, rule):
    torch, A, _ = env
    z, u, rng = batch(torch, rows, n, dtype)
    compare(torch, A, z, u, rng, **rule)


@pytest.mark.parametrize("rows,n,dtype", SIZES)
def test_settings_of_each_row(env, rows, n, dtype):
    torch, A, _ = env
    z, u, rng = batch(torch, rows, n, dtype)
    for turn in range(3):
        t = dev(torch, rng.choice([0.0, 0.3, 1.0, 2.0], rows).astype(np.float32))
        k = dev(torch, rng.choice([0, 1, 30, 200, 600, 1025, n], rows).astype(np.int32))
        p = dev(torch, rng.choice([0.0, 0.3, 0.9, 1.0], rows).astype(np.float32))
        m = dev(torch, rng.choice([0.0, 0.001, 0.2], rows).astype(np.float32))
        compare(torch, A, z, u, rng, temperature=t, top_k=k, top_p=p, min_p=m)
        compare(torch, A, z, u, rng, temperature=t, top_k=200, top_p=p, min_p=m)
