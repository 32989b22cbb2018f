"""ann_sample against its definition in 64 bits."""
import numpy as np
import pytest

import mx_plain as P
from helpers import dev

pytestmark = pytest.mark.gpu


def check(torch, A, scores, u, **settings):
    """Ids equal; log-probabilities within their rounding to fp32 and the sums' own (n terms in fp64)."""
    ids, logprobs = A.ann_sample(scores, u, **settings)
    z, uh = scores.double().cpu().numpy(), u.double().cpu().numpy()
    rows = len(z)
    per = {k: v.double().cpu().numpy() if isinstance(v, torch.Tensor) else np.full(rows, np.float32(v), np.float64) for k, v in settings.items()}
    for r in range(rows):
        s = {k: (int(v[r]) if k == "top_k" else float(v[r])) for k, v in per.items()}
        i, lp = P.draw(np.where(np.isnan(z[r]), -np.inf, z[r]), uh[r], **s)
        assert int(ids[r]) == i, (r, s, i, int(ids[r]))
        got = float(logprobs[r])
        assert got == lp or abs(got - lp) <= 2.0 ** -24 * abs(lp) + 1e-12 + 2.0 ** -149, (r, s, lp, got)
    return ids


def scores_of(torch, rng, rows, n, dtype, masked=0.0):
    z = 3.0 * rng.standard_normal((rows, n))
    z[rng.random((rows, n)) < masked] = -np.inf
    return dev(torch, z).to(getattr(torch, dtype))


def uniform(torch, rng, rows):
    return dev(torch, rng.random(rows).astype(np.float32) * np.float32(1 - 2.0 ** -24))


RULES = ({}, dict(temperature=0.7), dict(temperature=1.5, top_k=1), dict(top_k=50), dict(top_p=0.9, temperature=0.8), dict(min_p=0.05),
         dict(top_k=40, top_p=0.8, min_p=0.02, temperature=1.3), dict(temperature=0.0), dict(top_k=10 ** 9, top_p=0.999999), dict(top_p=1e-6),
         dict(min_p=1.0), dict(min_p=5.0), dict(temperature=1e-30), dict(temperature=float("inf"), top_p=0.5), dict(temperature=float("nan")))


@pytest.mark.parametrize("dtype", ("float32", "float16", "bfloat16"))
@pytest.mark.parametrize("rows,n", [(1, 1), (2, 2), (5, 63), (3, 64), (7, 1000), (4, 1025), (2, 5003), (1, 40_000), (130, 257)])
def test_rules(env, dtype, rows, n):
    torch, A, _ = env
    rng = np.random.default_rng(rows * n)
    for i, rule in enumerate(RULES):
        z = scores_of(torch, rng, rows, n, dtype, masked=(0.0, 0.3, 0.97)[i % 3])
        check(torch, A, z, uniform(torch, rng, rows), **rule)


@pytest.mark.parametrize("rows,n", [(1, 128_000), (3, 200_003)])
def test_long_rows(env, rows, n):
    torch, A, _ = env
    rng = np.random.default_rng(n)
    for dtype, rule in (("float32", {}), ("bfloat16", dict(top_p=0.95)), ("float16", dict(top_k=64, min_p=0.01)), ("float32", dict(top_p=0.5, temperature=2.0))):
        check(torch, A, scores_of(torch, rng, rows, n, dtype), uniform(torch, rng, rows), **rule)


@pytest.mark.parametrize("dtype", ("float32", "float16", "bfloat16"))
@pytest.mark.parametrize("rows,n", [(1, 16_384), (3, 16_383), (5, 20_001), (2, 70_003), (1, 1_100_000)])
def test_rules_on_long_rows(env, dtype, rows, n):
    """Rows that several workgroups share, and just shorter ones."""
    torch, A, _ = env
    rng = np.random.default_rng(rows * n)
    for i, rule in enumerate(RULES + (dict(top_k=2000), dict(top_k=900, top_p=0.7), dict(top_k=5000, min_p=0.001), dict(top_k=3000, top_p=0.5))):
        if n > 10 ** 6 and i % 3:
            continue
        z = scores_of(torch, rng, rows, n, dtype, masked=(0.0, 0.3, 0.97)[i % 3])
        check(torch, A, z, uniform(torch, rng, rows), **rule)


def test_settings_of_each_long_row(env):
    torch, A, _ = env
    rng = np.random.default_rng(15)
    rows, n = 60, 17_001
    t = dev(torch, rng.choice([0.0, 0.3, 1.0, 2.0, -1.0], rows).astype(np.float32))
    k = dev(torch, rng.choice([0, 1, 7, 500, 1024, 1025, 17_000, 100_000], rows).astype(np.int32))
    p = dev(torch, rng.choice([0.0, 0.2, 0.9, 1.0, 2.0], rows).astype(np.float32))
    m = dev(torch, rng.choice([0.0, 0.001, 0.2, 1.0], rows).astype(np.float32))
    for dtype in ("float32", "bfloat16"):
        z = scores_of(torch, rng, rows, n, dtype, 0.1)
        z[3] = -float("inf")
        z[4, 100:] = -float("inf")
        z[5] = 2.0
        z[6, ::3] = 5.0
        z[7, 1000] = float("inf")
        z[8, ::2] = float("nan")
        check(torch, A, z, uniform(torch, rng, rows), temperature=t, top_k=k, top_p=p, min_p=m)
        # equal scores around every cut
        z = torch.round(scores_of(torch, rng, rows, n, dtype)).to(z.dtype)
        check(torch, A, z, uniform(torch, rng, rows), temperature=t, top_k=k, top_p=p, min_p=m)


@pytest.mark.parametrize("rows,n", [(9, 1024), (9, 1025), (5, 4096), (5, 4097), (300, 33), (5000, 5), (4097, 4500)])
def test_sizes_at_which_rows_are_dealt_otherwise(env, rows, n):
    torch, A, _ = env
    rng = np.random.default_rng(rows + n)
    for i, rule in enumerate((dict(top_k=n // 3 + 1, top_p=0.9), dict(top_p=0.7), dict(min_p=0.1, temperature=0.5))):
        z = scores_of(torch, rng, rows, n, ("float32", "bfloat16", "float16")[i], 0.1)
        u = uniform(torch, rng, rows)
        if rows * n < 10 ** 6:
            check(torch, A, z, u, **rule)
        else:  # the last rows against a call of their own
            ids, logprobs = A.ann_sample(z, u, **rule)
            check(torch, A, z[-5:], u[-5:].contiguous(), **rule)
            check(torch, A, z[4090:4096], u[4090:4096].contiguous(), **rule)
            for lo in (0, 4000, rows - 50):
                i2, lp2 = A.ann_sample(z[lo:lo + 50], u[lo:lo + 50].contiguous(), **rule)
                assert torch.equal(i2, ids[lo:lo + 50]) and torch.equal(lp2, logprobs[lo:lo + 50])


def test_many_candidates_around_the_cut(env):
    """Long rows whose scores lie close together, and rows of few different scores."""
    torch, A, _ = env
    rng = np.random.default_rng(17)
    n = 300_000
    close = dev(torch, rng.standard_normal((3, n)).astype(np.float32) * 0.05)
    steps = dev(torch, rng.integers(0, 40, (3, n)).astype(np.float32) / 8)
    for rule in (dict(top_p=0.6), dict(top_k=70_000), dict(top_k=1000), dict(top_k=70_000, top_p=0.5), dict(top_p=0.999, min_p=0.9), {}):
        for z in (close, close.bfloat16(), steps, steps.half()):
            check(torch, A, z, uniform(torch, rng, 3), **rule)


def test_long_lists_of_equal_scores(env):
    """Some three thousand equal candidates at the cut, of which some are kept: they are told apart by their ids alone."""
    torch, A, _ = env
    rng = np.random.default_rng(23)
    z = dev(torch, rng.integers(0, 100, (4, 300_007)).astype(np.float32))
    for rule in (dict(top_p=0.9), dict(top_p=0.9, temperature=2.0), dict(top_p=0.3, temperature=8.0), dict(top_p=0.97, temperature=8.0, min_p=1e-4),
                 dict(top_k=4500), dict(top_k=100_000)):
        for scores in (z, -z, z.bfloat16()):
            check(torch, A, scores, uniform(torch, rng, 4), **rule)


@pytest.mark.parametrize("dtype", ("float32", "bfloat16"))
@pytest.mark.parametrize("n", (5000, 50_001, 300_007))
def test_top_k_of_rows_in_any_order(env, dtype, n):
    """Good scores side by side, few or no candidates, as many kept as there are parts of a row: one top-k for all rows, and
    one for each."""
    torch, A, _ = env
    rng = np.random.default_rng(n)
    z = 3.0 * rng.standard_normal((9, n))
    z[0].sort()
    z[1] = -np.sort(-z[1])
    z[2, 4096:] = -np.inf
    z[3, 30:] = -np.inf
    z[4] = -np.inf
    z[5] = np.round(z[5])
    z[6, :] = 1.5
    z[7, n // 2:n // 2 + 700] += 30.0
    z[8, ::7] = np.nan
    scores = dev(torch, z).to(getattr(torch, dtype))
    u = uniform(torch, rng, 9)
    for k in (1, 7, 16, 40, 64, 65, 160, 400, 512, 513, 1100):
        for more in ({}, dict(top_p=0.8, min_p=0.01)):
            check(torch, A, scores, u, top_k=k, temperature=0.9, **more)
    each = torch.tensor([3, 16, 0, 70, 12, 31, 512, 90, 1], dtype=torch.int32, device="cuda:0")
    for shift in range(9):
        check(torch, A, scores, u, top_k=each.roll(shift).contiguous(), top_p=0.9)


def test_draws_do_not_depend_on_the_other_rows(env):
    torch, A, _ = env
    rng = np.random.default_rng(16)
    z, u = scores_of(torch, rng, 700, 20_000, "bfloat16"), uniform(torch, rng, 700)
    for rule in ({}, dict(top_p=0.8), dict(top_k=30), dict(min_p=0.02)):
        ids, logprobs = A.ann_sample(z, u, **rule)
        for lo, hi in ((0, 1), (3, 5), (100, 400)):
            i, lp = A.ann_sample(z[lo:hi], u[lo:hi].contiguous(), **rule)
            assert torch.equal(i, ids[lo:hi]) and torch.equal(lp, logprobs[lo:hi])


def test_settings_of_each_row(env):
    torch, A, _ = env
    rng = np.random.default_rng(5)
    rows, n = 60, 3001
    t = dev(torch, rng.choice([0.0, 0.3, 1.0, 2.0, -1.0], rows).astype(np.float32))
    k = dev(torch, rng.choice([0, 1, 7, 500, 3001, 10_000], rows).astype(np.int32))
    p = dev(torch, rng.choice([0.0, 0.2, 0.9, 1.0, 2.0], rows).astype(np.float32))
    m = dev(torch, rng.choice([0.0, 0.001, 0.2, 1.0], rows).astype(np.float32))
    for dtype in ("float32", "bfloat16"):
        check(torch, A, scores_of(torch, rng, rows, n, dtype, 0.1), uniform(torch, rng, rows), temperature=t, top_k=k, top_p=p, min_p=m)


def test_equal_scores(env):
    torch, A, _ = env
    rng = np.random.default_rng(6)
    for n in (3, 64, 1024, 5000):
        z = dev(torch, rng.integers(0, 3, (20, n)).astype(np.float32))
        for rule in ({}, dict(top_k=n // 3 + 1), dict(top_p=0.5), dict(top_p=0.25, top_k=n // 2 + 1), dict(min_p=0.9)):
            check(torch, A, z, uniform(torch, rng, 20), **rule)
        check(torch, A, torch.zeros((20, n), device="cuda:0"), uniform(torch, rng, 20), top_p=0.75, top_k=n - 1)


def test_masks_infinities_and_nan(env):
    torch, A, _ = env
    rng = np.random.default_rng(7)
    inf, low = float("inf"), float(np.finfo(np.float32).min)
    z = 2.0 * rng.standard_normal((16, 1500)).astype(np.float32)
    z[0] = -inf                      # nothing to draw from
    z[1] = np.nan
    z[2, 5:] = -inf
    z[3] = low                       # the type's lowest value masks nothing when it is all there is
    z[4, 100:] = low
    z[5, [7, 900]] = inf             # infinite scores share the draw
    z[6, 3] = inf
    z[7, ::2] = np.nan
    z[8, 1:] = np.nan
    z[9, :] = -inf
    z[9, 1499] = -3.0
    z[10, 0] = 88.0                  # one candidate takes nearly all the mass
    z[11] = -0.0
    z[11, 700:] = 0.0                # zeros of either sign are equal
    z[12] *= 1e-42                   # subnormal scores
    z[13, 20] = 3.4e38
    z[13, 21] = -3.4e38
    z[14, :700] = 1e30
    z[15] = np.where(rng.random(1500) < 0.5, np.nan, -inf)
    for rule in RULES:
        for dtype in (torch.float32, torch.bfloat16, torch.float16):
            ids = check(torch, A, dev(torch, z).to(dtype), uniform(torch, rng, 16), **rule)
            assert ids[0] == -1 and ids[1] == -1 and ids[15] == -1


def test_ends_of_the_unit_interval(env):
    torch, A, _ = env
    rng = np.random.default_rng(8)
    z = scores_of(torch, rng, 6, 2000, "float32", 0.5)
    z[:, 0] = -float("inf")
    z[:, 1999] = -200.0  # a weight that rounding loses in the sum
    for v in (0.0, 1.0 - 2.0 ** -24, 1.0, 7.0, -3.0):
        for rule in ({}, dict(top_k=3), dict(top_p=0.5)):
            check(torch, A, z, torch.full((6,), v, device="cuda:0"), **rule)


def test_rows_with_a_stride(env):
    torch, A, _ = env
    rng = np.random.default_rng(9)
    for dtype, pad, at in (("float32", 3, 1), ("bfloat16", 8, 0), ("float16", 1, 1)):
        wide = scores_of(torch, rng, 9, 1001 + pad, dtype)
        u = uniform(torch, rng, 9)
        wide[:, :at] = 1e4
        wide[:, at + 1001:] = float("nan")
        check(torch, A, wide[:, at:at + 1001], u, top_p=0.9)
        check(torch, A, wide[:, at:at + 1001], u, top_k=5)


def test_frequencies(env):
    """A hundred thousand draws from one row: counts within five standard deviations of the probabilities."""
    torch, A, _ = env
    n = 100_000
    z = torch.tensor([1.0, 0.0, -1.0, 2.0, -float("inf"), 0.5], device="cuda:0")
    ids, logprobs = A.ann_sample(z.repeat(n, 1), torch.rand(n, device="cuda:0", generator=torch.Generator(device="cuda:0").manual_seed(3)))
    p = torch.softmax(z.double(), 0).cpu().numpy()
    c = torch.bincount(ids, minlength=6).cpu().numpy()
    assert (np.abs(c - n * p) <= 5 * np.sqrt(n * p * (1 - p)) + 1e-9).all()
    assert torch.allclose(logprobs.double(), torch.log_softmax(z.double(), 0)[ids], atol=1e-6)


def test_scores_beyond_32_bits(env):
    """Rows that start more than 4 GiB into the scores."""
    torch, A, _ = env
    rows, n = 17_000, 131_073
    z = torch.zeros((rows, n), dtype=torch.float16, device="cuda:0")
    tail = scores_of(torch, np.random.default_rng(1), 8, n, "float16")
    z[-8:] = tail
    u = torch.rand(rows, device="cuda:0")
    ids, logprobs = A.ann_sample(z, u, top_p=0.9)
    i, lp = A.ann_sample(tail, u[-8:].contiguous(), top_p=0.9)
    assert torch.equal(ids[-8:], i) and torch.equal(logprobs[-8:], lp)
