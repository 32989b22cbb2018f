"""Exact and rounded sums of ann_mx_search: rows whose blocks have scales of their own."""
import numpy as np
import pytest

import mx_plain as P
from helpers import dev
from test_gpu_mx import check_search, rows_of

pytestmark = pytest.mark.gpu

VALUES = np.array([0.5, 1, 1.5, 2, 3, 4, 6])


def blocks(rng, n, d, spread, alike):
    """Rows of E2M1 values whose blocks of 32 have exponents 0 to `spread`, both of them met in every row, a 6 in every
    block, so that quantising keeps the values.  `alike`: every row has long runs of the largest values of one sign, with
    the smallest value once, in the block of the smallest exponent: the sums reach their largest size, and need their last bit."""
    x = rng.choice(VALUES, (n, d)) * rng.choice([-1.0, 1.0], (n, d))
    if alike:
        x[:] = 6.0
        x[:, 1] = rng.choice(VALUES, n)
        x[rng.random((n, d)) < 0.02] = 0.5
    x[:, ::32] = 6.0
    e = rng.integers(0, spread + 1, (n, (d + 31) // 32))
    if alike:
        e[:] = spread
    e[:, 0] = 0
    e[:, -1] = spread
    return x * np.exp2(np.repeat(e, 32, axis=1)[:, :d])


@pytest.mark.parametrize("alike", (False, True))
@pytest.mark.parametrize("nq", (3, 70, 300))
@pytest.mark.parametrize("d,spread", [(64, 10), (512, 7), (4096, 4), (65_536, 0)])
def test_exact_inner_products(env, d, spread, nq, alike):
    """Exponents of the products within `spread` of each other, d * 2^spread = 2^16: all sums are exact."""
    torch, A, _ = env
    rng = np.random.default_rng(d + nq)
    x, q = blocks(rng, 150, d, spread, alike), blocks(rng, nq, d, 0, alike)
    rows, queries = (A.ann_mx_quantize(dev(torch, v.astype(np.float32)), norms=True) for v in (x, q))
    assert (P.values(rows.codes.cpu().numpy(), rows.scales.cpu().numpy(), d) == x).all()
    check_search(A, torch, rows, queries, 10, False)


@pytest.mark.parametrize("alike", (False, True))
@pytest.mark.parametrize("nq", (3, 70, 300))
@pytest.mark.parametrize("d,spread", [(128, 4), (512, 3), (2048, 2), (8192, 1), (32_768, 0)])
def test_exact_squared_distances(env, d, spread, nq, alike):
    """Exponents of a row's or query's blocks within `spread` of each other, those of products within twice that:
    d * 2^(2 spread) = 2^15."""
    torch, A, _ = env
    rng = np.random.default_rng(d + nq)
    x, q = blocks(rng, 150, d, spread, alike), blocks(rng, nq, d, spread, alike)
    rows, queries = (A.ann_mx_quantize(dev(torch, v.astype(np.float32)), norms=True) for v in (x, q))
    check_search(A, torch, rows, queries, 10, True)


@pytest.mark.parametrize("l2", (True, False))
@pytest.mark.parametrize("nq", (3, 70, 300))
@pytest.mark.parametrize("n,d,spread", [(1000, 100, 12), (3000, 200, 30), (700, 500, 8), (400, 1100, 20), (200, 8000, 6)])
def test_rounded_sums(env, n, d, spread, nq, l2):
    """Scales far apart: a sum of d products is off by at most d + 3 half steps of the sum of their magnitudes (and of the
    norms'), the distance by one more.  No row that is nearer by more than that is left out."""
    torch, A, _ = env
    rng = np.random.default_rng(n + d + nq)
    far = np.exp2(rng.integers(-spread // 2, spread // 2 + 1, (1, d)).astype(np.float64))
    made = []
    for rows in (n, nq):
        v = rng.standard_normal((rows, d)) * far * np.exp2(rng.integers(-2, 3, (rows, 1)))
        made.append(A.ann_mx_quantize(dev(torch, v.astype(np.float32)), norms=True))
    x, q = (P.values(r.codes.cpu().numpy(), r.scales.cpu().numpy(), d) for r in made)
    k = 20
    ids, dists = A.ann_mx_search(made[0], made[1], k, metric=A.L2SQ if l2 else A.MIPS)
    ids, dists = ids.cpu().numpy(), dists.cpu().numpy().astype(np.float64)
    want = -(q @ x.T)
    size = np.abs(q) @ np.abs(x).T
    if l2:
        qq, xx = (q ** 2).sum(1)[:, None], (x ** 2).sum(1)[None, :]
        want = np.maximum(qq + xx + 2 * want, 0.0)
        size = qq + xx + 2 * size
    off = (d + 4) * 2.0 ** -24 * size
    at = np.arange(nq)[:, None]
    assert (np.sort(ids, axis=1)[:, 1:] != np.sort(ids, axis=1)[:, :-1]).all() and (ids >= 0).all() and (ids < n).all()
    assert (np.abs(dists - want[at, ids]) <= off[at, ids]).all()
    assert (np.diff(dists, axis=1) >= 0).all()
    # a row that was left out is not nearer than the last one by more than both sums may be off
    out = np.ones((nq, n), bool)
    out[at, ids] = False
    assert (want + off >= dists[:, -1:])[out].all()
    again = A.ann_mx_search(made[0], made[1], k, metric=A.L2SQ if l2 else A.MIPS)
    assert (again[0].cpu().numpy() == ids).all()
