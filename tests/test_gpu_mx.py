"""The calls on microscaled 4-bit rows against their definitions in 64 bits."""
import numpy as np
import pytest

import mx_plain as P
from helpers import dev

pytestmark = pytest.mark.gpu

TYPES = ("uint8", "int8", "float32", "float16", "bfloat16")
OUT = ("float32", "float16", "bfloat16")
HALF_STEP = {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}


def rows_of(torch, rng, n, d, dtype, pad=0, spread=1):
    """(device tensor of n rows, possibly a slice of wider ones; the same in float64).  `spread`: exponents of the rows differ."""
    if dtype == "uint8":
        x = rng.integers(0, 256, (n, d + pad))
    elif dtype == "int8":
        x = rng.integers(-128, 128, (n, d + pad))
    else:
        x = rng.standard_normal((n, d + pad)) * 2.0 ** rng.integers(-spread, spread + 1, (n, 1))
    t = torch.from_numpy(np.ascontiguousarray(x)).to("cuda:0").to(getattr(torch, dtype))[:, pad // 2:pad // 2 + d]
    return t, t.double().cpu().numpy()


def packed(A, torch, codes, scales, d, norms=None):
    return A.MxRows(dev(torch, codes), dev(torch, scales), d, norms)


def check_quantized(A, torch, t, x):
    r = A.ann_mx_quantize(t, norms=True)
    codes, scales = P.quantize(x)
    assert (r.scales.cpu().numpy() == scales).all()
    assert (r.codes.cpu().numpy() == codes).all()
    v = P.values(codes, scales, x.shape[1])
    norms = (v ** 2).sum(1)
    got = r.norms.cpu().numpy().astype(np.float64)
    fine = np.isfinite(norms)
    assert (np.isnan(got) == np.isnan(norms)).all()
    # eight squares of a lane are exact; then one addition per 512 elements, and six across the lanes; sums beyond
    # the range of fp32 are infinite, and its smallest step is 2^-149
    over = norms >= 2.0 ** 128
    assert (got[fine & over] == np.inf).all()
    fine &= ~over
    assert (np.abs(got - norms)[fine] <= (x.shape[1] / 512 + 8) * (2.0 ** -24 * norms[fine] + 2.0 ** -149)).all()
    for dtype in OUT:
        want = torch.from_numpy(v).float().to(getattr(torch, dtype))
        back = A.ann_mx_dequantize(r, dtype=getattr(torch, dtype)).cpu()
        assert torch.equal(back.isnan(), want.isnan()) and torch.equal(back.nan_to_num(7.0), want.nan_to_num(7.0)), dtype
    return r


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,d,pad", [(1, 1, 0), (3, 31, 0), (5, 32, 0), (7, 33, 3), (37, 100, 0), (9, 127, 1), (16, 128, 0), (11, 129, 0), (37, 200, 8),
                                     (4, 511, 0), (3, 1000, 0), (2, 4097, 5), (513, 128, 16), (0, 100, 0)])
def test_quantize(env, dtype, n, d, pad):
    torch, A, _ = env
    t, x = rows_of(torch, np.random.default_rng(n * d + pad), n, d, dtype, pad)
    check_quantized(A, torch, t, x)


def test_quantize_ties_and_extremes(env):
    torch, A, _ = env
    # every boundary between levels and its neighbours, at several scales; signs; zeros; the ends of the range
    mids = np.array([0.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 7.999], np.float32)
    near = np.concatenate([mids, np.nextafter(mids, np.float32(100)), np.nextafter(mids, np.float32(-100))])[:31]
    rows = []
    for e in (-149, -148, -140, -130, -127, -126, -125, -124, -30, 0, 30, 100, 125):
        with np.errstate(over="ignore"):
            block = np.float32(np.concatenate([[7.5], near]).astype(np.float64) * 2.0 ** e)
        block[~np.isfinite(block)] = np.float32(3e38)
        rows += [block, -block]
    rows += [np.zeros(32, np.float32), np.full(32, -0.0, np.float32), np.full(32, 1e-45, np.float32), np.full(32, 3.4028235e38, np.float32)]
    for bad in (np.nan, np.inf, -np.inf):
        row = np.ones(32, np.float32)
        row[17] = bad
        rows.append(row)
    x = np.stack(rows)
    check_quantized(A, torch, dev(torch, x), x.astype(np.float64))
    # the same blocks next to each other in longer rows: a bad block spoils itself only
    wide = np.concatenate([x, x[::-1], np.roll(x, 3, axis=0)], axis=1)
    check_quantized(A, torch, dev(torch, wide), wide.astype(np.float64))


def check_product(A, torch, x, w, got, xv, wv, extra=0.0):
    """Sums of d products in fp32, in any order: each is off by at most d + 2 half steps of the sum of the products'
    magnitudes; then one rounding."""
    want = xv @ wv.T
    most = (xv.shape[1] + 2) * 2.0 ** -24 * (np.abs(xv) @ np.abs(wv).T)
    dtype = str(got.dtype).split(".")[1]
    least = 2.0 ** -25 if dtype == "float16" else 2.0 ** -140
    off = np.abs(got.double().cpu().numpy() - want)
    limit = most + HALF_STEP[dtype] * (np.abs(want) + most) + least
    assert (off <= limit).all(), (off / limit).max()


@pytest.mark.parametrize("dtype", ("float32", "float16", "bfloat16"))
@pytest.mark.parametrize("nx,n,d,pad,out", [(1, 1, 1, 0, "float32"), (1, 1000, 128, 0, "float32"), (1, 77, 4096, 0, "bfloat16"), (2, 65, 33, 3, "float16"),
                                            (5, 300, 100, 0, "float32"), (15, 129, 257, 1, "bfloat16"), (16, 4096, 200, 0, "float32"), (17, 130, 640, 8, "float16"),
                                            (33, 1001, 200, 5, "float32"), (64, 64, 128, 0, "float16"), (100, 257, 1000, 0, "bfloat16"),
                                            (130, 260, 96, 0, "float32"), (257, 513, 384, 0, "bfloat16"), (300, 15, 2048, 0, "float32")])
def test_product(env, dtype, nx, n, d, pad, out):
    torch, A, _ = env
    rng = np.random.default_rng(nx * n + d)
    t, x = rows_of(torch, rng, nx, d, dtype, pad)
    w = A.ann_mx_quantize(rows_of(torch, rng, n, d, "float32", spread=4)[0])
    wv = P.values(w.codes.cpu().numpy(), w.scales.cpu().numpy(), d)
    check_product(A, torch, t, w, A.ann_mx_product(t, w, dtype=getattr(torch, out)), x, wv)


@pytest.mark.parametrize("nx,n,d,out", [(1, 1, 1, "float32"), (1, 1000, 128, "float32"), (3, 77, 4096, "bfloat16"), (16, 65, 33, "float16"), (37, 300, 100, "float32"),
                                        (64, 129, 257, "bfloat16"), (65, 4096, 200, "float32"), (130, 260, 640, "float16"), (257, 515, 1100, "float32"),
                                        (1000, 64, 128, "bfloat16"), (300, 15, 2048, "float32")])
def test_product_of_packed_rows(env, nx, n, d, out):
    torch, A, _ = env
    rng = np.random.default_rng(nx * n + d)
    x = A.ann_mx_quantize(rows_of(torch, rng, nx, d, "bfloat16", spread=3)[0])
    w = A.ann_mx_quantize(rows_of(torch, rng, n, d, "float32", spread=4)[0])
    xv, wv = (P.values(r.codes.cpu().numpy(), r.scales.cpu().numpy(), d) for r in (x, w))
    check_product(A, torch, x, w, A.ann_mx_product(x, w, dtype=getattr(torch, out)), xv, wv)


@pytest.mark.parametrize("dtype", ("float32", "float16", "bfloat16", "mx"))
@pytest.mark.parametrize("nx,n,d,pad,out", [(8, 1, 1024, 0, "float32"), (16, 33, 1025, 0, "bfloat16"), (31, 500, 1100, 4, "float16"), (48, 100, 4096, 0, "float32"),
                                            (65, 31, 2047, 1, "bfloat16"), (300, 129, 1536, 8, "float32"), (520, 64, 1152, 0, "float16")])
def test_product_of_few_long_rows(env, dtype, nx, n, d, pad, out):
    torch, A, _ = env
    rng = np.random.default_rng(nx * n + d)
    t, x = rows_of(torch, rng, nx, d, "bfloat16" if dtype == "mx" else dtype, pad)
    w = A.ann_mx_quantize(rows_of(torch, rng, n, d, "float32", spread=4)[0])
    wv = P.values(w.codes.cpu().numpy(), w.scales.cpu().numpy(), d)
    if dtype == "mx":
        t = A.ann_mx_quantize(t)
        x = P.values(t.codes.cpu().numpy(), t.scales.cpu().numpy(), d)
    got = A.ann_mx_product(t, w, dtype=getattr(torch, out))
    check_product(A, torch, t, w, got, x, wv)
    assert torch.equal(got, A.ann_mx_product(t, w, dtype=getattr(torch, out)))


@pytest.mark.parametrize("dtype", ("uint8", "float16", "bfloat16", "float32"))
@pytest.mark.parametrize("n,d,ld,at", [(9, 31, 31, 0), (50, 33, 35, 1), (3, 8, 9, 1), (21, 333, 337, 3), (1, 129, 131, 1)])
def test_rows_that_begin_anywhere(env, dtype, n, d, ld, at):
    """Rows at every alignment that their elements allow, read and written as they are elsewhere."""
    torch, A, _ = env
    rng = np.random.default_rng(n * d)
    t = rows_of(torch, rng, n, d, dtype)[0]
    wide = torch.zeros((n, ld), dtype=t.dtype, device=t.device)
    wide[:, at:at + d] = t
    r, s = A.ann_mx_quantize(t, norms=True), A.ann_mx_quantize(wide[:, at:at + d], norms=True)
    for a, b in ((r.codes, s.codes), (r.scales, s.scales), (r.norms, s.norms)):
        assert torch.equal(a, b)
    if dtype != "uint8":
        back = torch.full((n, ld), -7.0, dtype=t.dtype, device=t.device)
        A.ann_mx_dequantize(r, out=back[:, at:at + d])
        assert torch.equal(back[:, at:at + d], A.ann_mx_dequantize(r, dtype=t.dtype))
        assert (back[:, :at] == -7.0).all() and (back[:, at + d:] == -7.0).all()


def test_product_takes_blocks_apart(env):
    """Every element and every block's scale counts where it belongs: one at a time, exact."""
    torch, A, _ = env
    d = 300
    x = np.eye(d, dtype=np.float32) * np.float32(3.0)
    w = np.zeros((d, d), np.float32)
    w[np.arange(d), np.arange(d)] = np.float32(2.0) ** (np.arange(d) % 40 - 20)
    w[:, 5] += np.float32(0.5)
    for t in (dev(torch, x), dev(torch, x).bfloat16(), dev(torch, x).half(), A.ann_mx_quantize(dev(torch, x))):
        r = A.ann_mx_quantize(dev(torch, w))
        wv = P.values(r.codes.cpu().numpy(), r.scales.cpu().numpy(), d)
        got = A.ann_mx_product(t, r).cpu().numpy()
        assert (got == 3.0 * wv.T).all()


def test_product_extreme_scales_and_values(env):
    torch, A, _ = env
    d, n = 160, 20
    rng = np.random.default_rng(3)
    w = rng.standard_normal((n, d)) * np.exp2(rng.integers(-120, 100, (n, 1)).astype(np.float64))
    w[3] = 0.0
    r = A.ann_mx_quantize(dev(torch, w.astype(np.float32)))
    wv = P.values(r.codes.cpu().numpy(), r.scales.cpu().numpy(), d)
    x = rng.standard_normal((17, d)).astype(np.float32)
    x[5] *= np.float32(1e-20)
    x[6, :] = 0.0
    x[7] *= np.float32(2.0) ** 100  # products with the large rows leave the range of fp32, to both sides
    got = A.ann_mx_product(dev(torch, x), r).double().cpu().numpy()
    want, most = x.astype(np.float64) @ wv.T, np.abs(x.astype(np.float64)) @ np.abs(wv).T
    safe = most < 2.0 ** 127
    # (parts of a float below 2^-126 are lost: at most 2^-126 of each factor)
    limit = (d + 2) * 2.0 ** -23 * most + 2.0 ** -126 * np.abs(wv).sum(1)[None, :] + 2.0 ** -126 * d
    assert (np.abs(got - want) <= limit)[safe].all()
    assert not np.isfinite(got[np.abs(want) > 2.0 ** 129]).any()
    # a NaN or infinity in x spoils its row only, a NaN block of the 4-bit rows its column only
    x = rng.standard_normal((20, d)).astype(np.float32)
    x[2, 159], x[9, 0], x[11, 31] = np.nan, np.inf, -np.inf
    w = (rng.integers(1, 5, (n, d)) * rng.choice([-1.0, 1.0], (n, d))).astype(np.float32)
    w[4, 70] = np.nan
    r = A.ann_mx_quantize(dev(torch, w))
    for t in (dev(torch, x), dev(torch, x).half(), dev(torch, x).bfloat16()):
        got = A.ann_mx_product(t, r).cpu().numpy()
        assert np.isnan(got[:, 4]).all() and np.isnan(got[2]).all()
        other = np.arange(n) != 4
        assert (np.isinf(got[9, other]) | np.isnan(got[9, other])).all() and (got[9, other] == np.sign(w[other, 0]) * np.inf).all()
        assert (got[11, other] == -np.sign(w[other, 31]) * np.inf).all()
        rest = np.isin(np.arange(20), (2, 9, 11), invert=True)
        assert np.isfinite(got[np.ix_(rest, other)]).all()
    q = A.ann_mx_quantize(dev(torch, x))
    got = A.ann_mx_product(q, r).cpu().numpy()
    bad = np.isin(np.arange(20), (2, 9, 11))
    assert np.isnan(got[bad]).all() and np.isnan(got[:, 4]).all() and np.isfinite(got[np.ix_(~bad, other)]).all()


def test_product_ends_of_rows_are_not_read_as_values(env):
    """What lies past d in a wider row of x does not enter, NaN or not."""
    torch, A, _ = env
    x = torch.full((5, 140), float("nan"), device="cuda:0")
    x[:, :100] = 1.0
    r = A.ann_mx_quantize(torch.ones((9, 100), device="cuda:0"))
    assert (A.ann_mx_product(x[:, :100], r) == 100.0).all()
    assert (A.ann_mx_dequantize(A.ann_mx_quantize(x[:, :100])) == 1.0).all()


def test_product_writes_into_wider_rows(env):
    torch, A, _ = env
    rng = np.random.default_rng(9)
    r = A.ann_mx_quantize(rows_of(torch, rng, 130, 64, "float32")[0])
    x = rows_of(torch, rng, 19, 64, "float32")[0]
    for dtype, pad, at in ((torch.float32, 4, 0), (torch.bfloat16, 3, 1), (torch.float16, 6, 2)):
        wide = torch.full((19, 130 + pad), -7.0, dtype=dtype, device="cuda:0")
        A.ann_mx_product(x, r, out=wide[:, at:at + 130])
        assert torch.equal(wide[:, at:at + 130], A.ann_mx_product(x, r, dtype=dtype))
        assert (wide[:, :at] == -7.0).all() and (wide[:, at + 130:] == -7.0).all()
        back = torch.full((130, 64 + pad), -7.0, dtype=dtype, device="cuda:0")
        A.ann_mx_dequantize(r, out=back[:, at:at + 64])
        assert torch.equal(back[:, at:at + 64], A.ann_mx_dequantize(r, dtype=dtype))
        assert (back[:, :at] == -7.0).all() and (back[:, at + 64:] == -7.0).all()


def check_search(A, torch, rows, queries, k, l2):
    """Exact sums: ids equal, distances equal after one rounding."""
    rv, qv = (P.values(r.codes.cpu().numpy(), r.scales.cpu().numpy(), r.d) for r in (rows, queries))
    ids, dists = A.ann_mx_search(rows, queries, k, metric=A.L2SQ if l2 else A.MIPS)
    want_i, want_d = P.nearest(rv, qv, k, l2)
    assert (ids.cpu().numpy() == want_i).all()
    assert (dists.cpu().numpy() == want_d.astype(np.float32)).all()


@pytest.mark.parametrize("l2", (True, False))
@pytest.mark.parametrize("n,d,nq,k,dtype", [(1, 1, 1, 1, "int8"), (5, 16, 3, 10, "int8"), (63, 100, 7, 64, "int8"), (64, 128, 64, 10, "uint8"),
                                            (65, 33, 65, 5, "uint8"), (1000, 100, 130, 10, "int8"), (4097, 128, 37, 100, "uint8"),
                                            (3000, 200, 20, 128, "int8"), (10_000, 128, 300, 1, "uint8"), (20_001, 256, 5, 40, "int8"), (700, 500, 9, 7, "uint8"), (300, 1024, 4, 33, "int8"),
                                            (2500, 3, 11, 20, "int8")])
def test_search(env, n, d, nq, k, dtype, l2):
    torch, A, _ = env
    rng = np.random.default_rng(n + d + nq)
    rows = A.ann_mx_quantize(rows_of(torch, rng, n, d, dtype)[0], norms=True)
    queries = A.ann_mx_quantize(rows_of(torch, rng, nq, d, dtype)[0], norms=True)
    check_search(A, torch, rows, queries, k, l2)


@pytest.mark.parametrize("l2", (True, False))
@pytest.mark.parametrize("nq", (17, 33, 65, 200, 300, 600, 1100))
@pytest.mark.parametrize("n,d", [(700, 100), (2049, 130), (1500, 300), (3000, 450), (900, 600)])
def test_search_of_larger_batches(env, n, d, nq, l2):
    """Every way that rows and queries are dealt to waves."""
    torch, A, _ = env
    rng = np.random.default_rng(n + d + nq)
    rows = A.ann_mx_quantize(rows_of(torch, rng, n, d, "int8")[0], norms=True)
    queries = A.ann_mx_quantize(rows_of(torch, rng, nq, d, "int8")[0], norms=True)
    check_search(A, torch, rows, queries, 10, l2)


@pytest.mark.parametrize("l2", (True, False))
@pytest.mark.parametrize("nq", (3, 100, 700))
def test_search_equal_rows(env, nq, l2):
    """All rows equal: the first k ids; and only every other row with a distance."""
    torch, A, _ = env
    x = torch.ones((70_000, 100), device="cuda:0")
    queries = A.ann_mx_quantize(torch.ones((nq, 100), device="cuda:0"), norms=True)
    for k in (1, 10, 100):
        ids, dists = A.ann_mx_search(A.ann_mx_quantize(x, norms=True), queries, k, metric=A.L2SQ if l2 else A.MIPS)
        assert (ids.cpu() == torch.arange(k, dtype=torch.int32)).all() and (dists == (0.0 if l2 else -100.0)).all()
    x[::2, 40] = float("inf")
    ids, _ = A.ann_mx_search(A.ann_mx_quantize(x, norms=True), queries, 50, metric=A.L2SQ if l2 else A.MIPS)
    assert (ids.cpu() == torch.arange(1, 101, 2, dtype=torch.int32)).all()


@pytest.mark.parametrize("l2", (True, False))
def test_search_ties_and_rows_without_a_distance(env, l2):
    torch, A, _ = env
    rng = np.random.default_rng(1)
    x = rng.integers(0, 2, (5000, 40)).astype(np.float32)  # many equal distances
    x[100:4000] = x[7]
    q = np.concatenate([x[7:8], np.zeros((1, 40), np.float32), rng.integers(0, 2, (20, 40)).astype(np.float32)])
    rows, queries = (A.ann_mx_quantize(dev(torch, v), norms=True) for v in (x, q))
    for k in (1, 10, 65, 128):
        check_search(A, torch, rows, queries, k, l2)
    x[50:4990, 3] = np.nan  # no distance: never returned
    rows = A.ann_mx_quantize(dev(torch, x), norms=True)
    check = P.values(rows.codes.cpu().numpy(), rows.scales.cpu().numpy(), 40)
    assert np.isnan(check[50:4990]).any(axis=1).all()
    ids, dists = A.ann_mx_search(rows, queries, 128, metric=A.L2SQ if l2 else A.MIPS)
    ids, dists = ids.cpu().numpy(), dists.cpu().numpy()
    assert (np.sort(ids[:, :60]) == np.concatenate([np.arange(50), np.arange(4990, 5000)])).all()
    assert (ids[:, 60:] == -1).all() and (dists[:, 60:] == np.inf).all()
    rows = A.ann_mx_quantize(torch.full((70, 40), float("nan"), device="cuda:0"), norms=True)
    ids, dists = A.ann_mx_search(rows, queries, 3, metric=A.L2SQ if l2 else A.MIPS)
    assert (ids == -1).all() and (dists == float("inf")).all()


def test_search_of_norms_beyond_fp32(env):
    """Squared distances that leave fp32's range are infinite: those rows are not returned, whatever the products are."""
    torch, A, _ = env
    x = np.ones((200, 40), np.float32)
    x[5::20] = 2.0 ** 70
    q = np.stack([np.ones(40, np.float32), np.full(40, 2.0 ** 70, np.float32), np.full(40, -2.0 ** 60, np.float32)])
    rows, queries = (A.ann_mx_quantize(dev(torch, v), norms=True) for v in (x, q))
    assert torch.isinf(queries.norms[1]) and torch.isfinite(queries.norms[2])
    ids, dists = A.ann_mx_search(rows, queries, 128)
    ids, dists = ids.cpu().numpy(), dists.cpu().numpy()
    ones = np.setdiff1d(np.arange(200), np.arange(5, 200, 20))
    assert (ids[0] == ones[:128]).all() and (dists[0] == 0).all()
    assert (ids[1] == -1).all() and (dists[1] == np.inf).all()
    # 2^120 * 40 and 2^60 * 80 + 40, which fp32 rounds away
    assert (ids[2] == ones[:128]).all() and (dists[2] == np.float32(2.0 ** 120 * 40)).all()


def test_search_of_no_rows_or_queries(env):
    torch, A, _ = env
    rows = A.ann_mx_quantize(torch.ones((10, 40), device="cuda:0"), norms=True)
    none = A.ann_mx_quantize(torch.ones((0, 40), device="cuda:0"), norms=True)
    ids, dists = A.ann_mx_search(none, rows, 4)
    assert (ids == -1).all() and (dists == float("inf")).all()
    assert A.ann_mx_search(rows, none, 4)[0].shape == (0, 4)
    assert A.ann_mx_product(none, rows).shape == (0, 10) and A.ann_mx_product(rows, none).shape == (10, 0)


def test_search_in_several_launches(env):
    """More queries than the group maxima of one launch have room for."""
    torch, A, _ = env
    rng = np.random.default_rng(4)
    rows = A.ann_mx_quantize(torch.randint(-128, 128, (3_000_000, 32), dtype=torch.int8, device="cuda:0"), norms=True)
    queries = A.ann_mx_quantize(rows_of(torch, rng, 3000, 32, "int8")[0], norms=True)
    ids, dists = A.ann_mx_search(rows, queries, 10)
    for lo in (0, 1400, 2900):
        part = A.MxRows(queries.codes[lo:lo + 100].contiguous(), queries.scales[lo:lo + 100].contiguous(), 32, queries.norms[lo:lo + 100].contiguous())
        i, d = A.ann_mx_search(rows, part, 10)
        assert torch.equal(i, ids[lo:lo + 100]) and torch.equal(d, dists[lo:lo + 100])
    v, q = A.ann_mx_dequantize(rows).double(), A.ann_mx_dequantize(queries).double()
    for lo in (0, 2990):
        s = ((q[lo:lo + 10, None] - v[None]) ** 2).sum(2)
        assert torch.equal(torch.topk(s, 10, dim=1, largest=False, sorted=True).values.float(), dists[lo:lo + 10])


def test_offsets_beyond_32_bits(env):
    """Codes, inputs and outputs larger than 4 GiB: the last rows are the right ones."""
    torch, A, _ = env
    n, d = 1_100_001, 8192
    x = torch.zeros((n, d), dtype=torch.int8, device="cuda:0")
    g = torch.Generator(device="cuda:0").manual_seed(1)
    tail = torch.randint(-6, 7, (40, d), dtype=torch.int8, device="cuda:0", generator=g)
    x[-40:] = tail
    rows = A.ann_mx_quantize(x, norms=True)
    small = A.ann_mx_quantize(tail, norms=True)
    assert rows.codes.numel() > 1 << 32
    assert torch.equal(rows.codes[-40:], small.codes) and torch.equal(rows.norms[-40:], small.norms)
    b = torch.randn((3, d), dtype=torch.bfloat16, device="cuda:0", generator=g)
    assert torch.equal(A.ann_mx_product(b, rows)[:, -40:], A.ann_mx_product(b, small))
    assert torch.equal(A.ann_mx_product(small, rows)[:, -40:], A.ann_mx_product(small, small))
    ids, _ = A.ann_mx_search(rows, small, 1)
    assert (ids[:, 0].cpu().numpy() == np.arange(n - 40, n)).all()
    del x, rows
    w = A.ann_mx_quantize(torch.randint(-6, 7, (70_001, 64), dtype=torch.int8, device="cuda:0", generator=g))
    out = A.ann_mx_product(w, w, dtype=torch.float16)
    assert out.numel() > 1 << 32
    last = A.MxRows(w.codes[-50:].contiguous(), w.scales[-50:].contiguous(), 64)
    assert torch.equal(out[-50:], A.ann_mx_product(last, w, dtype=torch.float16))
    back = A.ann_mx_dequantize(w, dtype=torch.bfloat16)
    del out
    out = A.ann_mx_product(back, w, dtype=torch.float16)
    assert torch.equal(out[-50:], A.ann_mx_product(back[-50:], w, dtype=torch.float16))


def test_on_another_stream_and_in_a_graph(env):
    torch, A, _ = env
    rng = np.random.default_rng(12)
    x = rows_of(torch, rng, 40, 200, "float32")[0]
    r = A.ann_mx_quantize(rows_of(torch, rng, 3000, 200, "float32")[0], norms=True)

    def all_of(x, u):
        q = A.ann_mx_quantize(x, norms=True)
        ids, dists = A.ann_mx_search(r, q, 10)
        s16, s4 = A.ann_mx_product(x, r), A.ann_mx_product(q, r, dtype=torch.bfloat16)
        drawn, logprobs = A.ann_sample(s16, u, temperature=2.0, top_k=50, top_p=0.9, min_p=0.01)
        return A.ann_mx_dequantize(q), ids, dists, s16, s4, drawn, logprobs

    u = torch.rand(40, device="cuda:0")
    want = all_of(x, u)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = all_of(x, u)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    fixed, fixed_u = x.clone(), u.clone()
    with torch.cuda.graph(graph):
        held = all_of(fixed, fixed_u)
    for seed in range(4):
        new, new_u = rows_of(torch, np.random.default_rng(seed), 40, 200, "float32")[0], torch.rand(40, device="cuda:0")
        fixed.copy_(new)
        fixed_u.copy_(new_u)
        graph.replay()
        torch.cuda.synchronize()
        want = all_of(new, new_u)
        assert all(torch.equal(a, b) for a, b in zip(want, held)), seed


def test_calls_repeat_bit_for_bit(env):
    torch, A, _ = env
    rng = np.random.default_rng(2)
    x, w = rows_of(torch, rng, 33, 1000, "float32")[0], A.ann_mx_quantize(rows_of(torch, rng, 5001, 1000, "float32")[0], norms=True)
    q = A.ann_mx_quantize(x, norms=True)
    first = (A.ann_mx_product(x, w), A.ann_mx_product(q, w), *A.ann_mx_search(w, q, 50))
    for _ in range(3):
        again = (A.ann_mx_product(x, w), A.ann_mx_product(q, w), *A.ann_mx_search(w, q, 50))
        assert all(torch.equal(a, b) for a, b in zip(first, again))
