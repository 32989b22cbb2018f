"""Products whose sizes choose routes that batches of other sizes do not: the large tiles of two sides of 4 bits (from 24
tiles of 256 x 256 on, from 128 where rows have three to seven steps of 128 elements), and batches of more than 64 rows of
fewer than eight elements."""
import numpy as np
import pytest

import mx_plain as P
from test_gpu_mx import check_product, rows_of

pytestmark = pytest.mark.gpu


def held(r):
    return P.values(r.codes.cpu().numpy(), r.scales.cpu().numpy(), r.d)


@pytest.mark.parametrize("nx,n,d,out", [(600, 6001, 1100, "float32"),   # 72 tiles, nine steps: the last pair has one
                                        (1300, 8191, 300, "bfloat16"),  # 192 tiles, three steps
                                        (257, 3100, 1024, "float16"),   # 26 tiles, eight steps; one row in the second tile of the batch
                                        (2049, 769, 1920, "float32"),   # 36 tiles, fifteen steps; one row in the last tile of either side
                                        (1024, 8192, 896, "float16")])  # 128 whole tiles, seven steps
def test_large_tiles_of_packed_rows(env, nx, n, d, out):
    torch, A, _ = env
    rng = np.random.default_rng(nx + n + d)
    x = A.ann_mx_quantize(rows_of(torch, rng, nx, d, "bfloat16", spread=3)[0])
    w = A.ann_mx_quantize(rows_of(torch, rng, n, d, "float32", spread=4)[0])
    got = A.ann_mx_product(x, w, dtype=getattr(torch, out))
    check_product(A, torch, x, w, got, held(x), held(w))
    assert torch.equal(got, A.ann_mx_product(x, w, dtype=getattr(torch, out)))


@pytest.mark.parametrize("out,pad,at", [("float32", 0, 0), ("float32", 3, 1), ("float16", 5, 1), ("bfloat16", 4, 0), ("bfloat16", 8, 3)])
def test_large_tiles_of_packed_rows_with_bad_blocks(env, out, pad, at):
    """A block without values in the last step (of nine) spoils its row or column only; rows of any distance are written."""
    torch, A, _ = env
    nx, n, d = 300, 3100, 1030
    rng = np.random.default_rng(pad)
    x, xv = rows_of(torch, rng, nx, d, "float32")
    w, wv = rows_of(torch, rng, n, d, "float32")
    bad_x, bad_w = [0, 77, 255, 256, 299], [5, 127, 128, 2000, 3071, 3099]
    x[bad_x, d - 1] = float("nan")
    w[bad_w, d - 3] = float("inf")
    x, w = A.ann_mx_quantize(x), A.ann_mx_quantize(w)
    wide = torch.full((nx, n + pad), -7.0, dtype=getattr(torch, out), device="cuda:0")
    got = A.ann_mx_product(x, w, out=wide[:, at:at + n])
    good_x, good_w = np.setdiff1d(np.arange(nx), bad_x), np.setdiff1d(np.arange(n), bad_w)
    assert got[bad_x].isnan().all() and got[:, bad_w].isnan().all()
    check_product(A, torch, x, w, got[good_x][:, good_w], held(x)[good_x], held(w)[good_w])
    assert (wide[:, :at] == -7.0).all() and (wide[:, at + n:] == -7.0).all()


@pytest.mark.parametrize("dtype", ("float32", "float16", "bfloat16"))
@pytest.mark.parametrize("d", range(1, 8))
def test_batches_of_very_short_rows(env, dtype, d):
    torch, A, _ = env
    rng = np.random.default_rng(d)
    w = A.ann_mx_quantize(rows_of(torch, rng, 300, d, "float32", spread=4)[0])
    for nx, pad in ((65, 0), (100, 3), (300, 0)):
        t, x = rows_of(torch, rng, nx, d, dtype, pad)
        check_product(A, torch, t, w, A.ann_mx_product(t, w), x, held(w))
