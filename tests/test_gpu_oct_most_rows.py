"""Products with as many rows as one launch's threads of 32 bits allow for, and more."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,d,batches", [((1 << 27) - 1, 512, (1, 16)), ((1 << 27) + 77, 512, (1, 16)), ((1 << 30) - 1, 100, (1, 17))])
def test_product_with_very_many_rows(env, n, d, batches):
    """Rows of zeros with others at the beginning, in the middle and at the end.  (Batches of up to 16 rows with up to 2^27 rows
    of four steps and more share a tile's steps between waves; more rows of them, and up to 2^30 of fewer steps, have a tile a wave.)"""
    torch, A, _ = env
    steps = (d + 127) // 128
    codes = torch.zeros((n, 128 * steps), dtype=torch.uint8, device="cuda")
    scales = torch.full((n, (steps + 3) // 4 * 4), 127, dtype=torch.uint8, device="cuda")
    g = torch.Generator("cuda").manual_seed(8)
    some = A.ann_oct_quantize(torch.randn((100, d), device="cuda", generator=g))
    places = (0, n // 2 + 5, n - 100)
    for at in places:
        codes[at:at + 100], scales[at:at + 100] = some.codes, some.scales
    for nx in batches:
        x = A.ann_oct_quantize(torch.randn((nx, d), device="cuda", generator=g))
        dtype = torch.float32 if nx == 1 else torch.bfloat16
        got = A.ann_oct_product(x, A.OctRows(codes, scales, d), dtype=dtype)
        want = A.ann_oct_dequantize(x).double() @ A.ann_oct_dequantize(some).double().T
        sums = d * 2.0 ** -23 * (A.ann_oct_dequantize(x).double().abs() @ A.ann_oct_dequantize(some).double().abs().T)
        if nx > 16:  # codes are multiplied: of eight products at most 7 * 2^-13 of their magnitudes is dropped
            sums += 7 * 2.0 ** -13 / (d * 2.0 ** -23) * sums
        for at in places:
            off = (got[:, at:at + 100].double() - want).abs()
            assert (off <= sums + (2.0 ** -24 if nx == 1 else 2.0 ** -8) * (want.abs() + sums)).all(), (nx, at)
            got[:, at:at + 100] = 0
        for at in range(0, n, 1 << 26):
            assert not got[:, at:at + (1 << 26)].any(), (nx, at)
        del got
