"""What the sums of ann_oct_product hold: whole products, every step of long rows, tiles of very many rows."""
import pytest

pytestmark = pytest.mark.gpu

# few rows; few tiles; narrow, small and large tiles
ROUTES = [(5, 3000, 300), (17, 33, 640), (33, 10_300, 140), (200, 8192, 1030), (2048, 4096, 2048), (2047, 4101, 1536)]


def rows_of(torch, A, n, d, seed, large=0.01):
    """Normal numbers, a hundredth of whose channels (the same ones for all) are twelve times as large."""
    g = torch.Generator("cuda").manual_seed(seed)
    c = torch.Generator("cuda").manual_seed(7)
    x = torch.randn((n, d), device="cuda", generator=g) * torch.where(torch.rand(d, device="cuda", generator=c) < large, 12.0, 1.0)
    return A.ann_oct_quantize(x)


@pytest.mark.parametrize("nx,n,d", ROUTES)
@pytest.mark.parametrize("large", (0.0, 0.01))
def test_fp16_results_are_the_fp32_ones_rounded(env, nx, n, d, large):
    """Products are whole for both, and their sums the same: one rounding between them."""
    torch, A, _ = env
    x, w = rows_of(torch, A, nx, d, 1, large), rows_of(torch, A, n, d, 2, large)
    assert torch.equal(A.ann_oct_product(x, w, dtype=torch.float16), A.ann_oct_product(x, w).half())
