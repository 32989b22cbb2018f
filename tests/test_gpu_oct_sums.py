"""What the sums of ann_oct_product hold: whole products, every step of long rows, tiles of every kind."""
import pytest

from test_gpu_oct import check_product

pytestmark = pytest.mark.gpu

# few rows; few tiles; narrow and small tiles; large ones, which need a chip of them: whole ones, and ends of both sides
LARGE = [(2048, 8192, 640), (1999, 8101, 513), (2047, 8190, 1536), (1800, 8000, 4200)]
ROUTES = [(5, 3000, 300), (17, 33, 640), (33, 10_300, 140), (200, 8192, 1030), (2048, 4096, 2048), (2047, 4101, 1536), *LARGE]


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


@pytest.mark.parametrize("nx,n,d", LARGE)
@pytest.mark.parametrize("out", ("float32", "float16", "bfloat16"))
def test_product_by_large_tiles(env, nx, n, d, out):
    torch, A, _ = env
    x, w = rows_of(torch, A, nx, d, 3), rows_of(torch, A, n, d, 4)
    known = None
    for pad in (0, 7):
        known = check_product(torch, A, x, w, out, pad, known)


def test_not_a_number_by_large_tiles(env):
    """A step of NaN on either side makes the results that it takes part in NaN, and no others."""
    torch, A, _ = env
    x, w = torch.zeros((2048, 600), device="cuda"), torch.zeros((8192, 600), device="cuda")
    x[3, 7], x[2047, 599], w[5, 130], w[8191, 0] = torch.nan, torch.inf, -torch.inf, torch.nan
    want = torch.zeros((2048, 8192), dtype=torch.bool, device="cuda")
    want[[3, 2047]] = True
    want[:, [5, 8191]] = True
    for t in (torch.float32, torch.float16, torch.bfloat16):
        got = A.ann_oct_product(A.ann_oct_quantize(x), A.ann_oct_quantize(w), dtype=t)
        assert torch.equal(got.isnan(), want), t


# by a wave, and by eight and four that share a tile's steps, of one row and of more; few tiles; narrow, small and large ones
@pytest.mark.parametrize("nx,n,d", [(1, 40, 70_000), (5, 16, 20_000), (3, 70, 1 << 20), (16, 33_000, 300), (9, 66_000, 1030), (2, 66_000, 1030), (7, 65_600, 4100),
                                    (1, 65_600, 4999), (40, 50, 20_001), (300, 100, 70_000), (50, 12_001, 9000), (200, 8192, 5003), (1999, 8101, 5003)])
def test_every_step_of_long_rows(env, nx, n, d):
    """Whole numbers whose products, and all sums of them, fp32 holds: at most 8, or 3, in magnitude, d of them times 64 or 9 below
    2^24.  The codes hold them (four bits), and the cut of eight products takes nothing from whole numbers.  So results are
    the sum, rounded once; each step has its share of nearly all of them."""
    torch, A, _ = env
    most = 8 if d * 64 < 1 << 24 else 3
    assert d * most * most < 1 << 24
    g = torch.Generator("cuda").manual_seed(n + d)
    x, w = (torch.randint(-most, most + 1, (r, d), device="cuda", generator=g).float() for r in (nx, n))
    want = x.double() @ w.double().T
    x, w = A.ann_oct_quantize(x), A.ann_oct_quantize(w)
    for t in (torch.float32, torch.float16, torch.bfloat16):
        assert torch.equal(A.ann_oct_product(x, w, dtype=t), want.to(t)), t


@pytest.mark.parametrize("nx,n,d", [(64, 12_001, 1000), (200, 8192, 2048), (2048, 8192, 2048)])
@pytest.mark.parametrize("large", (0.0, 0.01))
def test_what_the_cut_takes_from_bf16_results(env, nx, n, d, large):
    """The cut's errors e, of each eight products what lies below 2^(E - 13), are made anew here for 64 x 256 of the results.  A
    result rounds to another bf16 number than the whole sum with a probability of |e| over a step of it (at most 2^-7 of it), and then is a step
    and |e| away: of the mean square of the difference no more than 2^-7 rms(e) rms(results) + rms(e)^2.  Twice rms(e) allows
    for how well 16,384 results stand for all, and for a cut that does not look at signs."""
    torch, A, _ = env
    x, w = rows_of(torch, A, nx, d, 5, large), rows_of(torch, A, n, d, 6, large)
    xv, wv = (A.ann_oct_dequantize(A.OctRows(r.codes[:m].contiguous(), r.scales[:m].contiguous(), d)).double() for r, m in ((x, 64), (w, 256)))
    e = torch.zeros((64, 256), dtype=torch.float64, device="cuda")
    for i in range(0, d, 8):
        p = xv[:, None, i:i + 8] * wv[None, :, i:i + 8]
        unit = torch.exp2(torch.floor(torch.log2(p.abs().amax(dim=2, keepdim=True).clamp_min(1e-300))) - 13)
        e += (torch.trunc(p / unit) * unit - p).sum(dim=2)
    whole = A.ann_oct_product(x, w)
    rms = whole.double().square().mean().sqrt()
    cut = 2 * e.square().mean().sqrt()
    assert cut < 2.0 ** -12 * rms  # (a sixteenth of what bf16 may round)
    off = (A.ann_oct_product(x, w, dtype=torch.bfloat16).double() - whole.bfloat16().double()).square().mean()
    assert off <= 2.0 ** -7 * cut * rms + cut * cut, (off.sqrt() / rms, cut / rms)


def test_large_tiles_in_a_graph(env):
    """Captured and replayed on new contents, with eager work between."""
    torch, A, _ = env
    g = torch.Generator("cuda").manual_seed(9)
    x, w = torch.randn((2048, 700), device="cuda", generator=g), torch.randn((8192, 700), device="cuda", generator=g)

    def chain():
        return [A.ann_oct_product(A.ann_oct_quantize(x), A.ann_oct_quantize(w), dtype=t) for t in (torch.float32, torch.float16, torch.bfloat16)]

    chain()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = chain()
    for turn in range(4):
        x.copy_(torch.roll(x, 1, 0))
        want = chain()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), turn
