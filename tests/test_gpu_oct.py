"""8-bit rows and their products against the definition in 64 bits."""
import numpy as np
import pytest

import oct_plain as P
from helpers import dev

pytestmark = pytest.mark.gpu

HALF = {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}  # of a step, relative to the value
SMALLEST = {"float32": 2.0 ** -149, "float16": 2.0 ** -24, "bfloat16": 2.0 ** -133}


def rows_of(torch, rng, n, d, dtype):
    if dtype in ("uint8", "int8"):
        lo, hi = (0, 256) if dtype == "uint8" else (-128, 128)
        return dev(torch, rng.integers(lo, hi, (n, d)).astype(dtype))
    x = rng.standard_normal((n, d)) * np.exp2(rng.integers(-12, 13, (n, d)))
    x[rng.random((n, d)) < 0.05] = 0.0
    return dev(torch, x.astype(np.float32)).to(getattr(torch, dtype))


def wider(torch, x, pad):
    wide = torch.full((x.shape[0], x.shape[1] + pad), 77, dtype=x.dtype, device=x.device)
    wide[:, pad // 2:pad // 2 + x.shape[1]] = x
    return wide[:, pad // 2:pad // 2 + x.shape[1]]


@pytest.mark.parametrize("dtype", ("float32", "float16", "bfloat16", "uint8", "int8"))
@pytest.mark.parametrize("n,d", [(1, 1), (3, 7), (5, 8), (2, 127), (4, 128), (3, 129), (70, 200), (9, 256), (5, 257), (6, 512), (3, 513), (2, 1300),
                                 (130, 100), (1, 4097), (257, 65)])
@pytest.mark.parametrize("columns", (False, True))
def test_quantize(env, dtype, n, d, columns):
    """Codes and scale bytes, bit by bit, of rows anywhere in wider ones; padding 0."""
    torch, A, _ = env
    rng = np.random.default_rng(n * d)
    x = rows_of(torch, rng, n, d, dtype)
    want = P.quantize(x.double().cpu().numpy())
    for pad in (0, 3, 8):
        given = wider(torch, x.T.contiguous() if columns else x, pad)
        got = A.ann_oct_quantize(given, columns=columns)
        assert (got.scales.cpu().numpy() == want[1]).all(), pad
        assert (got.codes.cpu().numpy() == want[0]).all(), pad
    exact = P.values(*want, d)
    for out in ("float32", "float16", "bfloat16"):
        v = A.ann_oct_dequantize(got, dtype=getattr(torch, out))
        assert torch.equal(v.cpu(), torch.from_numpy(exact).to(v.dtype)), out
        room = wider(torch, torch.zeros((n, d), dtype=v.dtype, device=v.device), 5)
        around = room._base.clone()
        A.ann_oct_dequantize(got, out=room)
        assert torch.equal(room, v)
        around[:, 2:2 + d] = v
        assert torch.equal(room._base, around), "elements beside the rows changed"


@pytest.mark.parametrize("dtype", ("float32", "bfloat16", "int8"))
@pytest.mark.parametrize("n,d", [(1, 20_000), (33, 16_384), (64, 513), (70, 385), (999, 130), (1000, 1), (40, 640), (11, 100_003), (2, 1 << 20), (300, 2000)])
def test_steps_of_many_rows(env, dtype, n, d):
    """Long rows, and rows that begin and end inside what a workgroup takes at once; there and back, in wider rows too."""
    torch, A, _ = env
    x = rows_of(torch, np.random.default_rng(n + d), n, d, dtype)
    want = P.quantize(x.double().cpu().numpy())
    for given in (x, wider(torch, x, 5)):
        got = A.ann_oct_quantize(given)
        assert (got.scales.cpu().numpy() == want[1]).all() and (got.codes.cpu().numpy() == want[0]).all()
    exact = torch.from_numpy(P.values(*want, d))
    for out in (torch.float32, torch.bfloat16):
        room = wider(torch, torch.zeros((n, d), dtype=out, device=x.device), 7)
        around = room._base.clone()
        A.ann_oct_dequantize(got, out=room)
        around[:, 3:3 + d] = exact.to(out).to(x.device)
        assert torch.equal(room._base, around)


@pytest.mark.parametrize("columns", (False, True))
def test_quantize_edges(env, columns):
    """Every code and every middle between two, numbers at the ends of fp32, infinities and NaN in a step of their own."""
    torch, A, _ = env
    v = P.code_values()[:127]
    every = np.concatenate([v, -v, (v[1:] + v[:-1]) / 2, np.nextafter(((v[1:] + v[:-1]) / 2).astype(np.float32), np.float32(0)),
                            np.nextafter(((v[1:] + v[:-1]) / 2).astype(np.float32), np.float32(1e9))])
    rows = []
    for scale in (0, -100, -126, 100, 115):
        x = np.zeros((128, 130))
        for i in range(0, len(every), 127):
            part = every[i:i + 127]
            x[i // 127, 1:1 + len(part)] = part
            x[i // 127, 0] = 448.0  # the scale
        rows.append(x * 2.0 ** scale)
    x = np.concatenate(rows).astype(np.float32)
    x[5, 7], x[6, 9], x[7, 129] = np.inf, np.nan, -np.inf
    tiny = np.zeros((4, 130), np.float32)
    tiny[0, :3] = 2.0 ** -149, 2.0 ** -130, -2.0 ** -140
    tiny[1, 0] = np.finfo(np.float32).max
    tiny[2, 0] = -np.finfo(np.float32).max
    x = np.concatenate([x, tiny])
    t = dev(torch, x)
    got = A.ann_oct_quantize(t.T.contiguous() if columns else t, columns=columns)
    want = P.quantize(x.astype(np.float64))
    assert (got.scales.cpu().numpy() == want[1]).all()
    assert (got.codes.cpu().numpy() == want[0]).all()
    back = A.ann_oct_dequantize(got).cpu()
    assert torch.equal(back.isnan(), torch.from_numpy(np.isnan(P.values(*want, 130))))


def product_bound(torch, xv, wv, out):
    """Sums in fp32: each of the d additions is off by at most a step of what the sum of magnitudes allows.  Where the matrix
    instruction takes the codes (results of 16 bits, batches above 16) it drops, of eight neighbouring products, what
    lies below 2^(E - 13), E the largest one's exponent, of up to seven of them.  Then one rounding to the output's type."""
    d = xv.shape[1]
    x, w = xv.abs(), wv.abs()
    bound = d * 2.0 ** -23 * (x @ w.T)
    if out != "float32" and len(xv) > 16:
        for e in range(0, d, 8):
            best = x[:, e, None] * w[None, :, e]
            for k in range(e + 1, min(e + 8, d)):
                best = torch.maximum(best, x[:, k, None] * w[None, :, k])
            bound += 7 * 2.0 ** -13 * best
    return bound


def values_of(torch, rows):
    return dev(torch, P.values(rows.codes.cpu().numpy(), rows.scales.cpu().numpy(), rows.d))


def check_product(torch, A, x, w, out="float32", pad=0, known=None):
    xv, wv = values_of(torch, x), values_of(torch, w)
    want = xv @ wv.T
    room = wider(torch, torch.zeros(want.shape, dtype=getattr(torch, out), device="cuda"), pad) if pad else None
    got = A.ann_oct_product(x, w, dtype=None if pad else getattr(torch, out), out=room)
    sums = product_bound(torch, xv, wv, out) if known is None else known
    off = (got.double() - want).abs()
    assert (off <= sums + HALF[out] * (want.abs() + sums) + SMALLEST[out]).all(), (off.max().item(), want.abs().max().item())
    if pad:
        side = room._base.clone()
        side[:, pad // 2:pad // 2 + want.shape[1]] = 77
        assert (side == 77).all(), "elements beside the results changed"
    return sums


# (few rows; few tiles; narrow, small and large tiles: whole ones, ends of both sides, one step and more than whole words)
@pytest.mark.parametrize("out", ("float32", "float16", "bfloat16"))
@pytest.mark.parametrize("nx,n,d", [(1, 1, 1), (1, 5000, 128), (2, 3, 130), (16, 64, 512), (17, 33, 640), (33, 1001, 200), (64, 500, 1000), (65, 129, 384),
                                    (130, 70, 4097), (5, 16, 20_000), (257, 300, 96), (400, 1030, 257), (1, 40, 70_000), (7, 40_000, 700),
                                    (33, 10_300, 140), (64, 12_001, 96), (18, 20_500, 1500), (130, 5003, 257), (200, 8192, 1030), (129, 6000, 96),
                                    (2100, 4000, 513), (2048, 4096, 1030), (2047, 4101, 1536)])
def test_product(env, out, nx, n, d):
    torch, A, _ = env
    rng = np.random.default_rng(nx * n + d)
    x, w = (dev(torch, (0.3 * rng.standard_normal((r, d)) * np.exp2(rng.integers(-2, 3, (r, 1)))).astype(np.float32)) for r in (nx, n))
    # scales of their own for every step
    for t in (x, w):
        for e in range(0, d, 128):
            t[:, e:e + 128] *= 2.0 ** int(rng.integers(-3, 4))
    x, w = A.ann_oct_quantize(x), A.ann_oct_quantize(w)
    known = None
    for pad in (0, 7, 8):
        known = check_product(torch, A, x, w, out, pad, known)


# (tiles of 32 and of 64 rows, whole steps of a wave and shared ones; the last workgroup's waves partly without a tile)
@pytest.mark.parametrize("nx,n,d", [(1, 70_001, 300), (16, 33_000, 128), (4, 66_000, 600), (16, 65_573, 1000), (1, 65_600, 1030), (3, 131_071, 2000), (5, 65_537, 2300),
                                    (1, 65_601, 2980), (16, 65_540, 3200), (9, 40_001, 800), (2, 20_003, 200)])
def test_few_rows_by_many(env, nx, n, d):
    torch, A, _ = env
    g = torch.Generator("cuda").manual_seed(n)
    x, w = (torch.randn((r, d), device="cuda", generator=g) * torch.exp2(torch.randint(-3, 4, (r, 1), device="cuda", generator=g)) for r in (nx, n))
    x, w = A.ann_oct_quantize(x), A.ann_oct_quantize(w)
    xv, wv = A.ann_oct_dequantize(x).double(), A.ann_oct_dequantize(w).double()
    want, sums = xv @ wv.T, d * 2.0 ** -23 * (xv.abs() @ wv.abs().T)
    for out in ("float32", "bfloat16"):
        room = wider(torch, torch.zeros((nx, n), dtype=getattr(torch, out), device="cuda"), 5)
        got = A.ann_oct_product(x, w, out=room)
        assert ((got.double() - want).abs() <= sums + HALF[out] * (want.abs() + sums)).all()
        assert torch.equal(got, A.ann_oct_product(x, w, dtype=got.dtype))
        side = room._base.clone()
        side[:, 2:2 + n] = 77
        assert (side == 77).all(), "elements beside the results changed"


def test_product_of_every_code(env):
    """All codes of one side by all of the other, in every place of a step, with scales far apart."""
    torch, A, _ = env
    codes = np.array([c for c in range(256) if c not in (127, 255)], np.uint8)
    d = 300
    x = np.zeros((len(codes), 384), np.uint8)
    for i, c in enumerate(codes):
        x[i, i % d] = c
    w = np.zeros((len(codes), 384), np.uint8)
    w[:, :d] = codes[:, None]
    scales = np.zeros((len(codes), 4), np.uint8)
    for i in range(len(codes)):
        scales[i, :3] = 100 + i % 50, 127, 150 - i % 30
    xo = A.OctRows(dev(torch, x), dev(torch, scales), d)
    wo = A.OctRows(dev(torch, w), dev(torch, scales[::-1].copy()), d)
    got = A.ann_oct_product(xo, wo).double().cpu().numpy()
    want = P.values(x, scales, d) @ P.values(w, scales[::-1], d).T
    assert (got == want).all()  # one product each: exact
    # the same in every place of a step, by tiles: rows enough for the codes themselves to be multiplied
    reps = 16
    xo, wo = (A.OctRows(o.codes.repeat(reps, 1), o.scales.repeat(reps, 1), d) for o in (xo, wo))
    for t in (torch.float32, torch.bfloat16):
        got = A.ann_oct_product(xo, wo, dtype=t)
        assert torch.equal(got, dev(torch, want).to(t).repeat(reps, reps)), t


@pytest.mark.parametrize("nx,n,d", [(3, 100, 200), (70, 300, 520), (40, 11_000, 130), (140, 5100, 300), (2048, 4096, 520)])
def test_scales_far_from_one(env, nx, n, d):
    """Small numbers by large ones, in steps whose scales differ by 2^30."""
    torch, A, _ = env
    rng = np.random.default_rng(n)
    x, w = (dev(torch, rng.standard_normal((r, d)).astype(np.float32)) for r in (nx, n))
    x *= 2.0 ** -100
    w *= 2.0 ** 90
    x[:, 128:] *= 2.0 ** 30
    w[:, 128:] *= 2.0 ** -30
    x, w = A.ann_oct_quantize(x), A.ann_oct_quantize(w)
    for out in ("float32", "bfloat16"):
        check_product(torch, A, x, w, out)


def test_not_a_number(env):
    """A step of NaN on either side makes the results that it takes part in NaN, and no others."""
    torch, A, _ = env
    rng = np.random.default_rng(3)
    x = rng.standard_normal((70, 400)).astype(np.float32)
    w = rng.standard_normal((300, 400)).astype(np.float32)
    x[3, 7], x[69, 399], w[5, 130], w[299, 0] = np.nan, np.inf, -np.inf, np.nan
    got = A.ann_oct_product(A.ann_oct_quantize(dev(torch, x)), A.ann_oct_quantize(dev(torch, w))).cpu().numpy()
    want = np.zeros((70, 300), bool)
    want[[3, 69]] = True
    want[:, [5, 299]] = True
    assert (np.isnan(got) == want).all()
    for nx, n in ((40, 11_000), (140, 5100), (2048, 4096)):  # tiles
        x, w = (torch.zeros((r, 400), device="cuda") for r in (nx, n))
        x[3, 7], x[nx - 1, 399], w[5, 130], w[n - 1, 0] = np.nan, np.inf, -np.inf, np.nan
        want = torch.zeros((nx, n), dtype=torch.bool, device="cuda")
        want[[3, nx - 1]] = True
        want[:, [5, n - 1]] = True
        for t in (torch.float32, torch.bfloat16):
            got = A.ann_oct_product(A.ann_oct_quantize(x), A.ann_oct_quantize(w), dtype=t)
            assert torch.equal(got.isnan(), want), (nx, n, t)


def test_gradients(env):
    """The gradients of sum(Y * G), Y = X W^T, as products of rows and columns, against the formula and against differences of
    the forward product, in values that 8 bits hold exactly."""
    torch, A, _ = env
    rng = np.random.default_rng(11)
    nx, n, d = 60, 90, 210
    x, w, g = (dev(torch, rng.integers(-8, 9, s).astype(np.float32) / 8) for s in ((nx, d), (n, d), (nx, n)))
    q = A.ann_oct_quantize
    dx = A.ann_oct_product(q(g), q(w, columns=True)).double().cpu()
    dw = A.ann_oct_product(q(g, columns=True), q(x, columns=True)).double().cpu()
    # sums of at most 210 multiples of 1/64 below 2^2: exact in fp32
    assert torch.equal(dx, g.double().cpu() @ w.double().cpu())
    assert torch.equal(dw, g.double().cpu().T @ x.double().cpu())

    def loss(x, w):
        return (A.ann_oct_product(q(x), q(w)).double() * g.double()).sum().item()

    base = loss(x, w)
    for i, e in ((0, 0), (59, 209), (31, 128)):
        moved = x.clone()
        moved[i, e] += 0.125 if moved[i, e] < 0 else -0.125
        assert (loss(moved, w) - base) / (moved[i, e] - x[i, e]).item() == dx[i, e].item()
    for j, e in ((0, 3), (89, 209)):
        moved = w.clone()
        moved[j, e] += 0.125 if moved[j, e] < 0 else -0.125
        assert (loss(x, moved) - base) / (moved[j, e] - w[j, e]).item() == dw[j, e].item()


def test_empty(env):
    torch, A, _ = env
    none, some = A.ann_oct_quantize(torch.zeros((0, 100), device="cuda")), A.ann_oct_quantize(torch.zeros((3, 100), device="cuda"))
    assert A.ann_oct_product(none, some).shape == (0, 3) and A.ann_oct_product(some, none).shape == (3, 0)
    assert A.ann_oct_dequantize(none).shape == (0, 100)
    assert A.ann_oct_quantize(torch.zeros((100, 0), device="cuda"), columns=True).codes.shape == (0, 128)
    assert (A.ann_oct_product(some, some) == 0).all()


def test_offsets_beyond_32_bits(env):
    """Codes of more than 2^32 bytes, results of more than 2^32 elements."""
    torch, A, _ = env
    n = (1 << 32) // 1024 + 5000
    x = torch.zeros((n, 1000), dtype=torch.int8, device="cuda")
    last = torch.arange(1000, device="cuda").to(torch.int8)
    x[-1] = last
    rows = A.ann_oct_quantize(x)
    want = A.ann_oct_quantize(x[-1:].clone())
    assert torch.equal(rows.codes[-1:], want.codes) and torch.equal(rows.scales[-1:], want.scales)
    got = A.ann_oct_product(want, rows)
    assert got[0, -1] == A.ann_oct_product(want, want)[0, 0] and (got[0, :-1] == 0).all()
    back = A.ann_oct_dequantize(rows, dtype=torch.bfloat16)
    assert torch.equal(back[-1:], A.ann_oct_dequantize(want, dtype=torch.bfloat16))
    del back, x
    few = A.OctRows(rows.codes[-1100:], rows.scales[-1100:], 1000)
    out = A.ann_oct_product(few, rows, dtype=torch.bfloat16)  # 1,100 x 4.2 million
    assert out.numel() > 1 << 32 and torch.equal(out[-1].float(), A.ann_oct_product(want, rows, dtype=torch.bfloat16)[0].float())
    assert (out[:-1, :-1] == 0).all() and (out[:-1, -1] == 0).all()


def test_values_of_more_pieces_than_32_bits_count(env):
    """2^27 rows and some of 127 fp32 values, 32 pieces of 16 bytes each."""
    torch, A, _ = env
    n = (1 << 27) + 77
    codes = torch.zeros((n, 128), dtype=torch.uint8, device="cuda")
    scales = torch.full((n, 4), 127, dtype=torch.uint8, device="cuda")
    some = A.ann_oct_quantize(torch.randn((100, 127), device="cuda", generator=torch.Generator("cuda").manual_seed(4)))
    for at in (0, 1 << 26, n - 100):
        codes[at:at + 100], scales[at:at + 100] = some.codes, some.scales
    out = A.ann_oct_dequantize(A.OctRows(codes, scales, 127))
    want = A.ann_oct_dequantize(some)
    for at in (0, 1 << 26, n - 100):
        assert torch.equal(out[at:at + 100], want)
        out[at:at + 100] = 0
    for at in range(0, n, 1 << 24):
        assert not out[at:at + (1 << 24)].any()


def test_streams_graphs_and_repeats(env):
    """On another stream, captured and replayed on new contents with eager work between, and twice the same bits."""
    torch, A, _ = env
    rng = np.random.default_rng(5)
    x, w = dev(torch, rng.standard_normal((50, 700)).astype(np.float32)), dev(torch, rng.standard_normal((900, 700)).astype(np.float32))

    def chain():
        return A.ann_oct_product(A.ann_oct_quantize(x), A.ann_oct_quantize(w)), A.ann_oct_quantize(x, columns=True).codes

    want = chain()
    assert all(torch.equal(a, b) for a, b in zip(chain(), want))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = chain()
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = chain()
    for turn in range(4):
        x.copy_(torch.roll(x, turn, 0))
        want = chain()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), turn
