"""ann_distill and ann_distill_grad against the formulas in 64 bits."""
import numpy as np
import pytest

from helpers import dev

pytestmark = pytest.mark.gpu

HALF = {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}
SMALLEST = {"float32": 2.0 ** -149, "float16": 2.0 ** -24, "bfloat16": 2.0 ** -133}
U = 2.0 ** -24  # half a step of fp32


def plain(z, ids, teacher, t):
    """(losses, gradients of the losses, and how far the kernels' fp32 steps may take them from these), row by row."""
    rows, n = z.shape
    losses, grads = np.zeros(rows), np.zeros((rows, n))
    loss_off, grad_off = np.zeros(rows), np.zeros((rows, n))
    for r in range(rows):
        there = (ids[r] >= 0) & (ids[r] < n) & (teacher[r] != -np.inf)
        if not there.any() or (z[r] == -np.inf).all():
            continue
        with np.errstate(all="ignore"):
            x = (z[r] - z[r].max()) / t
            e = np.exp(x)
            s = e.sum()
            q = e / s
            a = (teacher[r][there] - teacher[r][there].max()) / t
            w = np.exp(a)
            p = w / w.sum()
            at = ids[r][there]
            losses[r] = t * t * np.where(p > 0, p * (np.log(p) - (x[at] - np.log(s))), 0.0).sum()
        share = np.zeros(n)
        np.add.at(share, at, p)
        grads[r] = t * (q - share)
        # A term of S: its argument is rounded in the difference, the factor and the product (half a step each of the argument),
        # exp2 is off by a step, half a step more for the product with 1 / S and for 1 / S.  A sum of up to n / 256 + 64
        # terms one after another and 14 joins with an exp2 and a product each.
        finite = np.where(np.isfinite(x), np.abs(x), 0.0)
        term = 3 * U * finite + 2 * U
        total = (q * term).sum() + (n / 256 + 64 + 14 * 5) * U
        loss_off[r] = t * t * total + HALF["float32"] * abs(losses[r]) + 1e-12 * t * t * (np.abs(x[at][p > 0]).max(initial=0) + 50)
        share_off = np.zeros(n)
        np.add.at(share_off, at, p * (3 * U * np.abs(np.where(p > 0, a, 0.0)) + 8 * U))
        grad_off[r] = t * (q * (term + total + 3 * U) + share_off + len(at) * U * share + 3 * U * (q + share))
    return losses, grads, loss_off, grad_off


def check(torch, A, z, ids, teacher, t=1.0, up=None, scale=1.0, out=None):
    losses, stats = A.ann_distill(z, ids, teacher, temperature=t)
    grads = A.ann_distill_grad(z, ids, teacher, stats, grad_losses=up, temperature=t, scale=scale, out=out)
    zh, th, ih = z.double().cpu().numpy(), teacher.double().cpu().numpy(), ids.cpu().numpy()
    want, wgrads, loss_off, grad_off = plain(zh, ih, th, t)
    got = losses.double().cpu().numpy()
    with np.errstate(all="ignore"):
        assert ((got == want) | (np.abs(got - want) <= loss_off)).all(), (np.abs(got - want) / loss_off).max()
    f = (up.double().cpu().numpy()[:, None] if up is not None else 1.0) * float(np.float32(scale))
    name = str(z.dtype).split(".")[1]
    off = np.abs(grads.double().cpu().numpy() - wgrads * f)
    may = grad_off * np.abs(f) + 3 * U * np.abs(wgrads * f)
    may = may + HALF[name] * (np.abs(wgrads * f) + may) + SMALLEST[name] + 2.0 ** -120 * np.abs(f)
    assert grads.dtype == z.dtype and (off <= may).all(), (off / may).max()
    return losses, stats, grads


def inputs(torch, rng, rows, n, k, dtype, masked=0.0, short=False, tdtype="float32"):
    z = 3.0 * rng.standard_normal((rows, n))
    ids = np.stack([rng.permutation(n)[:k] if k <= n else rng.integers(0, n, k) for _ in range(rows)])
    if masked:
        m = rng.random((rows, n)) < masked
        m[np.arange(rows)[:, None], ids] = False  # (the loss of a teacher's masked entry is +inf: tested apart)
        z[m] = -np.inf
    teacher = 2.0 * rng.standard_normal((rows, k))
    if short:
        gone = rng.random((rows, k)) < 0.4
        ids = np.where(gone, rng.choice([-1, n, 2 ** 31 - 1], (rows, k)), ids)
        teacher[rng.random((rows, k)) < 0.1] = -np.inf
        ids[0] = -1
    return dev(torch, z).to(getattr(torch, dtype)), dev(torch, ids.astype(np.int32)), dev(torch, teacher).to(getattr(torch, tdtype))


def wider(torch, x, pad):
    wide = torch.full((x.shape[0], x.shape[1] + pad), 77, dtype=x.dtype, device=x.device)
    wide[:, :x.shape[1]] = x
    return wide[:, :x.shape[1]]


@pytest.mark.parametrize("dtype", ("float32", "float16", "bfloat16"))
@pytest.mark.parametrize("rows,n,k", [(1, 1, 1), (3, 2, 2), (2, 7, 3), (5, 8, 8), (4, 9, 20), (3, 100, 10), (7, 1025, 64), (2, 5000, 1024), (1, 8192, 5), (3, 8193, 10), (2, 16_384, 9), (1, 16_385, 9),
                                      (2, 16_391, 33), (600, 130, 7), (37, 10_000, 10)])
def test_sizes(env, dtype, rows, n, k):
    torch, A, _ = env
    rng = np.random.default_rng(rows * n + k)
    for i, (t, masked, short, tdtype) in enumerate(((1.0, 0.0, False, "float32"), (2.0, 0.3, True, "float16"), (0.25, 0.95, True, "bfloat16"))):
        z, ids, teacher = inputs(torch, rng, rows, n, k, dtype, masked, short, tdtype)
        z = wider(torch, z, (0, 3, 8)[i])
        up = dev(torch, rng.standard_normal(rows).astype(np.float32)) if i else None
        check(torch, A, z, ids, teacher, t, up, scale=(1.0, 0.5, 7.0)[i])


@pytest.mark.parametrize("rows,n,dtype", [(1, 128_000, "bfloat16"), (5, 200_003, "float32"), (40, 50_001, "float16"), (1, 3_000_001, "float32")])
def test_long_rows(env, rows, n, dtype):
    torch, A, _ = env
    rng = np.random.default_rng(n)
    z, ids, teacher = inputs(torch, rng, rows, n, 50, dtype, masked=0.2)
    check(torch, A, z, ids, teacher, 1.5)


def test_in_place_and_beside(env):
    """Gradients in the scores' place, and in a wider array whose other elements stay as they were."""
    torch, A, _ = env
    rng = np.random.default_rng(7)
    for dtype, rows, n in (("float32", 6, 1003), ("bfloat16", 3, 40_001), ("float16", 700, 66)):
        z, ids, teacher = inputs(torch, rng, rows, n, 12, dtype, masked=0.1, short=True)
        _, stats, want = check(torch, A, z, ids, teacher, 2.0)
        room = wider(torch, torch.zeros_like(z), 5)
        A.ann_distill_grad(z, ids, teacher, stats, temperature=2.0, out=room)
        assert torch.equal(room, want) and (room._base[:, n:] == 77).all()
        strided = wider(torch, z, 5)
        for place in (z, strided):
            A.ann_distill_grad(place, ids, teacher, stats, temperature=2.0, out=place)
            assert torch.equal(place, want)
        assert (strided._base[:, n:] == 77).all()
    both = torch.zeros((5, 700), device="cuda")  # scores and gradients side by side in the same rows
    z, ids, teacher = inputs(torch, rng, 5, 300, 4, "float32")
    both[:, :300] = z
    _, stats, want = check(torch, A, z, ids, teacher)
    A.ann_distill_grad(both[:, :300], ids, teacher, stats, out=both[:, 350:650])
    assert torch.equal(both[:, 350:650], want) and torch.equal(both[:, :300], z)
    for out in (both[:, 299:599], both[1:, :300], both.view(-1)[200:1700].view(5, 300)):
        with pytest.raises(A.AnnError):
            A.ann_distill_grad(both[:len(out), :300], ids[:len(out)], teacher[:len(out)], stats[:len(out)], out=out)


@pytest.mark.parametrize("dtype,n", [("float32", 8193), ("float32", 20_001), ("bfloat16", 33_000)])
@pytest.mark.parametrize("k", (5, 64, 65, 200))
def test_parts_of_many_rows(env, dtype, n, k):
    """Rows of which several workgroups take a part each; the teacher's entries at the parts' ends, some named twice and more;
    beside the scores, and in their place."""
    torch, A, _ = env
    rng = np.random.default_rng(n + k)
    z, ids, teacher = inputs(torch, rng, 520, n, k, dtype, masked=0.1, short=True)
    part = 32768 // z.element_size()
    ends = [0, 1, part - 1, part, n - 1, n - 2, n // 2]
    for r in range(1, 520, 3):
        ids[r, :] = dev(torch, rng.choice(ends, k).astype(np.int32))
    z[:, ends] = dev(torch, rng.standard_normal((520, len(ends)))).to(z.dtype)
    up = dev(torch, rng.standard_normal(520).astype(np.float32))
    _, stats, want = check(torch, A, z, ids, teacher, 2.0, up)
    for _ in range(3):
        place = z.clone()
        assert torch.equal(A.ann_distill_grad(place, ids, teacher, stats, grad_losses=up, temperature=2.0, out=place), want)


def test_same_id_twice(env):
    torch, A, _ = env
    rng = np.random.default_rng(8)
    z, ids, teacher = inputs(torch, rng, 5, 300, 400, "float32")  # 400 of 300: many named twice and more
    check(torch, A, z, ids, teacher)
    ids[:] = 17
    check(torch, A, z, ids, teacher)


def test_empty_rows_and_values_that_are_no_numbers(env):
    torch, A, _ = env
    rng = np.random.default_rng(9)
    z, ids, teacher = inputs(torch, rng, 9, 500, 6, "float32")
    z[0] = -np.inf             # nothing left of the scores
    ids[1] = -1                # no teacher
    teacher[2] = -np.inf
    z[3, 100] = np.nan
    z[4, 3] = np.inf
    z[5, ids[5, 2].long()] = -np.inf   # the teacher names a masked entry
    teacher[6, 1] = np.nan
    teacher[7, 0] = np.inf
    losses, stats = A.ann_distill(z, ids, teacher)
    g = A.ann_distill_grad(z, ids, teacher, stats)
    assert (losses[:3] == 0).all() and (g[:3] == 0).all()
    assert losses[3:5].isnan().all() and g[3:5].isnan().all()
    assert losses[5] == np.inf
    _, want, _, off = plain(z[5:6].double().cpu().numpy(), ids[5:6].cpu().numpy(), teacher[5:6].double().cpu().numpy(), 1.0)
    assert (np.abs(g[5].double().cpu().numpy() - want[0]) <= off[0] + 4 * U * np.abs(want[0]) + 2.0 ** -120).all()
    assert losses[6:8].isnan().all()
    for r in (6, 7):
        named = torch.zeros(500, dtype=torch.bool, device="cuda")
        named[ids[r].long()] = True
        assert torch.equal(g[r].isnan(), named)
    check(torch, A, z[8:], ids[8:], teacher[8:])
    ids[8, 0] = 10 ** 9                 # an id that no score has
    check(torch, A, z[8:], ids[8:], teacher[8:])
    # large scores: differences alone count
    z = 1e30 * torch.randn((3, 400), device="cuda")
    check(torch, A, z, ids[:3].contiguous(), torch.zeros_like(teacher[:3]) + torch.arange(6, device="cuda"))


def test_lowest_values_as_masks(env):
    """Masks of the type's lowest number count as scores: a row of nothing else is uniform."""
    torch, A, _ = env
    for dtype in (torch.float32, torch.float16, torch.bfloat16):
        z = torch.full((2, 256), torch.finfo(dtype).min, dtype=dtype, device="cuda")
        z[1, 3] = 0.0
        ids = torch.tensor([[5, 9], [3, 3]], dtype=torch.int32, device="cuda")
        teacher = torch.zeros((2, 2), device="cuda")
        losses, stats = A.ann_distill(z, ids, teacher)
        # (1: the same id twice, half a share each: the sum of 1/2 (log 1/2 - log 1), twice)
        assert abs(losses[0].item() - np.log(128)) < 300 * U and abs(losses[1].item() + np.log(2)) < U
        g = A.ann_distill_grad(z, ids, teacher, stats).float()
        want = torch.full((256,), 2.0 ** -8, device="cuda")
        want[5] -= 0.5
        want[9] -= 0.5
        assert (g[0] - want.to(dtype).float()).abs().max() <= 2 * HALF[str(dtype).split(".")[1]] and (g[1] == 0).all()


def test_gradients_against_differences(env):
    """(f(z + h) - f(z - h)) / 2h: f is off by some 4e-6 each, which h = 2^-5 makes 1.3e-4; its third derivative, T times
    that of log-sum-exp at T / T^3, is at most 1, times h^2 / 6 1.6e-4."""
    torch, A, _ = env
    rng = np.random.default_rng(10)
    z, ids, teacher = inputs(torch, rng, 3, 60, 5, "float32")
    losses, stats = A.ann_distill(z, ids, teacher, temperature=1.0)
    g = A.ann_distill_grad(z, ids, teacher, stats)
    h = 2.0 ** -5
    for i in [*ids[0].tolist(), *range(0, 60, 7)]:
        up, down = z.clone(), z.clone()
        up[:, i] += h
        down[:, i] -= h
        d = (A.ann_distill(up, ids, teacher)[0].double() - A.ann_distill(down, ids, teacher)[0].double()) / (2 * h)
        assert (d - g[:, i]).abs().max() <= 3e-4, i


def test_offsets_beyond_32_bits(env):
    torch, A, _ = env
    rows, n = 36_000, 128_000  # 4.6e9 scores
    z = torch.zeros((rows, n), dtype=torch.float16, device="cuda")
    z[-1] = dev(torch, np.random.default_rng(1).standard_normal(n).astype(np.float16))
    ids = torch.arange(8, device="cuda").int().repeat(rows, 1) * 15_000
    teacher = torch.arange(8, device="cuda").float().repeat(rows, 1)
    losses, stats = A.ann_distill(z, ids, teacher)
    one = A.ann_distill(z[-1:].clone(), ids[-1:].contiguous(), teacher[-1:].contiguous())
    assert (losses[:-1] == losses[0]).all()
    assert abs(losses[-1].item() - one[0][0].item()) <= 2 * (n / 256 + 200) * U  # (its parts are joined in another order)
    want = A.ann_distill_grad(z[-1:].clone(), ids[-1:].contiguous(), teacher[-1:].contiguous(), stats[-1:].contiguous())
    A.ann_distill_grad(z, ids, teacher, stats, out=z)
    assert torch.equal(z[-1:], want) and torch.equal(z[0], z[-2])


def test_streams_graphs_and_repeats(env):
    torch, A, _ = env
    rng = np.random.default_rng(11)
    for rows, n in ((5, 60_000), (20, 3000)):
        z, ids, teacher = inputs(torch, rng, rows, n, 20, "bfloat16", masked=0.1)

        def chain():
            losses, stats = A.ann_distill(z, ids, teacher, temperature=2.0)
            return losses, stats, A.ann_distill_grad(z, ids, teacher, stats, temperature=2.0, scale=1 / rows)

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
            teacher.copy_(torch.roll(teacher, 1, 1))
            want = chain()
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want)), turn
