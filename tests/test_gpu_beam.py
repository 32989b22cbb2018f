"""ann_beam_select and ann_beam_reorder against their definitions."""
import numpy as np
import pytest

import beam_plain as P
from helpers import dev

pytestmark = pytest.mark.gpu


def check(torch, A, z, totals, beams, k, finished=None, pad=0):
    """Beams and entries equal; totals within their rounding to fp32 and the sums' own 1e-11."""
    got = A.ann_beam_select(z, totals, beams, k, finished=finished, pad_id=pad)
    want = P.select(z.double().cpu().numpy(), totals.double().cpu().numpy(), beams, k, None if finished is None else finished.cpu().numpy(), pad)
    assert (got[0].cpu().numpy() == want[0]).all(), np.argwhere(got[0].cpu().numpy() != want[0])[:3]
    assert (got[1].cpu().numpy() == want[1]).all(), np.argwhere(got[1].cpu().numpy() != want[1])[:3]
    v = got[2].double().cpu().numpy()
    with np.errstate(all="ignore"):
        assert ((v == want[2]) | (np.abs(v - want[2]) <= 2.0 ** -24 * np.abs(want[2]) + 1e-11)).all()
    return got


def scores_of(torch, rng, rows, n, dtype, masked=0.0):
    z = 3.0 * rng.standard_normal((rows, n))
    z[rng.random((rows, n)) < masked] = -np.inf
    return dev(torch, z).to(getattr(torch, dtype))


def wider(torch, x, pad):
    wide = torch.full((x.shape[0], x.shape[1] + pad), 77, dtype=x.dtype, device=x.device)
    wide[:, :x.shape[1]] = x
    return wide[:, :x.shape[1]]


@pytest.mark.parametrize("dtype", ("float32", "float16", "bfloat16"))
@pytest.mark.parametrize("groups,beams,n,k", [(1, 1, 1, 1), (2, 3, 2, 6), (2, 1, 3, 5), (1, 64, 100, 128), (1, 1, 500, 128), (3, 4, 4096, 8), (2, 5, 4097, 10),
                                              (1, 2, 8192, 128), (5, 8, 13_000, 16), (300, 4, 50, 4), (1, 4, 128_000, 8), (7, 3, 8, 128)])
def test_sizes(env, dtype, groups, beams, n, k):
    torch, A, _ = env
    rng = np.random.default_rng(groups * n + k)
    rows = groups * beams
    for i, masked in enumerate((0.0, 0.3, 0.97)):
        z = wider(torch, scores_of(torch, rng, rows, n, dtype, masked), (0, 3, 8)[i])
        totals = dev(torch, (-3.0 * rng.random(rows)).astype(np.float32))
        finished = dev(torch, rng.random(rows) < 0.3) if i else None
        check(torch, A, z, totals, beams, k, finished, pad=min(i, n - 1))


def test_first_step_and_dead_beams(env):
    """One beam alive of each group; totals of NaN; groups without any."""
    torch, A, _ = env
    rng = np.random.default_rng(2)
    z = scores_of(torch, rng, 20, 3000, "float32")
    totals = torch.full((20,), -np.inf, device="cuda")
    totals[::5] = 0.0
    totals[7] = np.nan
    totals[15] = -np.inf
    check(torch, A, z, totals, 5, 10)
    check(torch, A, z, totals, 5, 10, finished=torch.ones(20, dtype=torch.uint8, device="cuda"), pad=2999)
    totals[3] = np.inf
    check(torch, A, z, totals, 5, 10)


@pytest.mark.parametrize("n", (100, 5000, 20_000))
def test_ties_and_orders(env, n):
    """Equal scores by id, equal beams by number, rows in order either way."""
    torch, A, _ = env
    rng = np.random.default_rng(n)
    totals = torch.zeros(4, device="cuda")
    few = dev(torch, rng.integers(0, 3, (4, n)).astype(np.float32))
    same = few[:1].repeat(4, 1)
    up = torch.arange(n, device="cuda").float().repeat(4, 1) * 0.01
    for z in (few, same, torch.zeros_like(few), up, -up, up.sin()):
        for k in (1, 7, 128):
            check(torch, A, z, totals, 4, k)
            check(torch, A, z.to(torch.bfloat16), totals, 2, k)
    # the best of many chunks all in one thread's sixteen entries, and all in one chunk
    z = torch.zeros((2, n), device="cuda")
    z[:, 8:16] = 5.0 + torch.arange(8, device="cuda")
    z[1, : min(n, 4096)] += 2.0
    check(torch, A, z, totals[:2], 2, 20)


@pytest.mark.parametrize("dtype", ("float32", "bfloat16"))
def test_many_equal_scores(env, dtype):
    """Chunks with more entries at the bound than are listed at once, of one value and of few."""
    torch, A, _ = env
    rng = np.random.default_rng(15)
    totals = dev(torch, -rng.random(6).astype(np.float32))
    for n in (3000, 4096, 9000):
        z = torch.zeros((6, n), dtype=getattr(torch, dtype), device="cuda")
        for k in (1, 5, 128):
            check(torch, A, z, totals, 3, k)
        z[:, ::3] = 1.0
        z[1, 5] = z[4, n - 1] = 2.0
        z[2, :1500] = -np.inf
        z[3] = -0.0
        for k in (2, 100):
            check(torch, A, z, totals, 2, k)


def test_values_that_are_no_numbers(env):
    torch, A, _ = env
    rng = np.random.default_rng(4)
    z = scores_of(torch, rng, 12, 9000, "float32", 0.5)
    z[0, 17] = np.inf
    z[0, 8999] = np.inf
    z[1] = -np.inf
    z[2] = np.nan
    z[3, ::2] = np.nan
    z[4:6] = torch.finfo(torch.float32).min
    z[6] = -np.inf
    z[6, 8500] = -50.0
    z[7, :4096] = -np.inf
    z[8] = 0.0
    z[8, 5] = -0.0
    z[9] *= 1e30
    totals = torch.zeros(12, device="cuda")
    for beams, k in ((1, 5), (2, 8), (12, 128)):
        check(torch, A, z, totals, beams, k)
    check(torch, A, torch.full((4, 70), -np.inf, device="cuda"), totals[:4], 2, 3)
    for dtype in (torch.float16, torch.bfloat16):
        low = torch.full((2, 300), torch.finfo(dtype).min, dtype=dtype, device="cuda")
        low[0, 7] = 1.0
        check(torch, A, low, totals[:2], 2, 6)


def test_offsets_beyond_32_bits(env):
    torch, A, _ = env
    rows, n = 36_000, 128_000
    z = torch.zeros((rows, n), dtype=torch.float16, device="cuda")
    rng = np.random.default_rng(3)
    z[-4:] = dev(torch, rng.standard_normal((4, n)).astype(np.float16))
    totals = torch.zeros(rows, device="cuda")
    got = A.ann_beam_select(z, totals, 4, 6)
    want = P.select(z[-4:].double().cpu().numpy(), np.zeros(4), 4, 6)
    assert (got[0][-1].cpu().numpy() == want[0][0]).all() and (got[1][-1].cpu().numpy() == want[1][0]).all()
    assert (got[0][:-1] == 0).all() and (got[1][:-1] == torch.arange(6, device="cuda")).all()


def test_long_rows(env):
    """The longest rows that are served."""
    torch, A, _ = env
    n = (1 << 24) - 1
    z = torch.zeros((2, n), dtype=torch.bfloat16, device="cuda")
    z[0, n - 1], z[1, 12_345_678], z[1, 3] = 9.0, 9.0, 8.0
    check(torch, A, z, torch.tensor([0.0, 0.5], device="cuda"), 2, 5)


def states_of(torch, rng, shape, dtype):
    return dev(torch, rng.integers(-100, 100, shape).astype(np.float32)).to(dtype)


def gathered(torch, states, parents, beams, dim, out):
    """The definition, row by row."""
    want = out.clone()
    for g in range(parents.shape[0]):
        for i, p in enumerate(parents[g].tolist()):
            if 0 <= p < beams:
                want.select(dim, g * parents.shape[1] + i).copy_(states.select(dim, g * beams + p))
    return want


@pytest.mark.parametrize("groups,beams,k", [(1, 1, 1), (3, 4, 4), (2, 5, 9), (4, 8, 8), (1, 12, 12), (2, 16, 3), (1, 30, 30), (2, 64, 64)])
def test_reorder(env, groups, beams, k):
    torch, A, _ = env
    rng = np.random.default_rng(groups * beams)
    parents = dev(torch, rng.integers(0, beams, (groups, k)).astype(np.int32))
    rows = groups * beams
    for shape, dim, dtype in (((rows, 7), 0, torch.float32), ((2, rows, 3, 40, 16), 1, torch.bfloat16), ((rows,), 0, torch.int8), ((3, rows, 33), 1, torch.uint8),
                              ((rows, 4096), 0, torch.float16), ((5, 2, rows, 50), 2, torch.float32)):
        states = states_of(torch, rng, shape, dtype)
        got = A.ann_beam_reorder(states, parents, beams, dim=dim)
        want = gathered(torch, states, parents, beams, dim, got)
        assert torch.equal(got, want), (shape, dim)
        if k == beams:
            A.ann_beam_reorder(states, parents, beams, dim=dim, out=states)
            assert torch.equal(states, want), (shape, dim)


@pytest.mark.parametrize("bytes_of_a_row", (4096 * 511, 4096 * 512, 4096 * 513 + 16, 4096 * 70 + 4, 1_000_003))
def test_reorder_of_long_rows(env, bytes_of_a_row):
    """Rows whose pieces take whole runs of workgroups, and not."""
    torch, A, _ = env
    rng = np.random.default_rng(bytes_of_a_row)
    states = states_of(torch, rng, (2, 6, bytes_of_a_row), torch.int8)
    parents = dev(torch, rng.integers(0, 3, (2, 3)).astype(np.int32))
    got = A.ann_beam_reorder(states, parents, 3, dim=1)
    assert torch.equal(got, gathered(torch, states, parents, 3, 1, got))
    A.ann_beam_reorder(states, parents, 3, dim=1, out=states)
    assert torch.equal(states, got)


def test_reorder_of_slices(env):
    """The used part of caches with room for more: what lies behind it stays as it was, in place and not; parents that are
    none leave their rows."""
    torch, A, _ = env
    rng = np.random.default_rng(6)
    groups, beams = 3, 4
    for dtype, width, used in ((torch.bfloat16, 64, 37), (torch.bfloat16, 7, 5), (torch.int8, 5, 3), (torch.float32, 1, 1)):
        cache = states_of(torch, rng, (2, groups * beams, 3, 50, width), dtype)
        room = states_of(torch, rng, (2, groups * beams, 3, 60, width), dtype)
        parents = dev(torch, rng.integers(0, beams, (groups, beams)).astype(np.int32))
        parents[0, 1], parents[1, 3], parents[2, 0] = -1, beams, 2 ** 31 - 1
        part = cache[:, :, :, :used]
        want = room.clone()
        want[:, :, :, :used] = gathered(torch, part, parents, beams, 1, room[:, :, :, :used])
        A.ann_beam_reorder(part, parents, beams, dim=1, out=room[:, :, :, :used])
        assert torch.equal(room, want), dtype
        want = cache.clone()
        want[:, :, :, :used] = gathered(torch, part, parents, beams, 1, part)
        A.ann_beam_reorder(part, parents, beams, dim=1, out=part)
        assert torch.equal(cache, want), dtype
    # rows that are not the slowest dimension, columns in the place of rows
    x = states_of(torch, rng, (40, groups * beams), torch.float32)
    parents.clamp_(0, beams - 1)
    assert torch.equal(A.ann_beam_reorder(x, parents, beams, dim=1), gathered(torch, x, parents, beams, 1, x))
    with pytest.raises(ValueError):
        A.ann_beam_reorder(states_of(torch, rng, (4, 3, 3, 6), torch.float32)[:, :2, :2, :3], parents[:1], 4)
    with pytest.raises(A.AnnError):
        A.ann_beam_reorder(cache[:, :, 0], parents, beams, dim=1, out=cache[:, :, 1])  # interleaved: refused
    with pytest.raises(A.AnnError):
        A.ann_beam_reorder(x[0].expand(groups * beams, groups * beams), parents, beams)  # rows that are one


def test_reorder_beyond_32_bits(env):
    torch, A, _ = env
    states = torch.zeros((2, 6, 450_000_000), dtype=torch.int8, device="cuda")  # 5.4e9 bytes
    states[1, 5, -3:] = torch.tensor([1, 2, 3], dtype=torch.int8, device="cuda")
    states[0, 3, 0] = 9
    parents = torch.tensor([[0, 2, 1], [2, 2, 0]], dtype=torch.int32, device="cuda")
    A.ann_beam_reorder(states, parents, 3, dim=1, out=states)
    want = torch.tensor([0, 0, 0, 0, 0, 9], dtype=torch.int8, device="cuda")
    assert torch.equal(states[0, :, 0], want) and (states[1, :, -3:].sum(1).tolist() == [0, 0, 0, 6, 6, 0])
    assert states.sum(dtype=torch.int64).item() == 9 + 12


def test_totals_in_place(env):
    torch, A, _ = env
    rng = np.random.default_rng(12)
    z = scores_of(torch, rng, 400, 300, "float32")
    totals = dev(torch, -rng.random(400).astype(np.float32))
    want = check(torch, A, z, totals, 4, 4)
    got = A.ann_beam_select(z, totals, 4, 4, totals_out=totals.view(100, 4))
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.equal(totals.view(100, 4), want[2])


def test_totals_of_the_last_step(env):
    torch, A, _ = env
    rng = np.random.default_rng(14)
    z = scores_of(torch, rng, 12, 300, "float32")
    finished = dev(torch, rng.random(12) < 0.3)
    _, _, totals = A.ann_beam_select(z, dev(torch, -rng.random(12).astype(np.float32)), 4, 4)
    assert totals.shape == (3, 4)
    want = A.ann_beam_select(z, totals.flatten(), 4, 4, finished=finished, pad_id=2)
    got = A.ann_beam_select(z, totals, 4, 4, finished=finished.view(3, 4), pad_id=2)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_streams_graphs_and_repeats(env):
    torch, A, _ = env
    rng = np.random.default_rng(5)
    z = scores_of(torch, rng, 15, 20_000, "float32", 0.1)
    totals = dev(torch, -rng.random(15).astype(np.float32))
    states = states_of(torch, rng, (2, 15, 300), torch.float32)

    def chain():
        parents, ids, out = A.ann_beam_select(z, totals, 5, 5)
        return parents, ids, out, A.ann_beam_reorder(states, parents, 5, dim=1)

    want = chain()
    for _ in range(3):
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
        z.copy_(torch.roll(z, 1, 0))
        want = chain()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), turn
