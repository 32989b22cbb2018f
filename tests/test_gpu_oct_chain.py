"""The calls on 8-bit rows, distillation and beam steps as a program runs them together."""
import numpy as np
import pytest

import beam_plain as B
import oct_plain as P
from helpers import dev
from test_gpu_distill import check as check_distill

pytestmark = pytest.mark.gpu


def test_a_training_step(env):
    """Embeddings under a teacher whose neighbours a search has named: scores by 8-bit rows, loss, and the gradients of both
    sides through the quantised products; every link against its own definition."""
    torch, A, _ = env
    rng = np.random.default_rng(1)
    n, d, nx, k, t = 700, 96, 90, 10, 0.5
    points = dev(torch, rng.standard_normal((n, d)).astype(np.float32))
    asked = points[:nx] + 0.1 * dev(torch, rng.standard_normal((nx, d)).astype(np.float32))
    graph = A.ann_build(points, R=16, L=32, alpha=1.2)
    ids, dists = A.ann_search(graph, points, asked, k=k, L=40)
    x, w = dev(torch, (rng.standard_normal((nx, d)) / 4).astype(np.float32)), dev(torch, (rng.standard_normal((n, d)) / 4).astype(np.float32))
    scores = A.ann_oct_product(A.ann_oct_quantize(x), A.ann_oct_quantize(w))
    losses, _, grads = check_distill(torch, A, scores, ids, -0.05 * dists, t, scale=1 / nx)
    dx = A.ann_oct_product(A.ann_oct_quantize(grads), A.ann_oct_quantize(w, columns=True))
    dw = A.ann_oct_product(A.ann_oct_quantize(grads, columns=True), A.ann_oct_quantize(x, columns=True))
    assert losses.isfinite().all() and (losses > 0).any()

    def values(a):
        a = a.double().cpu().numpy()
        return P.values(*P.quantize(a), a.shape[1])

    for got, left, right in ((dx, values(grads), values(w.T)), (dw, values(grads.T), values(x.T))):
        bound = left.shape[1] * 2.0 ** -23 * (np.abs(left) @ np.abs(right).T) + 2.0 ** -140
        assert (np.abs(got.double().cpu().numpy() - left @ right.T) <= bound).all()
    # quantising costs at most 2^-4 of a value (and what is below a step's range): the direction stays
    exact = grads.double() @ w.double()
    assert torch.nn.functional.cosine_similarity(dx.double().flatten(), exact.flatten(), dim=0) > 0.99


def test_a_decoder_step(env):
    """Scores of an output layer of 8-bit rows, the beams that go on, their states in order in place; three steps, replayed from
    a graph as well, against the steps one by one."""
    torch, A, _ = env
    rng = np.random.default_rng(2)
    groups, beams, n, d = 3, 4, 5000, 256
    rows = A.ann_oct_quantize(dev(torch, rng.standard_normal((n, d)).astype(np.float32)))
    table = P.values(rows.codes.cpu().numpy(), rows.scales.cpu().numpy(), d)
    first = dev(torch, rng.standard_normal((groups * beams, d)).astype(np.float32))
    state, totals = first.clone(), torch.zeros(groups * beams, device="cuda")
    totals.view(groups, beams)[:, 1:] = -np.inf
    begin = totals.clone()

    def step():
        scores = A.ann_oct_product(A.ann_oct_quantize(state), rows)
        parents, ids, best = A.ann_beam_select(scores, totals, beams, beams)
        A.ann_beam_reorder(state, parents, beams, out=state)
        state.add_(0.01 * ids.view(-1, 1).float().sin())
        totals.copy_(best.view(-1))
        return scores, parents, ids

    seen = []
    for _ in range(3):
        before, old = totals.clone(), state.clone()
        scores, parents, ids = step()
        q = P.values(*P.quantize(old.double().cpu().numpy()), d)
        bound = d * 2.0 ** -23 * (np.abs(q) @ np.abs(table).T)
        assert (np.abs(scores.double().cpu().numpy() - q @ table.T) <= bound).all()
        want = B.select(scores.double().cpu().numpy(), before.double().cpu().numpy(), beams, beams)
        assert (parents.cpu().numpy() == want[0]).all() and (ids.cpu().numpy() == want[1]).all()
        seen.append((parents, ids, totals.clone(), state.clone()))
    state.copy_(first)
    totals.copy_(begin)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _, parents, ids = step()
    for want in seen:
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((parents, ids, totals, state), want))
