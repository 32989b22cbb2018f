"""The example that takes the calls on 4-bit rows, the graph and the draw together."""
import os
import sys

import pytest

from conftest import ROOT

pytestmark = pytest.mark.gpu


def test_draw_neighbours(env):
    torch, _, _ = env
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import draw_neighbours
    recall, near, drawn, logprobs, scores = draw_neighbours.main(["--n", "5000", "--d", "100", "--nq", "37", "--k", "10"])
    assert 0.0 < recall <= 1.0
    # only the ten best of each question can be drawn
    tenth = torch.topk(scores, 10, dim=1).values[:, -1]
    assert (scores.gather(1, drawn.long().unsqueeze(1)).squeeze(1) >= tenth).all()
    assert (logprobs <= 0).all() and near > scores.mean().item()
