"""The graph's search in the example finds most of the neighbours that the search over all 4-bit rows gives."""
import os
import sys

import pytest

from conftest import ROOT

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("seed", (1, 2, 3))
def test_recall_of_the_example(env, seed):
    """5,000 rows in 64 clusters: 0.80 to 0.81 for these seeds.  What is missing is what 4 bits move among the ten nearest;
    rows at random would share 0.002."""
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import draw_neighbours
    recall = draw_neighbours.main(["--n", "5000", "--d", "100", "--nq", "37", "--k", "10", "--seed", str(seed)])[0]
    assert recall >= 0.7
