"""The example that trains a scoring head on an index's lists, run as it is used."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu


def test_a_head_learns_an_index_s_lists():
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import distill_neighbours
    losses, first = distill_neighbours.train(steps=40, items=3000, queries=200, features=130, topk=10)
    assert losses[0] > 0 and losses[-1] < 0.5 * losses[0]
    assert first > 0.5
    again, _ = distill_neighbours.train(steps=3, items=3000, queries=200, features=130, topk=10)
    assert again.tolist() == losses[:3].tolist()              # the same bits each time
