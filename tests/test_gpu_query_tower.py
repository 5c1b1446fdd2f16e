"""The operators together, as examples/query_tower.py uses them: training brings a tower's query vectors to their base vectors, and
the search finds these."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


def test_training_a_query_tower():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "query_tower.py")
    spec = importlib.util.spec_from_file_location("query_tower", path)
    tower = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(tower)
    first, last, before, after = tower.main(steps=150, tokens=500, n=5000)
    # untrained: about 100 of 5000 by chance, and vectors a unit apart; trained: every token has a row of its own to learn one vector with
    assert before[0] < 0.2 and last < 0.2 * first
    assert after[0] > 0.9 and after[1] > 0.9
