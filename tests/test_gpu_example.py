"""The example that runs the operators on dense rows together: it learns, and more beams find better answers."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_distill_and_search():
    spec = importlib.util.spec_from_file_location("distill_and_search", os.path.join(ROOT, "examples", "distill_and_search.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    first, last, score, greedy = example.main(["--vocabulary", "1501", "--steps", "150", "--length", "6"])
    assert last < 0.7 * first
    assert bool((score[:, :-1] >= score[:, 1:]).all())
    # a wide search is not always better than a narrow one, but it is over several prompts
    assert float(score[:, 0].sum()) >= float(greedy[:, 0].sum()) - 1e-4
