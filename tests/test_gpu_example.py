"""The example that trains the rows of an index and searches it, at a small size."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_training_brings_the_items_of_a_topic_together():
    spec = importlib.util.spec_from_file_location("train_rows", os.path.join(ROOT, "examples", "train_rows.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    first, last, share = m.train(items=4_000, topics=80, d=32, batch=512, steps=120, mine_every=30, say=None)
    # 50 items a topic: untrained rows find 1 in 80 of their own
    assert last < 0.7 * first and share > 0.5
