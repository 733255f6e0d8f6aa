"""The draft-head example runs end to end and learns in every stage."""
import math
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_draft_head_example():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import draft_head
    finally:
        sys.path.pop(0)
    from paper_2602_05774_gb300 import build, vsd
    build.build_library()
    vsd.load()
    got = draft_head.train(rows=256, vocab=2000, hidden=128, steps=20, log=lambda *_: None)
    for name, (first, last) in got.items():
        assert math.isfinite(last) and last < first, (name, first, last)
    # an untrained head is near the uniform distribution's cross entropy
    assert abs(got["labels"][0] - math.log(2000)) < 0.5
    # the last stage goes on from the loss that the one before reached
    assert abs(got["logits"][0] - got["teacher"][1]) < 0.1 * got["teacher"][0]
