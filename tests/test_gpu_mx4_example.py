"""The example that runs the backbone's blocks together: tuning brings its states nearer, adapters learn from the cache it fills."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_backbone_example_runs_and_learns():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import mx4_backbone
    finally:
        sys.path.pop(0)
    said = []
    tuned, losses = mx4_backbone.main(say=said.append)
    assert len(said) == 2 and all(v == v for v in tuned + losses)
    assert tuned[-1] < tuned[0] and sum(losses[-4:]) < sum(losses[:4])
