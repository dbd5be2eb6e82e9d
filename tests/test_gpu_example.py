"""The example that trains a head and drafts with it."""
import importlib.util
from pathlib import Path

import pytest

pytestmark = pytest.mark.gpu


def test_distilled_head_drafts_better():
    spec = importlib.util.spec_from_file_location("distill_head", Path(__file__).parent.parent / "examples/distill_head.py")
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    before, after, losses = example.main(steps=150)
    assert losses[-1] < 0.8 * losses[0]
    assert after[0] > before[0] and after[1] > before[1]
