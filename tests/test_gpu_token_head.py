"""The example that trains a token encoder's head, quantises it and searches its tokens (run on an MI355X)."""
from __future__ import annotations

import os
import sys

import pytest

pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_trained_head_finds_the_passages():
    """Training has to separate the passages: from a few per cent found to nearly all."""
    import token_head

    before, after = token_head.main(["--steps", "150"])
    assert before < 0.3 and after > 0.9
