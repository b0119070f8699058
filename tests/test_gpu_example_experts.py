"""The example of a mixture of experts: a token alone and in the prompt gives the same bits, the balance bias empties the fullest expert,
the router's steps lower the loss."""
import os
import runpy

import pytest

EXAMPLE = os.path.join(os.path.dirname(os.path.abspath(__file__)), os.pardir, "examples", "experts.py")


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", [dict(tokens=96, experts=16, chosen=3, width=256, hidden=176), dict(tokens=512, experts=64, chosen=8, width=512, hidden=352)])
def test_example(sizes):
    out = runpy.run_path(EXAMPLE)["run"](**sizes, say=lambda line: None)
    assert out["same"]
    assert out["fullest"][1] < out["fullest"][0]
    assert out["losses"][-1] < out["losses"][0]
