"""The example that trains a small model around the layer and serves it from 4-bit values."""
import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("storage", ["f32", "bf16"])
def test_train_and_serve(storage):
    import torch
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import train_and_serve as example
    got = example.run(storage, 200, say=lambda *a: print(*a, flush=True))
    assert got["losses"][-1] < 0.1 * got["losses"][0]
    assert got["own"] > 0.8 and got["served"] > got["own"] - 0.25        # ten of a hundred topics have lost a label
    for lab in (got["first"], got["second"]):
        assert (lab >= 0).all() and not torch.isin(lab, got["forbidden"]).any()
    shown = (got["first"][:, :, None] == got["second"][:, None, :]).any()
    assert not shown                                                     # the penalty is larger than any difference of scores here
    assert torch.equal(got["values"], got["adjusted"].gather(1, got["second"].long()))
