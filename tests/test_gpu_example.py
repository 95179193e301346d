"""The example trains through the operators, and serves the frames that the packed pass says."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_packed_layer_learns_and_serves():
    import packed_layer
    losses, served, packed = packed_layer.train(steps=40, n=60, t_blk=96, dtype=torch.float32)
    assert losses[-1] < 0.5 * losses[0], losses
    # float32: the two ways add the same products in another order, some hundred terms of size 1 in each of four layers
    assert torch.allclose(served, packed, rtol=1e-3, atol=1e-3)
    assert torch.isfinite(packed).all()


def test_packed_layer_in_half_precision():
    import packed_layer
    losses, served, packed = packed_layer.train(steps=10, n=60, t_blk=96, dtype=torch.bfloat16)
    assert losses[-1] < losses[0], losses
    # a chain of eight roundings of 2^-8 each (projection, turn, attention, mix, gate, state in, state out, answer), on sums of 64 terms of
    # random sign: a few times 8 * 2^-8 of the largest answer
    assert float((served.float() - packed.float()).abs().max()) <= 0.1 * max(1.0, float(packed.float().abs().max()))
