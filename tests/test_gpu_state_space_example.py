"""The state space example runs, its gradients are its losses' differences, and it serves the frames that the packed pass says."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_serves_what_it_packed():
    import packed_state_space
    losses, served, packed = packed_state_space.train(steps=3, n=40, t_blk=64, dtype=torch.float32)
    assert all(x == x for x in losses)
    # float32: the two ways add the same products in another order, some hundred terms of size 1 in each of six layers
    assert torch.allclose(served, packed, rtol=1e-3, atol=1e-3)


def test_in_half_precision():
    import packed_state_space
    losses, served, packed = packed_state_space.train(steps=3, n=40, t_blk=64, dtype=torch.bfloat16)
    assert all(x == x for x in losses)
    # eight roundings of 2^-8 in a row (norm, projection, conv, steps, B and C, scan, projection, sum), on sums of terms of random
    # sign: a few times 8 * 2^-8 of the largest answer
    assert float((served.float() - packed.float()).abs().max()) <= 0.1 * max(1.0, float(packed.float().abs().max()))


def test_gradients_are_differences():
    import packed_state_space as example
    device = torch.device("cuda")
    frames, lengths = example.recordings(30, 48, 16, torch.float32, device, seed=2)
    layer = example.Layer(16, 32, 8, 4, torch.float32, device, seed=3)
    b = example.Batch(frames, lengths, 48, seed=1)
    example.loss_of(layer, b).backward()
    g = torch.Generator(device=device).manual_seed(4)
    for i, w in enumerate(layer.weights):
        d = torch.empty_like(w).normal_(generator=g)
        d /= d.norm()
        step = 3e-2
        with torch.no_grad():
            up, down = [], []
            for sign, to in ((1, up), (-1, down)):
                w += sign * step * d
                to.append(float(example.loss_of(layer, b).double()))
                w -= sign * step * d
        rise, want = (up[0] - down[0]) / (2 * step), float((w.grad * d).sum())
        # a loss of some 1 in float32, rounded in sums of thousands of terms (2^-18 of it or so), over 2 * 3e-2; and the third
        # derivative along a unit direction, of the gradient's size, times step^2 / 6
        assert abs(rise - want) <= 2.0 ** -18 / step + 4 * step ** 2 * max(abs(want), float(w.grad.norm()) * 0.1), (i, rise, want)
