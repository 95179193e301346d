"""The model's operators at the edges of what their callers may do, on the GPU."""
import numpy as np
import pytest
import torch

import operators_reference as ref
from gpu_util import binding, to_dev

pytestmark = pytest.mark.gpu


# rows that are no whole number of a lane's elements: their last lane and its neighbour meet at the borders of wavefronts and workgroups
@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("B,T,D", [(130, 1, 9), (200, 1, 37), (130, 1, 81), (130, 1, 257), (130, 1, 1025), (2, 1, 2049), (130, 8, 9),
                                   (130, 3, 81), (300, 1, 3), (130, 2, 40)])
def test_gated_state_in_place(B, T, D, dtype):
    """A state that is advanced where it lies, and its gradient, bit for bit as from one buffer to another."""
    print(f"gated in place B={B} T={T} D={D} {dtype}", flush=True)
    bl = binding()
    rng = np.random.default_rng([B, T, D])
    gate, x, w = (ref.draw(rng, (B, T, D), dtype).cuda() for _ in range(3))
    gate = gate.sigmoid()
    reset, valid = (to_dev((rng.random((B, T)) < p).astype(np.uint8)) for p in (0.1, 0.9))
    state, dstate = (torch.from_numpy(rng.standard_normal((B, D)).astype(np.float32)).cuda() for _ in range(2))
    h, last = bl.bload_gated_scan(gate, x, reset, valid, h0=state)
    dgate, dx, dh0 = bl.bload_gated_scan_backward(w, gate, h, reset, valid, h0=state, dstate=dstate)
    here, there = state.clone(), dstate.clone()
    h_in_place, same = bl.bload_gated_scan(gate, x, reset, valid, h0=here, state=here)
    assert same is here and torch.equal(h_in_place, h) and torch.equal(here, last)
    grads = torch.empty_like(dgate), torch.empty_like(dx), there
    bl.bload_gated_scan_backward(w, gate, h, reset, valid, h0=state, dstate=there, grads=grads)
    assert torch.equal(grads[0], dgate) and torch.equal(grads[1], dx) and torch.equal(there, dh0)
