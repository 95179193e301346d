"""Calls of the norms, the short convolution and the selective scan at the edges of what their documentation allows."""
import pytest
import torch

import operators_reference as ref
from gpu_util import binding

pytestmark = pytest.mark.gpu


# the longest rows that a team holds, and rows beyond the registers, of one row and of several to a share of the columns' sums
@pytest.mark.parametrize("dtype,T,D", [("f16", 3, 16384), ("f16", 3, 20001), ("bf16", 7, 16391), ("f32", 5, 8192), ("f32", 3, 8197),
                                       ("f32", 1500, 8195)])
@pytest.mark.parametrize("center", [False, True])
def test_norm_gradients_in_the_place_of_what_they_come_from(dtype, T, D, center):
    """dx in the place of dout or dsum: the weights' gradients are still those of dout."""
    print(f"norm in place T={T} D={D} {dtype} center {center}", flush=True)
    bl = binding()
    x, dy, ds = (torch.randn((1, T, D), device="cuda").to(ref.TORCH[dtype]) for _ in range(3))
    w = torch.randn(D, device="cuda")
    valid = (torch.rand((1, T), device="cuda") < 0.8).to(torch.uint8)
    valid[0, 0] = 1
    _, stats = bl.bload_layer_norm(x, w, valid=valid, center=center, training=True)
    want = bl.bload_layer_norm_backward(dy, x, stats, w, valid=valid, dsum=ds, center=center)
    for place in (0, 1):
        a, b = dy.clone(), ds.clone()
        to = ((a, b)[place], torch.empty_like(w), torch.empty_like(w))
        bl.bload_layer_norm_backward(a, x, stats, w, valid=valid, dsum=b, center=center, grads=to)
        for name, got, there in zip(("dx", "dweight", "dbias"), to, want):
            assert torch.equal(got, there), (name, ("dout", "dsum")[place])
