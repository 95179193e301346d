"""Further refusals of the model's operators, answered on the host before anything is launched (no GPU)."""
import torch

from test_operators_refuse import EINVAL, EWORKSPACE, F16, P, bl  # noqa: F401

BIG = 1 << 40


def test_gated_states_that_meet(bl):
    """In one buffer where blocks are short, else apart: a state that another workgroup has advanced already is not the one
    that was handed in.  (States that lie apart get as far as the workspace, which is too small.)"""
    B, D = 4, 64
    size = 4 * B * D

    def forward(a, b, T):
        return bl._lib.bload_gated_scan(P, P, P, P, B, T, D, F16, a, P, b, P, 1, None)

    def backward(a, b, T):
        return bl._lib.bload_gated_scan_backward(P, P, P, P, P, B, T, D, F16, P, a, P, P, b, P, 1, None)

    def backward_state(a, b, T):
        return bl._lib.bload_gated_scan_backward(P, P, P, P, P, B, T, D, F16, a, P, P, P, b, P, 1, None)
    assert bl.bload_gated_scan_workspace_bytes(B, 5000, D, torch.float16) > 1
    for f in (forward, backward, backward_state):
        for t in (9, 5000):
            assert f(BIG, BIG, t) == f(BIG, BIG + size - 4, t) == f(BIG + 4, BIG, t) == EINVAL
        for t in (1, 8):
            assert f(BIG, BIG + 4, t) == f(BIG + size - 4, BIG, t) == EINVAL
        assert f(BIG, BIG + size, 5000) == f(BIG + size, BIG, 5000) == f(BIG, None, 5000) == EWORKSPACE
