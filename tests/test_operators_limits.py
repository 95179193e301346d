"""Further refusals, answered on the host before anything is launched (no GPU): of the model's operators, and of more work than a
launch holds by all entry points."""
import pytest
import torch

from test_operators_refuse import EINVAL, EOVERFLOW, EWORKSPACE, F16, F32, P, bl, heads  # noqa: F401

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


def test_more_workgroups_than_a_launch_holds(bl):
    """2^24 workgroups of 256 threads and more, which is beyond the 32 bits of a launch's grid: with a few numbers beyond them only
    the rest modulo 2^24 would run, and the call would say that all is well."""
    lib, h, most = bl._lib, heads(bl), 1 << 24
    for more in (0, 5, most):
        n = most + more
        assert lib.bload_segment_mask(P, P, None, n, 1, 1, None, 0, P, None) == EOVERFLOW
        assert lib.bload_segment_mask(P, P, None, (n + 1) // 2, 1025, 1, None, 0, P, None) == EOVERFLOW
        for B, T, H in ((n, 100, 1), ((n + 15) // 16, 100, 16), ((n + 31) // 32, 129, 16)):
            assert lib.bload_segment_attention(h, h, h, P, B, T, H, 1, 64, F16, 0.1, 0.0, None, h, None, None, None) == EOVERFLOW
            assert lib.bload_segment_attention_backward(h, h, h, h, h, P, None, P, B, T, H, 1, 64, F16, 0.1, 0.0, None, h, h, h, P, BIG, None) == EOVERFLOW
        assert lib.bload_segment_attention_decode(h, h, h, P, P, P, (n + 7) // 8, 4, 100, 8, 8, 64, F16, 0.1, 0.0, None, h, P, BIG, None) == EOVERFLOW
        assert lib.bload_gated_scan(P, P, P, P, n, 1, 1024, F16, None, P, None, None, 0, None) == EOVERFLOW
        assert lib.bload_gated_scan(P, P, P, P, n, 9, 4, F16, None, P, None, None, 0, None) == EOVERFLOW
        assert lib.bload_gated_scan_backward(P, P, P, P, P, n, 1, 1024, F16, None, None, P, P, None, None, 0, None) == EOVERFLOW
        assert lib.bload_rotary(h, P, n, 1, 40, 128, F16, P, 128, 0, 1.0, 0, h, None) == EOVERFLOW


def test_more_workgroups_than_a_launch_holds_on_the_packing_path(bl):
    """The packed tensor in 4 KiB tiles is 64 GiB from there on; reductions and scans of more than 2^24 chunks."""
    lib, room = bl._lib, 1 << 50
    for n in (1 << 20, (1 << 20) + 1, 1 << 21):
        assert lib.bload_pack(P, P, P, P, P, P, P, n, n, 16, 4096, P, P, P, P, P, P, room, None) == EOVERFLOW
        assert lib.bload_pack_noalloc(P, P, P, P, P, P, P, n, n, 16, 4096, P, P, P, P, P, None) == EOVERFLOW
    B = 1 << 24
    for dtype in (0, F16, F32):
        assert lib.bload_segment_scan(P, P, P, B, 2048, 64, dtype, 0.5, P, P, room, None) == EOVERFLOW
        for T, F in ((2048, 64), (16, 16384)):
            assert lib.bload_segment_reduce(P, P, P, P, B, T, F, dtype, 0, 1000, P, P, room, None) == EOVERFLOW


def test_binding_takes_no_other_order_of_dimensions(bl):
    """A tensor of as many elements in another order is refused before it is looked at; dimensions may be taken together."""
    B, T, D = 3, 10, 16
    byte = lambda *shape: torch.zeros(shape, dtype=torch.uint8)
    word = lambda *shape: torch.zeros(shape, dtype=torch.int32)
    real = lambda *shape: torch.zeros(shape)

    def refused(t, shape, dtype):
        with pytest.raises(ValueError, match="expected shape"):
            bl._sized(t, shape, dtype, "it")

    def taken(t, shape, dtype):                              # (as far as the check of the device: these lie on the host)
        with pytest.raises(ValueError, match="expected a device tensor"):
            bl._sized(t, shape, dtype, "it")
    for t in (word(T, B, 4), word(B, 4, T), word(4, B, T), word(B, T, 3), word(B, T), word(T, B * 4)):
        refused(t, (B, T, 4), torch.int32)
    for t in (word(B, T, 4), word(B * T, 4), word(B, T * 4), word(B * T * 4), word(1, B, T, 1, 4)):
        taken(t, (B, T, 4), torch.int32)
    for t in (real(B, D, T), real(T, B, D), real(D, B * T)):
        refused(t, (B, T, D), torch.float32)
    for t in (real(B, T, D), real(B * T, D), real(B, 1, T, D)):
        taken(t, (B, T, D), torch.float32)
    refused(byte(T, B), (B, T), torch.uint8)
    taken(byte(B, T), (B, T), torch.uint8)
    refused(real(D, B), (B, D), torch.float32)
    taken(real(B, 1, D), (B, D), torch.float32)
    assert bl._sized(None, (B, T), torch.uint8, "it") == 0
