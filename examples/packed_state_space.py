"""A state space layer on packed blocks, from ragged recordings to streams that are served frame by frame.

    python examples/packed_state_space.py [steps]

Recordings of unequal length are planned and packed into blocks; a layer of a norm, a short causal convolution and a selective scan
beside a residual stream learns to say each recording's next frame; then all recordings are answered again as streams would ask: one
frame at a time, with the convolution's last inputs and the scan's state advanced where they lie.  Neither a neighbour in the block
nor padding reaches a recording on either way.
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from packed_layer import Batch, recordings  # noqa: E402
from paper_2310_10879_amd import bload  # noqa: E402


class Norm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, valid):
        y, stats = bload.bload_layer_norm(x, weight, bias, valid=valid, training=True)
        ctx.save_for_backward(x, stats, weight, valid)
        return y

    @staticmethod
    def backward(ctx, dout):
        x, stats, weight, valid = ctx.saved_tensors
        return (*bload.bload_layer_norm_backward(dout.contiguous(), x, stats, weight, valid=valid), None)


class Conv(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, reset, valid):
        ctx.save_for_backward(x, weight, bias, reset, valid)
        return bload.bload_segment_conv(x, weight, reset, valid, bias=bias, silu=True)[0]

    @staticmethod
    def backward(ctx, dout):
        x, weight, bias, reset, valid = ctx.saved_tensors
        dx, dweight, dbias, _ = bload.bload_segment_conv_backward(dout.contiguous(), x, weight, reset, valid, bias=bias, silu=True)
        return dx, dweight, dbias, None, None


class Scan(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, dt, rate, b, c, skip, z, dt_bias, reset, valid):
        y, _, saved = bload.bload_selective_scan(x, dt, rate, b, c, reset, valid, skip=skip, z=z, dt_bias=dt_bias, training=True)
        ctx.save_for_backward(x, dt, rate, b, c, skip, z, dt_bias, reset, valid, saved)
        return y

    @staticmethod
    def backward(ctx, dout):
        x, dt, rate, b, c, skip, z, dt_bias, reset, valid, saved = ctx.saved_tensors
        return (*bload.bload_selective_scan_backward(dout.contiguous(), x, dt, rate, b, c, reset, valid, saved, skip=skip, z=z,
                                                     dt_bias=dt_bias)[:8], None, None)


class Layer:
    """x + out(scan(conv(u)), z) with u, z = in(norm(x)).  What is per feature stays in 32 bits, the projections have the frames' type."""

    def __init__(self, feat: int, inner: int, states: int, taps: int, dtype: torch.dtype, device, seed: int = 0):
        g = torch.Generator(device=device).manual_seed(seed)
        self.inner, self.states, self.dtype = inner, states, dtype

        def normal(*shape, std):
            return torch.empty(shape, device=device).normal_(std=std, generator=g).requires_grad_()
        self.scale, self.shift = torch.ones(feat, device=device).requires_grad_(), torch.zeros(feat, device=device).requires_grad_()
        self.into = normal(feat, 2 * inner, std=feat ** -0.5)
        self.taps, self.taps_bias = normal(inner, taps, std=taps ** -0.5), torch.zeros(inner, device=device).requires_grad_()
        self.say = normal(inner, 2 * states, std=inner ** -0.5)              # B and C
        self.steps = normal(inner, inner, std=0.1 * inner ** -0.5)
        self.steps_bias = torch.full((inner,), -3.0, device=device).requires_grad_()
        self.log_rate = torch.log(1.0 + torch.arange(states, device=device)).repeat(inner, 1).requires_grad_()
        self.skip = torch.ones(inner, device=device).requires_grad_()
        self.out = normal(inner, feat, std=inner ** -0.5)
        self.weights = [self.scale, self.shift, self.into, self.taps, self.taps_bias, self.say, self.steps, self.steps_bias, self.log_rate,
                        self.skip, self.out]

    def forward(self, x, reset, valid):
        """[B, T, feat] -> the same."""
        cast = lambda w: w.to(self.dtype)
        u, z = (Norm.apply(x, self.scale, self.shift, valid) @ cast(self.into)).split(self.inner, 2)
        u = Conv.apply(u, self.taps, self.taps_bias, reset, valid)
        b, c = (u @ cast(self.say)).unflatten(2, (1, -1)).split(self.states, 3)
        y = Scan.apply(u, u @ cast(self.steps), -torch.exp(self.log_rate), b, c, self.skip, z, self.steps_bias, reset, valid)
        return x + y @ cast(self.out)

    @torch.no_grad()
    def step(self, x, fresh, live, last_inputs, state):
        """One frame [n, 1, feat] of n streams; fresh: it is a stream's first; live: there is one.  States are advanced in place."""
        cast = lambda w: w.to(self.dtype)
        u, z = (bload.bload_layer_norm(x, self.scale, self.shift, valid=live) @ cast(self.into)).split(self.inner, 2)
        u, _ = bload.bload_segment_conv(u, self.taps, fresh, live, bias=self.taps_bias, silu=True, state_in=last_inputs, state=last_inputs)
        b, c = (u @ cast(self.say)).unflatten(2, (1, -1)).split(self.states, 3)
        y, _ = bload.bload_selective_scan(u, u @ cast(self.steps), -torch.exp(self.log_rate), b, c, fresh, live, skip=self.skip, z=z,
                                          dt_bias=self.steps_bias, h0=state, state=state)
        return x + y @ cast(self.out)


def loss_of(layer: Layer, b: Batch) -> torch.Tensor:
    said = layer.forward(b.x, b.reset, b.valid)
    goes_on = (b.valid[:, 1:] == 1) & (b.reset[:, 1:] == 0)
    return (said[:, :-1].float() - b.x[:, 1:].float())[goes_on].square().mean()


def serve(layer: Layer, frames, lengths):
    """The recordings' answers [n, longest, feat], asked one frame at a time by all of them together."""
    n, longest = len(lengths), int(lengths.max())
    first = torch.cumsum(lengths.long(), 0) - lengths
    last_inputs = frames.new_zeros((n, layer.taps.shape[1] - 1, layer.inner))
    state = torch.zeros((n, layer.inner, layer.states), device=frames.device)
    said = frames.new_zeros((n, longest, frames.shape[1]))
    for t in range(longest):
        live = (lengths > t).to(torch.uint8)[:, None]
        x = frames[(first + t).clamp(max=len(frames) - 1)][:, None]
        said[:, t] = layer.step(x, torch.full_like(live, t == 0), live, last_inputs, state)[:, 0] * live
    return said


def train(steps: int = 40, n: int = 60, t_blk: int = 96, feat: int = 32, dtype: torch.dtype = torch.bfloat16, rate: float = 3e-3):
    """Losses of the steps, and the streams' answers beside the packed ones, frame by frame of every recording."""
    device = torch.device("cuda")
    frames, lengths = recordings(n, t_blk, feat, dtype, device)
    layer = Layer(feat, 2 * feat, 16, 4, dtype, device)
    adam = torch.optim.Adam(layer.weights, lr=rate)
    losses = []
    for step in range(steps):
        b = Batch(frames, lengths, t_blk, seed=step)                             # another order of the blocks every time
        loss = loss_of(layer, b)
        adam.zero_grad()
        loss.backward()
        adam.step()
        losses.append(loss.detach())
    with torch.no_grad():
        packed = layer.forward(b.x, b.reset, b.valid).flatten(0, 1)
        first = b.plan.block_of_seq.long() * t_blk + b.plan.offset_of_seq
        at = torch.arange(int(lengths.max()), device=device)
        live = at[None, :] < lengths[:, None]
        packed = packed[torch.where(live, first[:, None] + at[None, :], 0)]
        return [float(x) for x in losses], serve(layer, frames, lengths)[live], packed[live]


if __name__ == "__main__":
    losses, served, packed = train(int(sys.argv[1]) if len(sys.argv) > 1 else 40)
    for i in range(0, len(losses), 10):
        print(f"step {i:4d}  loss {losses[i]:.4f}")
    print(f"step {len(losses) - 1:4d}  loss {losses[-1]:.4f}")
    print(f"all frames, served against packed: off by {float((served.float() - packed.float()).abs().max()):.4f} "
          f"of {float(packed.float().abs().max()):.4f}")
