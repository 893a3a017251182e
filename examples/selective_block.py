#!/usr/bin/env python3
"""A sequence-mixing block on the package's operators, as a model would use
them: packed prompts of unequal length, then token by token from the caches
they leave, then a training step.  Last, the case in which nothing varies with
the position, where the scan is a causal convolution and the DFT plans compute
the same result.

    x (rows, width) -> [v, g] = x W_in;  u = short_conv(v)
    [dt, B, C] = u W_x (dt through a low rank);  y = state_scan(u, dt, A, B, C, gate g)
    out = y W_out

  python examples/selective_block.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1908_06649_gb300 as tcu  # noqa: E402


class Block:
    """Projections in bf16, the operators' parameters in fp32."""

    def __init__(self, width=256, channels=512, states=16, rank=16, taps=4, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def randn(*shape, scale=1.0, dtype=torch.bfloat16):
            v = torch.randn(*shape, generator=gen, device="cuda") * scale
            return v.to(dtype).requires_grad_()

        f32 = torch.float32
        self.sizes = (rank, states)
        self.w_in = randn(width, 2 * channels, scale=width ** -0.5)
        self.w_x = randn(channels, rank + 2 * states, scale=channels ** -0.5)
        self.w_dt = randn(rank, channels, scale=rank ** -0.5)
        self.w_out = randn(channels, width, scale=channels ** -0.5)
        self.taps = randn(channels, taps, scale=taps ** -0.5, dtype=f32)
        self.tap_bias = randn(channels, scale=0.1, dtype=f32)
        rate = torch.arange(1, states + 1, device="cuda", dtype=f32).expand(channels, states)
        self.rate = rate.log().clone().requires_grad_()  # A = -exp(rate)
        self.skip = torch.ones(channels, device="cuda").requires_grad_()
        self.dt_bias = torch.full((channels,), -4.0, device="cuda").requires_grad_()

    def parameters(self):
        return [self.w_in, self.w_x, self.w_dt, self.w_out, self.taps, self.tap_bias, self.rate,
                self.skip, self.dt_bias]

    def _selective(self, u):
        rank, n = self.sizes
        dt, B, C = (u @ self.w_x).split([rank, n, n], -1)
        return dt @ self.w_dt, -torch.exp(self.rate), B, C

    def prompt(self, x, offsets=None):
        """x (rows, width) with offsets, or (batch, length, width): the outputs
        and the caches that `token` continues from."""
        v, g = (x @ self.w_in).chunk(2, -1)
        u, taps = tcu.short_conv(v, self.taps, self.tap_bias, silu=True, offsets=offsets)
        dt, A, B, C = self._selective(u)
        y, state = tcu.state_scan(u, dt, A, B, C, skip=self.skip, gate=g, dt_bias=self.dt_bias,
                                  softplus=True, offsets=offsets)
        return y @ self.w_out, (taps, state)

    @torch.no_grad()
    def token(self, x, caches, slots=None):
        """x (batch, width): one more row of every sequence, caches in place."""
        v, g = (x @ self.w_in).chunk(2, -1)
        u = tcu.short_conv_step(v, caches[0], self.taps, self.tap_bias, silu=True, slots=slots)
        dt, A, B, C = self._selective(u)
        y = tcu.state_scan_step(u, dt, A, B, C, caches[1], skip=self.skip, gate=g,
                                dt_bias=self.dt_bias, softplus=True, slots=slots)
        return y @ self.w_out


def serve(block, width=256):
    """Prompts of unequal length at once, then their next tokens; the same rows
    as whole prompts give the same outputs."""
    lengths, more = [5, 64, 1, 130], 6
    gen = torch.Generator(device="cuda").manual_seed(1)
    rows = [torch.randn(n + more, width, generator=gen, device="cuda").bfloat16() for n in lengths]
    whole = [block.prompt(r[None])[0][0] for r in rows]
    offsets = torch.tensor([0] + lengths, device="cuda").cumsum(0).to(torch.int32)
    with torch.no_grad():
        y, caches = block.prompt(torch.cat([r[:n] for r, n in zip(rows, lengths)]), offsets)
    worst = 0.0
    for i, n in enumerate(lengths):
        part = y[offsets[i]:offsets[i + 1]]
        worst = max(worst, float((part - whole[i][:n].detach()).abs().max()))
    for t in range(more):
        y = block.token(torch.stack([r[n + t] for r, n in zip(rows, lengths)]), caches)
        for i, n in enumerate(lengths):
            worst = max(worst, float((y[i] - whole[i][n + t].detach()).abs().max()))
    scale = max(float(w.detach().abs().max()) for w in whole)
    return worst / scale


def train(block, width=256, steps=8, rate=0.02):
    """Gradient steps towards a fixed target; returns the first and last loss."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(4, 96, width, generator=gen, device="cuda").bfloat16()
    target = torch.randn(4, 96, width, generator=gen, device="cuda") * 0.1
    losses = []
    for _ in range(steps):
        y, _ = block.prompt(x)
        loss = (y.float() - target).square().mean()
        losses.append(float(loss.detach()))
        grads = torch.autograd.grad(loss, block.parameters())
        with torch.no_grad():
            for p, g in zip(block.parameters(), grads):
                p -= (rate * g.float() / (g.float().norm() + 1e-12) * p.float().norm()).to(p.dtype)
    return losses[0], losses[-1]


def invariant(channels=64, rows=2048, states=16):
    """Constant d, B and C: the scan against the causal convolution with
    K_t = sum_n C[n] exp(d A[n] t) d B[n] by DFTs of 2 rows = 16^3 points."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    u = torch.randn(channels, rows, generator=gen, device="cuda")
    A = -torch.rand(channels, states, generator=gen, device="cuda") - 0.1
    B, C = (torch.randn(states, generator=gen, device="cuda") for _ in range(2))
    d = 0.05
    same = lambda v: v.expand(1, rows, 1, states)  # noqa: E731
    y, _ = tcu.state_scan(u.T[None].contiguous(), torch.full((1, rows, channels), d, device="cuda"),
                          A, same(B).contiguous(), same(C).contiguous())
    t = torch.arange(rows, device="cuda")
    K = (C * B * d * torch.exp(d * A[:, None] * t[:, None])).sum(-1)  # (channels, rows)
    plan = tcu.Plan(2 * rows, channels, 16, tcu.X3TF32)
    pad = lambda v: torch.cat([v, torch.zeros_like(v)], -1).to(torch.complex64)  # noqa: E731
    by_dft = plan.inverse(plan.forward(pad(u)) * plan.forward(pad(K)))
    plan.check()
    want = by_dft.reshape(channels, 2 * rows)[:, :rows].real
    return float((y[0].T - want).norm() / want.norm())


def main():
    block = Block()
    print("prompts and tokens against whole prompts: %.1e of the largest output" % serve(block))
    print("training: loss %.4f -> %.4f" % train(block))
    print("nothing varying, scan against DFT convolution: relative L2 %.1e" % invariant())


if __name__ == "__main__":
    main()
