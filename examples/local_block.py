#!/usr/bin/env python3
"""A layer of a gated linear recurrence and one of local attention on the
package's operators, as models that alternate them would use them: packed
prompts of unequal length, then token by token from the caches they leave, and
training steps.

    [v, f, a] = x W_in;  u = short_conv(v);  h = gated_scan(u, f, a)
    z = x + h W_mid
    [q, k, v] = z W_qkv;  q, k = norm_rotate(q, k);  y = window_attention(q, k, v)
    out = z + y W_out

  python examples/local_block.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1908_06649_gb300 as tcu  # noqa: E402


class Block:
    """Projections in bf16, the operators' parameters in fp32."""

    def __init__(self, width=128, channels=192, heads=4, kv_heads=2, dim=32, window=24, sinks=2,
                 taps=4, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def randn(*shape, scale=1.0, shift=0.0, dtype=torch.bfloat16):
            v = torch.randn(*shape, generator=gen, device="cuda") * scale + shift
            return v.to(dtype).requires_grad_()

        f32 = torch.float32
        self.heads, self.kv_heads, self.dim = heads, kv_heads, dim
        self.seen = {"window": window, "sinks": sinks}
        self.w_in = randn(width, 3 * channels, scale=width ** -0.5)
        self.w_mid = randn(channels, width, scale=channels ** -0.5)
        self.w_qkv = randn(width, (heads + 2 * kv_heads) * dim, scale=width ** -0.5)
        self.w_out = randn(heads * dim, width, scale=(heads * dim) ** -0.5)
        self.taps = randn(channels, taps, scale=taps ** -0.5, dtype=f32)
        self.log_rate = randn(channels, scale=0.5, shift=-2.0, dtype=f32)
        self.q_weight = randn(dim, scale=0.1, shift=1.0, dtype=f32)
        self.k_weight = randn(dim, scale=0.1, shift=1.0, dtype=f32)
        self.rates = 10000.0 ** (-torch.arange(dim // 2, device="cuda", dtype=f32) / (dim // 2))

    def parameters(self):
        return [self.w_in, self.w_mid, self.w_qkv, self.w_out, self.taps, self.log_rate,
                self.q_weight, self.k_weight]

    def _heads(self, z):
        h, kv = self.heads, self.kv_heads
        qkv = (z @ self.w_qkv).unflatten(-1, (h + 2 * kv, self.dim))
        return qkv.split([h, kv, kv], -2)

    def _turned(self, q, k, **where):
        return tcu.norm_rotate(q, k, self.rates, q_weight=self.q_weight, k_weight=self.k_weight,
                               **where)

    def prompt(self, x, offsets=None):
        """x (rows, width) with offsets, or (batch, length, width): the outputs,
        the recurrence's caches, and the rows that attention's are filled from."""
        v, f, a = (x @ self.w_in).chunk(3, -1)
        u, taps = tcu.short_conv(v, self.taps, silu=True, offsets=offsets)
        h, state = tcu.gated_scan(u, f, a, self.log_rate.exp(), offsets=offsets)
        z = x + h @ self.w_mid
        q, k, v = self._heads(z)
        q, k = self._turned(q, k, offsets=offsets)
        y = tcu.window_attention(q, k, v, offsets=offsets, **self.seen)
        return z + y.flatten(-2) @ self.w_out, (taps, state), (k, v)

    @torch.no_grad()
    def caches(self, entries, held, rows, offsets, slots):
        """Entries of all caches, those at slots from prompts."""
        taps, state = (torch.zeros(entries, *t.shape[1:], dtype=t.dtype, device="cuda") for t in held)
        taps[slots.long()], state[slots.long()] = held
        seen = self.seen["window"] + self.seen["sinks"]
        kv = torch.zeros(2, entries, seen, self.kv_heads, self.dim, dtype=torch.bfloat16, device="cuda")
        tcu.window_cache(*rows, *kv.unbind(0), offsets=offsets, slots=slots, **self.seen)
        return taps, state, kv

    @torch.no_grad()
    def token(self, x, caches, positions, slots):
        """x (batch, width): one more row of every sequence, caches in place."""
        taps, state, kv = caches
        v, f, a = (x @ self.w_in).chunk(3, -1)
        u = tcu.short_conv_step(v, taps, self.taps, silu=True, slots=slots)
        h = tcu.gated_scan_step(u, f, a, self.log_rate.exp(), state, slots=slots)
        z = x + h @ self.w_mid
        q, k, v = self._heads(z)
        q, k = self._turned(q, k, positions=positions)
        y = tcu.window_attention_step(q, k, v, *kv.unbind(0), positions, slots=slots, **self.seen)
        return z + y.flatten(-2) @ self.w_out


def offsets_of(lengths):
    return torch.tensor([0, *torch.tensor(lengths).cumsum(0).tolist()], dtype=torch.int32, device="cuda")


def serve(block, lengths=(5, 64, 1, 130), more=6, width=128):
    """Prompts of unequal length at once, then their next tokens; the same rows
    as whole prompts give the same outputs.  Returns how far they are apart,
    relative to their norm."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    rows = [torch.randn(n + more, width, generator=gen, device="cuda").bfloat16() for n in lengths]
    with torch.no_grad():
        whole, _, _ = block.prompt(torch.cat(rows), offsets_of([n + more for n in lengths]))
        want = torch.stack([w[-more:] for w in whole.split([n + more for n in lengths])], 1)
        off = offsets_of(lengths)
        _, held, kv = block.prompt(torch.cat([r[:n] for r, n in zip(rows, lengths)]), off)
        slots = torch.tensor([6, 0, 3, 5], dtype=torch.int32, device="cuda")
        caches = block.caches(7, held, kv, off, slots)
        place = off.diff()
        got = []
        for t in range(more):
            x = torch.stack([r[n + t] for r, n in zip(rows, lengths)])
            got.append(block.token(x, caches, place + t, slots))
    got = torch.stack(got).float()
    return ((got - want.float()).norm() / want.float().norm()).item()


def train(block, steps=20, width=128):
    """Learns to give the row before the last; returns the first and last loss."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    params, losses = block.parameters(), []
    optimizer = torch.optim.Adam(params, lr=3e-3)
    for _ in range(steps):
        x = torch.randn(4, 96, width, generator=gen, device="cuda").bfloat16()
        out, _, _ = block.prompt(x)
        loss = (out[:, 1:].float() - x[:, :-1].float()).square().mean()
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        losses.append(loss.item())
    return losses[0], losses[-1]


if __name__ == "__main__":
    print("tokens against whole prompts: relative difference %.1e" % serve(Block()))
    print("training: loss %.3f -> %.3f" % train(Block()))
