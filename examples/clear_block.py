"""The block in the clear, end to end: train it, then serve it token by token.

One block of the shape whose linear work the library carries under encryption
(residual and norm, projections, gated linear recurrence, skip, gate and norm,
projection back) learns to predict a slowly moving signal from its past, and
is then run as a server runs it: the prompts at once, each further token by
`scan_step` on a pool of states.

    python examples/clear_block.py [--steps 60] [--batch 8] [--length 512]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2608_17442_amd import clear  # noqa: E402


class Block:
    """d_model features, `heads` heads of `head_dim` channels, one group of
    `d_state` state entries."""

    def __init__(self, d_model=64, heads=4, head_dim=32, d_state=64, dtype=torch.bfloat16, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.heads, self.head_dim, self.d_state = heads, head_dim, d_state
        E = heads * head_dim
        self.split = [E, E, d_state, d_state, heads]          # z, x, B, C, decay logits

        def weight(*shape, scale):
            w = scale * torch.randn(*shape, generator=g, device="cuda")
            return w.to(dtype).requires_grad_()

        def full(n, value):
            return torch.full((n,), value, device="cuda", dtype=dtype).requires_grad_()

        self.w_in = weight(d_model, sum(self.split), scale=d_model ** -0.5)
        self.w_out = weight(E, d_model, scale=E ** -0.5)
        self.norm_in, self.scale = full(d_model, 1.0), full(d_model, 1.0)
        self.norm_out, self.skip = full(E, 1.0), full(E, 1.0)

    def parameters(self):
        return [self.w_in, self.w_out, self.norm_in, self.scale, self.norm_out, self.skip]

    def factors(self, u):
        """Gate and the recurrence's factors of the normed input: slices of one
        projection, which the calls read where they lie."""
        z, x, B, C, dt = (u @ self.w_in).split(self.split, -1)
        la = -torch.nn.functional.softplus(dt - 2.0)          # log decays, <= 0
        heads = (self.heads, self.head_dim)
        return z, x, x.unflatten(-1, heads), la, B.unsqueeze(-2), C.unsqueeze(-2)

    def leave(self, y, x, z):
        return clear.norm_gated(y.flatten(-2), x, z, self.skip, self.norm_out) @ self.w_out

    def __call__(self, o, r, h0=None):
        """o: the output of the layer before, r: the residual stream
        [batch, len, d_model].  Returns the block's output, the new stream and
        the state after the last token."""
        r, u = clear.norm_residual(o, r, self.scale, self.norm_in)
        z, x, xh, la, B, C = self.factors(u)
        y, h = clear.scan(xh, la, B, C, h0=h0, return_state=True)
        return self.leave(y, x, z), r, h

    @torch.no_grad()
    def step(self, o, r, pool, slots):
        """One token of each row: o, r [rows, d_model]; states in place."""
        r, u = clear.norm_residual(o, r, self.scale, self.norm_in)
        z, x, xh, la, B, C = self.factors(u)
        y = clear.scan_step(xh, la, B, C, pool, slots=slots)
        return self.leave(y, x, z), r


def signal(batch, length, d_model, dtype, seed):
    """Sums of three slow waves with noise, their features a random projection."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    t = torch.arange(length + 1, device="cuda")[None, :, None]
    f = 0.02 + 0.2 * torch.rand(batch, 1, 3, generator=g, device="cuda")
    p = 6.28 * torch.rand(batch, 1, 3, generator=g, device="cuda")
    w = torch.sin(f * t + p)
    g.manual_seed(12345)
    mix = torch.randn(3, d_model, generator=g, device="cuda")
    return (w @ mix).to(dtype)


def train(block, steps, batch, length, lr=3e-3):
    """Predict the next features; returns the first and the last loss."""
    master = [p.detach().float() for p in block.parameters()]
    moment = [(torch.zeros_like(m), torch.zeros_like(m)) for m in master]
    losses = []
    for k in range(steps):
        s = signal(batch, length, block.w_in.shape[0], block.w_in.dtype, seed=k)
        past = s[:, :-1].contiguous()
        out, r, _ = block(past, torch.zeros_like(past))
        loss = (r + out - s[:, 1:]).float().square().mean()
        grads = torch.autograd.grad(loss, block.parameters())
        losses.append(loss.item())
        with torch.no_grad():
            for p, m, (a, b), d in zip(block.parameters(), master, moment, grads):
                d = d.float()
                a.lerp_(d, 0.1)
                b.lerp_(d * d, 0.01)
                rate = lr * (1 - 0.99 ** (k + 1)) ** 0.5 / (1 - 0.9 ** (k + 1))
                m.addcdiv_(a, b.sqrt().add_(1e-8), value=-rate)
                p.copy_(m)
    return losses[0], losses[-1]


@torch.no_grad()
def serve(block, batch, prompt, tokens):
    """Prompts at once, then token by token from a pool in another order; the
    largest difference from the outputs of the whole sequences at once,
    relative to their root mean square."""
    s = signal(batch, prompt + tokens, block.w_in.shape[0], block.w_in.dtype, seed=1000003)
    s = s[:, :-1].contiguous()
    zero = torch.zeros_like(s)
    whole, _, _ = block(s, zero)
    first, _, h = block(s[:, :prompt].contiguous(), zero[:, :prompt].contiguous())
    pool = torch.zeros(batch + 2, *h.shape[1:], device="cuda")
    slots = torch.randperm(batch + 2, device="cuda")[:batch].to(torch.int32)
    pool[slots.long()] = h
    outs = [first]
    for t in range(prompt, prompt + tokens):
        o, _ = block.step(s[:, t], zero[:, t], pool, slots)
        outs.append(o[:, None])
    d = (torch.cat(outs, 1) - whole).float().abs().max()
    return (d / whole.float().square().mean().sqrt()).item()


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--batch", type=int, default=8)
    ap.add_argument("--length", type=int, default=512)
    a = ap.parse_args()
    block = Block()
    first, last = train(block, a.steps, a.batch, a.length)
    print(f"loss {first:.4f} -> {last:.4f} in {a.steps} steps")
    d = serve(block, a.batch, 100, 40)
    print(f"served token by token: at most {d:.2g} rms from the pass over whole sequences (bfloat16)")


if __name__ == "__main__":
    main()
