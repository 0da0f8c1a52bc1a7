"""The block in the clear from its definitions, token by token, in 64 bits on
the CPU (differentiable through torch's autograd), and the inputs its tests
share."""
import math

import torch


def scan(x, la, B, C, h0=None):
    b, L, H, P = x.shape
    G, N = B.shape[2:]
    S = x.new_zeros(b, H, P, N) if h0 is None else h0
    ys = []
    for t in range(L):
        Bt, Ct = (v[:, t].repeat_interleave(H // G, 1) for v in (B, C))
        # a reset forgets exactly (0 times the old state)
        S = la[:, t].exp()[..., None, None] * S + x[:, t, :, :, None] * Bt[:, :, None, :]
        ys.append((S * Ct[:, :, None, :]).sum(-1))
    return (torch.stack(ys, 1) if ys else x), S


def norm(v, w, eps):
    return v / torch.sqrt((v * v).mean(-1, keepdim=True) + eps) * w


def gated(m, x, z, skip, w, eps):
    return norm((m + skip * x) * z / (1 + torch.exp(-z)), w, eps)


def residual(o, r, scale, w, eps):
    v = r + scale * o
    return v, norm(v, w, eps)


def factors(seed, b, L, H, P, G, N, dtype, resets=()):
    """x, la, B, C on the CPU in `dtype`; decays from strong to a memory of
    hundreds of tokens, head by head."""
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)
    rate = torch.logspace(-2.5, 0.3, H)
    la = (-torch.nn.functional.softplus(r(b, L, H)) * rate).to(dtype)
    for t in resets:
        la[:, t] = -math.inf
    return r(b, L, H, P).to(dtype), la, r(b, L, G, N).to(dtype), r(b, L, G, N).to(dtype)


def rel(got, want):
    """2-norm of the difference over the 2-norm of the right answer."""
    got, want = got.detach().double().cpu(), want.detach().double()
    assert got.shape == want.shape, (got.shape, want.shape)
    if want.numel() == 0:
        return 0.0
    assert torch.isfinite(got).all()
    n = want.norm().item()
    d = (got - want).norm().item()
    return d / n if n else d
