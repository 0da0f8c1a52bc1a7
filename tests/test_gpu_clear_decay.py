"""The gradient of log decays where decays are strong, judged by itself.

In a head or at a token with a decay of e^-20 the gradient is some e^-20 of what
it is elsewhere; a norm over all of it would not see whether it is right.  Each
class of tokens is compared by its own norm.  Tolerances: every term that the
sum has carries the decay, so the result is as exact as a sum of fp32 products,
2^-16 of its norm; in bfloat16 the rounding of the right answer comes on top.
"""
import pytest
import torch

import clear_reference as R
from gpu_helpers import need_gpu, step

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
DECAYS = (-0.01, -1.0, -5.0, -10.0, -20.0)


@pytest.fixture(scope="module")
def clear():
    need_gpu()
    from paper_2608_17442_amd import clear
    return clear


def gradient(clear, la, dtype, P, N, seed):
    """dla of both, with states in and out; la [len, heads]."""
    L, H = la.shape
    x, _, B, C = R.factors(seed, 2, L, H, P, 1, N, dtype)
    g = torch.Generator().manual_seed(seed + 1)
    h0 = torch.randn(2, H, P, N, generator=g)
    dy = torch.randn(2, L, H, P, generator=g).to(dtype)
    dh = torch.randn(2, H, P, N, generator=g)
    la = la.to(dtype).expand(2, -1, -1).contiguous()
    on = [t.cuda().requires_grad_() for t in (x, la, B, C, h0)]
    got = torch.autograd.grad(clear.scan(*on, return_state=True), on[1], [dy.cuda(), dh.cuda()])[0]
    leaves = [t.double().requires_grad_() for t in (x, la, B, C, h0)]
    want = torch.autograd.grad(list(R.scan(*leaves)), leaves[1], [dy.double(), dh.double()])[0]
    return got.cpu(), want


def check(got, want, dtype, what):
    allowed = 2.0 ** -16
    if dtype == BF16:
        allowed = R.rel(want.to(BF16), want) + 2 * allowed
    e = R.rel(got, want)
    assert e <= allowed, f"{what}: off by {e:.4g}, allowed {allowed:.4g}"


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("L", [64, 150])
@pytest.mark.parametrize("P,N", [(64, 128), (33, 20)])
def test_heads_of_one_decay(clear, dtype, L, P, N):
    step(f"dla head by head {dtype} {L} {P} {N}")
    la = torch.tensor(DECAYS).expand(L, -1)
    got, want = gradient(clear, la, dtype, P, N, 70)
    for h, d in enumerate(DECAYS):
        check(got[..., h], want[..., h], dtype, f"head of la = {d}")


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_strong_decays_between_weak_ones(clear, dtype):
    step(f"dla of strong tokens {dtype}")
    L, every = 150, 7
    la = torch.full((L, len(DECAYS) - 1), DECAYS[0])
    for h, d in enumerate(DECAYS[1:]):
        la[h::every, h] = d
    got, want = gradient(clear, la, dtype, 64, 128, 72)
    for h, d in enumerate(DECAYS[1:]):
        strong = la[:, h] == d
        check(got[:, strong, h], want[:, strong, h], dtype, f"tokens of la = {d}")
        check(got[:, ~strong, h], want[:, ~strong, h], dtype, f"tokens beside la = {d}")
