"""bfloat16 outputs of the recurrence in the clear: computed in 32 bits, rounded
once.

Tolerance: with w the answer in 64 bits, w + d what is formed in 32 bits (or in
two bfloat16 parts, within 2^-18) and |d| <= 2^-16 |w| in the 2-norm, the
distance of a value to the nearest bfloat16 number moves by no more than the
value, so |round(w + d) - w| <= |round(w) - w| + 2 |d|.  A second rounding on the
way adds as much again as the first.
"""
import pytest
import torch

import clear_reference as R
from gpu_helpers import need_gpu, step

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def clear():
    need_gpu()
    from paper_2608_17442_amd import clear
    return clear


def check_once(got, want, what):
    want = want.double().cpu()
    allowed = R.rel(want.to(BF16), want) + 2 * 2.0 ** -16
    e = R.rel(got, want)
    assert e <= allowed, f"{what}: off by {e:.4g}, allowed {allowed:.4g}"


def inputs(seed, shape, state):
    b, L, H, P, G, N = shape
    f = [t.cuda() for t in R.factors(seed, *shape, BF16, resets=[L // 2])]
    g = torch.Generator().manual_seed(seed + 1)
    return f, torch.randn(b, H, P, N, generator=g).cuda() if state else None


# whole sequences, segments, segments of two channel tiles; states that fill
# one and two halves; rows at any alignment
SHAPES = [
    (1, 64, 2, 64, 1, 128),
    (2, 130, 3, 64, 1, 64),
    (8, 200, 24, 64, 1, 128),
    (2, 700, 6, 64, 2, 128),
    (2, 5500, 24, 64, 1, 128),
    (2, 5500, 24, 64, 1, 32),
    (2, 333, 4, 100, 2, 33),
    (1, 150, 2, 33, 1, 100),
]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("state", [False, True])
def test_scan_rounds_once(clear, shape, state):
    step(f"scan rounds once {shape} state={state}")
    f, h0 = inputs(60, shape, state)
    y = clear.scan(*f, h0=h0, return_state=state)
    y = y[0] if state else y
    want = R.scan(*(t.double() for t in f), None if h0 is None else h0.double())[0]
    check_once(y, want, "y")


GRAD_SHAPES = [
    (1, 64, 2, 64, 1, 128),
    (2, 130, 3, 64, 1, 64),
    (2, 700, 6, 64, 2, 128),
    (1, 1300, 24, 64, 1, 128),
    (2, 333, 4, 100, 2, 33),
    (1, 150, 2, 33, 1, 100),
]


@pytest.mark.parametrize("shape", GRAD_SHAPES)
@pytest.mark.parametrize("state", [False, True])
def test_scan_gradient_rounds_once(clear, shape, state):
    step(f"scan gradient rounds once {shape} state={state}")
    f, h0 = inputs(64, shape, state)
    b, L, H, P, G, N = shape
    g = torch.Generator().manual_seed(65)
    dy = torch.randn(b, L, H, P, generator=g).to(BF16).cuda()
    on = [t.requires_grad_() for t in f + ([h0] if state else [])]
    got = torch.autograd.grad(clear.scan(*on), on, dy)
    leaves = [t.detach().double().requires_grad_() for t in on]
    want = torch.autograd.grad(R.scan(*leaves)[0], leaves, dy.double())
    for n, a, w in zip(("dx", "dla", "dB", "dC"), got, want):
        check_once(a, w, n)
