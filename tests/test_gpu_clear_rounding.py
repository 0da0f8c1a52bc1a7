"""bfloat16 outputs of the recurrence in the clear: computed in 32 bits, rounded
once.

Tolerance (2-norm of the error over that of the answer): the rounding of an
output moves it by at most half a unit of its eight bits, 2^-9 of itself, and so
their 2-norm; what comes before it is held in 32 bits, or in two bfloat16 parts
(2^-18), and sums to less than 2^-16 of the terms.
"""
import pytest
import torch

import clear_reference as R
from gpu_helpers import need_gpu, step

pytestmark = pytest.mark.gpu

ONCE = 2.0 ** -9 + 2.0 ** -16
BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def clear():
    need_gpu()
    from paper_2608_17442_amd import clear
    return clear


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
    e = R.rel(y, want.cpu())
    assert e <= ONCE, f"y: off by {e:.4g}, allowed {ONCE:.4g}"
