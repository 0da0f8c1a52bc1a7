"""A reset (la = -inf) forgets a state that is not finite, as it forgets any other."""
import math

import pytest
import torch

import clear_reference as R
from gpu_helpers import need_gpu, step

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def clear():
    need_gpu()
    from paper_2608_17442_amd import clear
    return clear


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_slot_is_taken_over(clear, dtype, bad):
    step(f"step after {bad} {dtype}")
    x, la, B, C = (t[:, 0].cuda() for t in R.factors(90, 3, 1, 4, 64, 2, 128, dtype))
    la[1] = -math.inf
    good = torch.randn(3, 4, 64, 128, device="cuda")
    state = good.clone()
    state[1] = bad
    y, want = clear.scan_step(x, la, B, C, state), clear.scan_step(x, la, B, C, good)
    assert torch.equal(y, want) and torch.equal(state, good)


# whole; in segments, joined on entry and by the kernel of its own; two channel tiles
@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", [(8, 84, 24, 64, 1, 128), (2, 500, 6, 64, 2, 128),
                                   (1, 2000, 4, 64, 1, 64), (2, 150, 2, 100, 1, 33)])
@pytest.mark.parametrize("at", [0, 70])
def test_a_state_is_forgotten(clear, dtype, shape, at, bad):
    """Outputs behind the reset, the final state and the gradients of what lies behind it
    are those of a finite state."""
    if at >= shape[1]:
        pytest.skip("no such token")
    step(f"scan after {bad} {shape} {dtype} reset at {at}")
    b, L, H, P, G, N = shape
    x, la, B, C = (t.cuda() for t in R.factors(91, *shape, dtype))
    la[:, at] = -math.inf
    good = torch.randn(b, H, P, N, device="cuda")
    dy = torch.randn(b, L, H, P, device="cuda").to(dtype)
    dh = torch.randn_like(good)

    def run(h0):
        on = [t.detach().clone().requires_grad_() for t in (x, la, B, C, h0)]
        y, h = clear.scan(*on, return_state=True)
        return [y.detach(), *torch.autograd.grad([y, h], on, [dy, dh])[:4]], h.detach()

    (got, h), (want, hw) = run(torch.full_like(good, bad)), run(good)
    assert torch.equal(h, hw)
    for n, a, c in zip(("y", "dx", "dla", "dB", "dC"), got, want):
        assert torch.equal(a[:, at:], c[:, at:]), n
        assert torch.isfinite(a[:, at:]).all(), n
    assert torch.equal(got[1], want[1]) and torch.equal(got[3], want[3])   # dx, dB: no state in them


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_gradient_is_forgotten(clear, dtype):
    """An incoming gradient of the final state that is not finite ends at a reset."""
    step(f"gradient behind a reset {dtype}")
    b, L, H, P, G, N = shape = (2, 200, 3, 64, 1, 128)
    f = [t.cuda() for t in R.factors(92, *shape, dtype)]
    f[1][:, 100] = -math.inf
    h0 = torch.randn(b, H, P, N, device="cuda")
    dy = torch.randn(b, L, H, P, device="cuda").to(dtype)

    def run(dh):
        on = [t.detach().clone().requires_grad_() for t in (*f, h0)]
        return torch.autograd.grad(list(clear.scan(*on, return_state=True)), on, [dy, dh])

    got, want = run(torch.full_like(h0, math.nan)), run(torch.randn_like(h0))
    for n, a, c in zip(("dx", "dla", "dB", "dC"), got, want):
        assert torch.equal(a[:, :100], c[:, :100]), n
    assert torch.equal(got[4], want[4])
