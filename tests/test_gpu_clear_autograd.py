"""What the block in the clear has no derivative for is refused, not dropped."""
import pytest
import torch
from torch.autograd import forward_ad

import clear_reference as R
from gpu_helpers import need_gpu, step

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def clear():
    need_gpu()
    from paper_2608_17442_amd import clear
    return clear


def calls(clear):
    """Each call as a function of its tensors, and the tensors."""
    x, la, B, C = (t.cuda() for t in R.factors(110, 2, 5, 2, 16, 1, 32, BF16))
    h = torch.randn(2, 2, 16, 32, device="cuda")
    m, r = (torch.randn(3, 24, device="cuda").to(BF16) for _ in range(2))
    w = torch.ones(24, device="cuda", dtype=BF16)
    return {
        "scan": (lambda *a: clear.scan(*a), [x, la, B, C, h]),
        "scan_step": (lambda *a: clear.scan_step(*a),
                      [x[:, 0], la[:, 0], B[:, 0], C[:, 0], h.clone()]),
        "norm_gated": (lambda *a: clear.norm_gated(*a), [m, r, m, w, w]),
        "norm_residual": (lambda *a: clear.norm_residual(*a)[1], [m, r, w, w]),
    }


NAMES = ["scan", "scan_step", "norm_gated", "norm_residual"]


@pytest.mark.parametrize("name", NAMES)
def test_tangents_are_refused(clear, name):
    step(f"tangents into {name}")
    f, ts = calls(clear)[name]
    f(*ts)
    with forward_ad.dual_level():
        f(*ts)                              # none of them has one
        for i in range(len(ts)):
            args = list(ts)
            args[i] = forward_ad.make_dual(ts[i], torch.ones_like(ts[i]))
            with pytest.raises(NotImplementedError):
                f(*args)
            with pytest.raises(NotImplementedError), torch.no_grad():
                f(*args)


@pytest.mark.parametrize("name", ["scan", "norm_gated", "norm_residual"])
def test_tangents_of_gradients_are_refused(clear, name):
    step(f"tangents into the gradient of {name}")
    f, ts = calls(clear)[name]
    on = [t.detach().requires_grad_() for t in ts]
    with forward_ad.dual_level():
        y = f(*on)
        d = forward_ad.make_dual(torch.ones_like(y), torch.ones_like(y))
        with pytest.raises(NotImplementedError):
            torch.autograd.grad(y, on, d)


@pytest.mark.parametrize("name", NAMES)
def test_traces_are_refused(clear, name):
    step(f"trace of {name}")
    f, ts = calls(clear)[name]
    with pytest.raises(NotImplementedError):
        torch.jit.trace(f, tuple(ts), check_trace=False)
