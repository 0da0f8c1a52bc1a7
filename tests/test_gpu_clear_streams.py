"""Inputs of a call on another stream may be dropped when it returns: their memory is not
handed out again while the stream may still read it."""
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


def factors():
    return [t.cuda() for t in R.factors(120, 3, 100, 4, 64, 1, 64, BF16)]


def calls(clear):
    f = factors()
    h = torch.randn(3, 4, 64, 64, device="cuda")
    m = torch.randn(500, 768, device="cuda").to(BF16)
    w = torch.ones(768, device="cuda", dtype=BF16)
    return {
        "scan": (clear.scan, [*f, h]),
        "scan_step": (clear.scan_step, [*(t[:, 0].contiguous() for t in f), h]),
        "norm_gated": (clear.norm_gated, [m, m.clone(), m.clone(), w, w.clone()]),
        "norm_residual": (clear.norm_residual, [m, m.clone(), w, w.clone()]),
    }


@pytest.mark.parametrize("name", ["scan", "scan_step", "norm_gated", "norm_residual"])
def test_inputs_dropped_behind_a_call(clear, name):
    step(f"inputs of {name} dropped")
    f, ts = calls(clear)[name]
    want = f(*(t.clone() for t in ts))
    side = torch.cuda.Stream()
    for i in range(len(ts)):
        args = [t.clone() for t in ts]
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)            # some ten milliseconds of work before it
        got = f(*args, stream=side)
        at, shape, dtype = args[i].data_ptr(), args[i].shape, args[i].dtype
        args[i] = None
        again = torch.full(shape, 7.0, dtype=dtype, device="cuda")
        assert again.data_ptr() != at, i
        torch.cuda.synchronize()
        for a, b in zip(*((t,) if torch.is_tensor(t) else t for t in (got, want))):
            assert torch.equal(a, b), i


def test_saved_inputs_of_a_gradient(clear):
    step("gradient on another stream")
    f = factors()
    dy = torch.randn(f[0].shape, device="cuda").to(BF16)
    on = [t.clone().requires_grad_() for t in f]
    want = torch.autograd.grad(clear.scan(*on), on, dy)
    side = torch.cuda.Stream()
    leaves = [t.clone().requires_grad_() for t in f]
    args = [t * 1 for t in leaves]
    torch.cuda.synchronize()
    y = clear.scan(*args, stream=side)
    del args                                        # only the graph holds on to them
    torch.cuda.current_stream().wait_stream(side)
    got = torch.autograd.grad(y, leaves, dy)
    del y
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
