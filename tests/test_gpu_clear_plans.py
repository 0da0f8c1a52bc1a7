"""Plans are kept by the values that they follow from."""
import pytest
import torch

from gpu_helpers import need_gpu, step

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["norm_gated", "norm_residual"])
def test_eps_in_a_tensor(name):
    need_gpu()
    from paper_2608_17442_amd import clear
    step(f"eps of {name} in a tensor")
    a = torch.randn(5, 40, device="cuda")
    w = torch.ones(40, device="cuda")
    ins = (a, a, a, w, w) if name == "norm_gated" else (a, a, w, w)
    f = getattr(clear, name)
    eps = torch.tensor(1e-5)
    for value in (1e-5, 1.0, 100.0):
        eps.fill_(value)
        got, want = f(*ins, eps=eps), f(*ins, eps=float(eps))
        for g, v in zip(*((t,) if torch.is_tensor(t) else t for t in (got, want))):
            assert torch.equal(g, v), value
