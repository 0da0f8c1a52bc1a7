"""Layouts of the recurrence's tensors that are nobody's choice: gradients as a
consumer of y leaves them, strides of dimensions of one entry."""
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


def test_gradient_of_a_time_major_consumer(clear):
    """y.transpose(0, 1).contiguous() hands back a gradient whose tokens lie further apart
    than any input's may."""
    step("time-major gradient of a large batch")
    b, L, H, P, N = 2800, 3, 24, 64, 16
    assert b * H * P > clear._MOST_TOKEN_STRIDE
    f = [t.cuda() for t in R.factors(100, b, L, H, P, 1, N, BF16)]
    dy = torch.randn(L, b, H, P, device="cuda").to(BF16)
    on = [t.requires_grad_() for t in f]
    got = torch.autograd.grad(clear.scan(*on).transpose(0, 1).contiguous(), on, dy)
    want = torch.autograd.grad(clear.scan(*on), on, dy.transpose(0, 1).contiguous())
    assert all(torch.equal(a, c) for a, c in zip(got, want))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_strides_of_single_tokens_and_sequences(clear, dtype):
    step(f"strides of dimensions of one entry {dtype}")
    H, P, N = 2, 16, 32
    far = clear._MOST_TOKEN_STRIDE + 8

    def apart(t, dim):
        s = list(t.stride())
        s[dim] = far if dim else (1 << 40) + 8
        return t.as_strided(t.shape, s)

    for b, L, dim in ((3, 1, 1), (1, 70, 0)):
        f = [t.cuda() for t in R.factors(101, b, L, H, P, 1, N, dtype)]
        odd = [apart(t, dim) for t in f]
        dy = torch.randn(b, L, H, P, device="cuda").to(dtype)
        on, at = ([t.detach().requires_grad_() for t in ts] for ts in (f, odd))
        y, z = clear.scan(*on), clear.scan(*at)
        assert torch.equal(y, z)
        for a, c in zip(torch.autograd.grad(z, at, apart(dy, dim)), torch.autograd.grad(y, on, dy)):
            assert torch.equal(a, c)
    # one row of a batch of single tokens
    x, la, B, C = (t[:, 0].cuda() for t in R.factors(102, 1, 1, H, P, 1, N, dtype))
    s1, s2 = torch.zeros(2, 1, H, P, N, device="cuda").unbind(0)
    far_rows = [apart(t, 0) for t in (x, la, B, C)]
    assert torch.equal(clear.scan_step(x, la, B, C, s1), clear.scan_step(*far_rows, s2))
    assert torch.equal(s1, s2)


def test_many_short_sequences(clear):
    """More sequences than fit a launch of one work item per state entry."""
    step("many short sequences")
    b, L, H, P, N = 30000, 2, 24, 64, 128
    f = [t.cuda() for t in R.factors(103, 100, L, H, P, 1, N, BF16)]
    many = [t.repeat(b // 100, *[1] * (t.dim() - 1)) for t in f]
    y = clear.scan(*many).unflatten(0, (b // 100, 100))
    assert (y == clear.scan(*f)).all()


def test_sizes_past_32_bits_are_refused(clear):
    """Tensors of 2^32 + 3 tokens or states that take no memory."""
    step("sizes past 32 bits")
    n = (1 << 32) + 3
    one = torch.zeros(1, device="cuda")
    x = one.expand(1, n, 1, 1)
    with pytest.raises(ValueError, match="2\\^32"):
        clear.scan(x, x[..., 0], x, x)
    row = torch.zeros(1, 1, 1, device="cuda")
    with pytest.raises(ValueError, match="2\\^32"):
        clear.scan_step(row, row[..., 0], row, row, one.expand(n, 1, 1, 1))
