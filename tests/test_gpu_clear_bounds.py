"""The recurrence in the clear writes its outputs and nothing beside them, in every
form of its kernels, with last chunks of one token up to all."""
import pytest
import torch

import clear_reference as R
from gpu_helpers import need_gpu, step

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
GUARD, MARK = 1 << 20, 160.0     # bytes behind each output, and what lies there


@pytest.fixture(scope="module")
def clear():
    need_gpu()
    from paper_2608_17442_amd import clear
    return clear


class Guarded:
    """Outputs of a call, each with marks before and behind it."""

    def __init__(self):
        self.all = []

    def __call__(self, shape, dtype):
        n = 1
        for s in shape:
            n *= s
        room = GUARD // (4 if dtype == F32 else 2)
        whole = torch.full((n + 2 * room,), MARK, dtype=dtype, device="cuda")
        self.all.append((whole, room, n))
        return whole[room:room + n].view(shape)

    def check(self):
        for whole, room, n in self.all:
            assert (whole[:room] == MARK).all() and (whole[room + n:] == MARK).all()


# sequences of a last chunk of 1, 20, 31, 33 and 64 tokens: whole, in segments, long ones;
# states of one half and two; unaligned rows
SHAPES = [
    (8, 84, 24, 64, 1, 128),
    (8, 65, 24, 64, 2, 64),
    (2, 1311, 6, 64, 2, 128),
    (3, 1281, 20, 16, 1, 16),
    (2, 10964, 24, 64, 1, 128),
    (2, 10975, 24, 16, 1, 16),
    (2, 97, 4, 100, 2, 33),
    (1, 64, 2, 33, 1, 100),
    (1, 1, 3, 64, 1, 128),
]


def call(clear, shape, dtype, seed):
    b, L, H, P, G, N = shape
    f = [t.cuda() for t in R.factors(seed, *shape, dtype)]
    h0 = torch.randn(b, H, P, N, device="cuda", generator=torch.Generator("cuda").manual_seed(seed))
    return f, h0, clear._scan_plan(*f, h0)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", SHAPES)
def test_scan(clear, shape, dtype):
    step(f"scan beside its outputs {shape} {dtype}")
    f, h0, plan = call(clear, shape, dtype, 80)
    out = Guarded()
    y, h = out(plan.shapes[0], dtype), out(plan.shapes[1], F32)
    w = torch.empty(max(1, plan.space), dtype=torch.uint8, device="cuda")
    clear._check(clear._lib.fesc_clear_scan(
        plan.ref, *(t.data_ptr() for t in (*f, h0, y, h, w)), plan.space, clear._stream(0)))
    out.check()
    want, hw = R.scan(*(t.double() for t in (*f, h0)))
    assert R.rel(y, want.cpu()) <= (2.0 ** -16 if dtype == F32 else 2.0 ** -8)
    assert R.rel(h, hw.cpu()) <= 2.0 ** -16


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", [s for s in SHAPES if s[1] < 5000])
def test_scan_gradient(clear, shape, dtype):
    step(f"scan gradient beside its outputs {shape} {dtype}")
    f, h0, plan = call(clear, shape, dtype, 81)
    dy, dh = torch.randn(shape[:4], device="cuda").to(dtype), torch.randn_like(h0)
    out = Guarded()
    grads = [out(t.shape, t.dtype) for t in (*f, h0)]
    w = torch.empty(plan.grad_space, dtype=torch.uint8, device="cuda")
    clear._check(clear._lib.fesc_clear_scan_bwd(
        plan.ref, *(t.data_ptr() for t in (*f, h0, dy, dh, *grads, w)), plan.grad_space,
        clear._stream(0)))
    out.check()
    on = [t.clone().requires_grad_() for t in (*f, h0)]
    want = torch.autograd.grad(list(clear.scan(*on, return_state=True)), on, [dy, dh])
    assert all(torch.equal(a, c) for a, c in zip(grads, want))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_that_overlap(clear, dtype):
    """Factors given once for all tokens (stride 0), and rows that begin inside one another."""
    step(f"scan of broadcast tokens {dtype}")
    b, L, H, P, G, N = 2, 150, 3, 64, 1, 128
    x, la, B, C = (t.cuda() for t in R.factors(82, b, L, H, P, G, N, dtype))
    x1, B1 = x[:, :1].expand(-1, L, -1, -1), B[:, :1].expand(-1, L, -1, -1)
    assert torch.equal(clear.scan(x1, la, B1, C), clear.scan(x1.contiguous(), la, B1.contiguous(), C))
    rows = torch.randn(b, L * 8 + N, device="cuda").to(dtype)
    B2 = rows.as_strided((b, L, 1, N), (rows.stride(0), 8, N, 1))
    assert torch.equal(clear.scan(x, la, B2, C), clear.scan(x, la, B2.contiguous(), C))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", SHAPES + [(2, 200, 4, 16, 1, 16), (1, 1300, 2, 80, 2, 40)])
def test_workspaces(clear, shape, dtype):
    """Nothing beside the workspace, of exactly the size that the library names; and nothing
    of what lies in it before a call shows in the outputs."""
    step(f"scan beside its workspace {shape} {dtype}")
    f, h0, plan = call(clear, shape, dtype, 83)
    dy = torch.randn(shape[:4], device="cuda").to(dtype)
    seen = []
    for fill in (0xFF, 0x00):
        grads = [torch.empty_like(t) for t in (*f, h0)]
        y = torch.empty(plan.shapes[0], dtype=dtype, device="cuda")
        spaces = [torch.full((size + 4096,), fill, dtype=torch.uint8, device="cuda")
                  for size in (plan.space, plan.grad_space)]
        clear._check(clear._lib.fesc_clear_scan(
            plan.ref, *(t.data_ptr() for t in (*f, h0, y)), None, spaces[0].data_ptr(), plan.space,
            clear._stream(0)))
        clear._check(clear._lib.fesc_clear_scan_bwd(
            plan.ref, *(t.data_ptr() for t in (*f, h0, dy)), None,
            *(t.data_ptr() for t in (*grads, spaces[1])), plan.grad_space, clear._stream(0)))
        for space, size in zip(spaces, (plan.space, plan.grad_space)):
            assert (space[size:] == fill).all()
        seen.append([y, *grads])
    assert all(torch.equal(a, c) for a, c in zip(*seen))
