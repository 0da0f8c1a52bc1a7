"""The block in the clear against its definitions in 64 bits.

Tolerances (2-norm of the error over that of the answer):
* float32 outputs, and states in either type: a path to an output sums some
  hundreds of products in fp32, whose rounding errors, 2^-24 each, add up to
  less than 2^-16 of the terms.
* bfloat16 outputs: two roundings lie on a path, that of an operand (the
  state, or the matrix of decays) and that of the output.  Each is off by at
  most 2^-8 of a value and by half of that in the mean over many, so 2^-8 for
  both; of fewer than 16 values, where no mean is taken, 2^-7.
"""
import math

import pytest
import torch

import clear_reference as R
from gpu_helpers import need_gpu, step

pytestmark = pytest.mark.gpu

TOL = {torch.float32: 2.0 ** -16, torch.bfloat16: 2.0 ** -8}
STATE_TOL = 2.0 ** -16
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def clear():
    need_gpu()
    from paper_2608_17442_amd import clear
    return clear


def dev(*ts):
    return [None if t is None else t.cuda() for t in ts]


def wide(*ts):
    return [None if t is None else t.double() for t in ts]


def check(got, want, dtype, what):
    e = R.rel(got, want)
    state = what in ("h", "dh0")
    assert str(got.dtype) == str(F32 if state else dtype), what
    tol = STATE_TOL if state else TOL[dtype]
    if not state and dtype == BF16 and want.numel() < 16:
        tol = 2.0 ** -7
    assert e <= tol, f"{what}: off by {e:.3g}, allowed {tol:.3g}"


# b, L, H, P, G, N: lengths around the chunk of 64 and over several segments,
# channels and states that fill their tiles, end inside them, or take two
SHAPES = [
    (1, 1, 1, 1, 1, 1),
    (2, 1, 4, 64, 1, 128),
    (1, 2, 2, 16, 2, 16),
    (2, 63, 2, 64, 1, 64),
    (1, 64, 3, 32, 3, 48),
    (2, 65, 2, 65, 1, 33),
    (1, 129, 4, 100, 2, 100),
    (1, 200, 2, 128, 1, 128),
    (1, 1000, 2, 64, 1, 128),
    (3, 333, 6, 64, 2, 72),
]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("state", [False, True])
def test_scan(clear, shape, dtype, state):
    step(f"scan {shape} {dtype} state={state}")
    b, L, H, P, G, N = shape
    f = R.factors(1, *shape, dtype, resets=[L // 2] if L > 100 else [])
    h0 = torch.randn(b, H, P, N, generator=torch.Generator().manual_seed(2)) if state else None
    got = clear.scan(*dev(*f), h0=None if h0 is None else h0.cuda(), return_state=state)
    want, hw = R.scan(*wide(*f, h0))
    y, h = got if state else (got, None)
    check(y, want, dtype, "y")
    if state:
        check(h, hw, dtype, "h")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("state", [False, True])
def test_scan_gradient(clear, shape, dtype, state):
    step(f"scan gradient {shape} {dtype} state={state}")
    b, L, H, P, G, N = shape
    f = R.factors(3, *shape, dtype, resets=[L // 3] if L > 100 else [])
    g = torch.Generator().manual_seed(4)
    dy = torch.randn(b, L, H, P, generator=g).to(dtype)
    h0 = torch.randn(b, H, P, N, generator=g) if state else None
    dh = torch.randn(b, H, P, N, generator=g) if state else None
    names = ["dx", "dla", "dB", "dC"] + (["dh0"] if state else [])
    leaves = [t.requires_grad_() for t in wide(*f, h0) if t is not None]
    y, h = R.scan(*leaves)
    want = torch.autograd.grad([y, h] if state else [y], leaves, wide(dy, dh) if state else
                               [dy.double()])
    on = [t.requires_grad_() for t in dev(*f, h0) if t is not None]
    out = clear.scan(*on, return_state=state)
    got = torch.autograd.grad(out, on, dev(dy, dh) if state else dev(dy))
    for n, a, w in zip(names, got, want):
        check(a, w, dtype, n)


# the ways to cut a bfloat16 sequence: whole; segments, one and two workgroups
# on a compute unit; segments of two channel tiles
CUTS = [(8, 130, 24, 16, 2, 16), (3, 700, 20, 16, 1, 16), (5, 1960, 20, 16, 1, 16),
        (4, 5490, 24, 16, 2, 16), (2, 5500, 24, 128, 1, 16)]


@pytest.mark.parametrize("shape", CUTS)
@pytest.mark.parametrize("state", [False, True])
def test_scan_cuts(clear, shape, state):
    step(f"scan cuts {shape} state={state}")
    b, L, H, P, G, N = shape
    f = dev(*R.factors(7, *shape, BF16, resets=[L // 2]))
    h0 = torch.randn(b, H, P, N, device="cuda") if state else None
    got = clear.scan(*f, h0=h0, return_state=state)
    want, hw = (t.cpu() for t in R.scan(*wide(*f, h0)))
    y, h = got if state else (got, None)
    check(y, want, BF16, "y")
    if state:
        check(h, hw, BF16, "h")


@pytest.mark.parametrize("shape", [(3, 300, 20, 16, 2, 8), (1, 1300, 20, 16, 1, 8),
                                   (1, 4490, 22, 16, 1, 8), (1, 12000, 22, 16, 1, 8)])
def test_scan_gradient_cuts(clear, shape):
    step(f"scan gradient cuts {shape}")
    f = [t.requires_grad_() for t in dev(*R.factors(8, *shape, BF16))]
    dy = torch.randn(shape[:4], device="cuda").to(BF16)
    got = torch.autograd.grad(clear.scan(*f), f, dy)
    leaves = [t.detach().double().requires_grad_() for t in f]
    want = torch.autograd.grad(R.scan(*leaves)[0], leaves, dy.double())
    for n, a, w in zip(("dx", "dla", "dB", "dC"), got, want):
        check(a, w.cpu(), BF16, n)


def test_scan_gradient_against_differences(clear):
    """<gradient, direction> against the central difference of the definition
    in 64 bits, whose error is some 1e-9 here."""
    step("scan gradient against differences")
    b, L, H, P, G, N = shape = (1, 70, 2, 24, 1, 20)
    f = R.factors(5, *shape, F32)
    g = torch.Generator().manual_seed(6)
    dy = torch.randn(b, L, H, P, generator=g)
    on = [t.requires_grad_() for t in dev(*f)]
    got = torch.autograd.grad(clear.scan(*on), on, dy.cuda())
    for i in range(4):
        v = torch.randn(f[i].shape, generator=g).double()
        at = []
        for sign in (1, -1):
            w = wide(*f)
            w[i] = w[i] + sign * 1e-5 * v
            at.append((R.scan(*w)[0] * dy.double()).sum())
        want = (at[0] - at[1]).item() / 2e-5
        have = (got[i].double().cpu() * v).sum().item()
        size = (got[i].double().cpu().norm() * v.norm()).item()
        assert abs(have - want) <= 2.0 ** -16 * size, (i, have, want)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_scan_resets_and_strong_decays(clear, dtype):
    """A log decay of -inf, of the type's lowest value, and sums so negative
    that only differences taken exactly are right behind them."""
    step(f"scan resets {dtype}")
    shape = b, L, H, P, G, N = (2, 150, 2, 32, 1, 32)
    x, la, B, C = R.factors(7, *shape, dtype)
    la[0, 0] = la[0, 5] = la[0, 64] = la[0, 149] = -math.inf
    la[0, 70:75] = torch.finfo(dtype).min
    la[0, 90:100] = -90.0
    la[1] = -math.inf                       # nothing is ever remembered
    la[0, 101:140] = -0.001
    h0 = torch.randn(b, H, P, N, generator=torch.Generator().manual_seed(8)) * 1e4
    y, h = clear.scan(*dev(x, la, B, C, h0), return_state=True)
    want, hw = R.scan(*wide(x, la, B, C, h0))
    check(y, want, dtype, "y")
    check(h, hw, dtype, "h")
    alone = (x.double() * (B.double() * C.double()).sum(-1)[..., None])[1]
    assert R.rel(y[1], alone) <= TOL[dtype]
    on = [t.requires_grad_() for t in dev(x, la, B, C, h0)]
    dy = torch.randn(b, L, H, P, generator=torch.Generator().manual_seed(9)).to(dtype)
    got = torch.autograd.grad(clear.scan(*on), on, dy.cuda())
    leaves = [t.requires_grad_() for t in wide(x, la, B, C, h0)]
    ref = torch.autograd.grad(R.scan(*leaves)[0], leaves, dy.double())
    for n, a, w in zip(["dx", "dla", "dB", "dC", "dh0"], got, ref):
        check(a, w, dtype, n)
    assert (got[1][1] == 0).all() and (got[1][0, 0] == 0).all()
    assert (got[4] == 0).all()              # both rows begin with a reset


def test_scan_without_tokens_or_rows(clear):
    step("scan of nothing")
    for dtype in (F32, BF16):
        x, la, B, C = dev(*R.factors(1, 2, 0, 2, 8, 1, 16, dtype))
        h0 = torch.randn(2, 2, 8, 16, device="cuda").requires_grad_()
        y, h = clear.scan(x, la, B, C, h0=h0, return_state=True)
        assert y.shape == (2, 0, 2, 8) and torch.equal(h, h0)
        dh = torch.randn_like(h)
        assert torch.equal(torch.autograd.grad(h, h0, dh)[0], dh)
        _, h = clear.scan(x, la, B, C, return_state=True)
        assert (h == 0).all()
        y = clear.scan(*dev(*R.factors(1, 0, 5, 2, 8, 1, 16, dtype)))
        assert y.shape == (0, 5, 2, 8)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("gap", [0, 8, 3])
def test_scan_on_slices_of_a_projection(clear, dtype, gap):
    """x, B and C side by side in one array, its rows `gap` elements apart
    from each other: aligned and unaligned slices, with their gradients."""
    step(f"scan slices {dtype} gap={gap}")
    b, L, H, P, G, N = 2, 100, 2, 64, 1, 64
    E = H * P
    g = torch.Generator().manual_seed(10)
    wide_row = torch.randn(b, L, E + 2 * N + gap, generator=g).to(dtype)
    la = R.factors(11, b, L, H, P, G, N, dtype)[1]
    dy = torch.randn(b, L, 2 * E, generator=g).to(dtype)

    def parts(t):
        at = gap
        return (t[..., at:at + E].unflatten(-1, (H, P)),
                t[..., at + E:at + E + N].unflatten(-1, (G, N)),
                t[..., at + E + N:].unflatten(-1, (G, N)))

    def run(t, a, d, f):
        t = t.requires_grad_()
        x, B, C = parts(t)
        y = f(x, a, B, C)
        return y, torch.autograd.grad(y, t, d[..., :E].unflatten(-1, (H, P)))[0]

    y, dt = run(wide_row.cuda(), la.cuda(), dy.cuda(), clear.scan)
    yw, dw = run(wide_row.double(), la.double(), dy.double(), lambda *a: R.scan(*a)[0])
    check(y, yw, dtype, "y")
    check(dt, dw, dtype, "dt")


def test_scan_gradient_of_a_broadcast_input(clear):
    """B given once for the whole batch (stride 0), its gradient summed."""
    step("scan broadcast")
    b, L, H, P, G, N = 3, 40, 2, 16, 1, 32
    x, la, B, C = R.factors(12, b, L, H, P, G, N, F32)
    dy = torch.randn(b, L, H, P, generator=torch.Generator().manual_seed(13))

    def grad(B1, x, la, C, dy, f):
        B1.requires_grad_()
        return torch.autograd.grad(f(x, la, B1.expand(b, -1, -1, -1), C), B1, dy)[0]

    got = grad(*dev(B[:1].clone(), x, la, C, dy), clear.scan)
    want = grad(*wide(B[:1].clone(), x, la, C, dy), lambda *a: R.scan(*a)[0])
    check(got, want, F32, "dB")


def test_scan_keeps_sequences_apart(clear):
    """Values that are not finite spoil their own sequence only."""
    step("scan NaN")
    x, la, B, C = R.factors(14, 3, 130, 2, 64, 1, 64, BF16)
    clean = clear.scan(*dev(x, la, B, C))
    x[1, 70, 0, 3], B[1, 5, 0, 0], la[1, 9, 1] = math.inf, math.nan, math.nan
    y = clear.scan(*dev(x, la, B, C))
    assert torch.equal(y[0], clean[0]) and torch.equal(y[2], clean[2])
    assert not torch.isfinite(y[1]).all()


def test_scan_is_deterministic(clear):
    step("scan twice")
    f = [t.requires_grad_() for t in dev(*R.factors(15, 2, 700, 6, 64, 1, 128, BF16))]
    a, b = (torch.autograd.grad(clear.scan(*f).sum(), f) for _ in range(2))
    assert all(torch.equal(s, t) for s, t in zip(a, b))


def test_scan_past_32_bit_offsets(clear):
    """The second sequence 2^31 + 64 elements behind the first."""
    step("scan far apart")
    b, L, H, P, G, N = 2, 70, 1, 16, 1, 16
    x, la, B, C = R.factors(16, b, L, H, P, G, N, BF16)
    far = (1 << 31) + 64
    big = torch.empty(far + L * P, dtype=BF16, device="cuda")
    xv = big.as_strided(x.shape, (far, P, P, 1))
    xv.copy_(x)
    assert torch.equal(clear.scan(xv, *dev(la, B, C)), clear.scan(*dev(x, la, B, C)))


# ------------------------------------------------------------------ one token

@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("H,P,G,N", [(4, 64, 1, 128), (2, 7, 2, 5), (6, 100, 3, 64),
                                     (1, 1, 1, 1), (2, 130, 1, 66)])
def test_step(clear, dtype, H, P, G, N):
    step(f"step {dtype} {(H, P, G, N)}")
    rows, pool = 5, 9
    x, la, B, C = (t[:, 0] for t in R.factors(20, rows, 1, H, P, G, N, dtype))
    la[3, 0] = -math.inf
    g = torch.Generator().manual_seed(21)
    state = torch.randn(pool, H, P, N, generator=g)
    slots = torch.tensor([7, -1, 0, 3, pool], dtype=torch.int32)   # the 2nd and 5th idle
    state[1] = math.nan                                           # nobody's
    on = state.cuda()
    y = clear.scan_step(*dev(x, la, B, C), on, slots=slots.cuda())
    want = state.clone()
    for i, s in enumerate(slots.tolist()):
        if not 0 <= s < pool:
            assert (y[i] == 0).all()
            continue
        yw, hw = R.scan(*(t[i:i + 1, None].double() for t in (x, la, B, C)),
                        state[s:s + 1].double())
        assert R.rel(y[i], yw[0, 0]) <= TOL[dtype]
        assert R.rel(on[s], hw[0]) <= STATE_TOL
        want[s] = on[s].cpu()
    assert torch.equal(on.cpu().nan_to_num(5.0), want.nan_to_num(5.0))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_steps_go_on_from_a_scan(clear, dtype):
    step(f"steps after a scan {dtype}")
    f = R.factors(22, 2, 90, 4, 64, 2, 128, dtype)
    y, h = clear.scan(*dev(*(t[:, :70] for t in f)), return_state=True)
    ys = [y]
    for t in range(70, 90):
        ys.append(clear.scan_step(*dev(*(v[:, t] for v in f)), h)[:, None])
    want, hw = R.scan(*wide(*f))
    check(torch.cat(ys, 1), want, dtype, "y")
    check(h, hw, dtype, "h")


def test_step_is_seen_by_autograd(clear):
    """A gradient that needs the state from before a step in place is refused."""
    step("step between a scan and its gradient")
    x, la, B, C = dev(*R.factors(25, 2, 5, 3, 16, 1, 32, F32))
    state = torch.zeros(2, 3, 16, 32, device="cuda")
    y = clear.scan(x.requires_grad_(), la, B, C, state)
    with torch.no_grad():
        clear.scan_step(x[:, 0], la[:, 0], B[:, 0], C[:, 0], state)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_step_past_32_bit_offsets(clear):
    """A pool of more than 2^32 state entries."""
    step("step in a large pool")
    H, P, N = 24, 64, 128
    pool = (1 << 32) // (H * P * N) + 2
    state = torch.empty(pool, H, P, N, device="cuda")
    g = torch.Generator().manual_seed(23)
    first = torch.randn(2, H, P, N, generator=g)
    state[-1], state[0] = dev(*first)
    x, la, B, C = (t[:, 0] for t in R.factors(24, 2, 1, H, P, 1, N, BF16))
    small = first.cuda()
    slots = torch.tensor([pool - 1, 0], dtype=torch.int32, device="cuda")
    y = clear.scan_step(*dev(x, la, B, C), state, slots=slots)
    assert torch.equal(y, clear.scan_step(*dev(x, la, B, C), small))
    assert torch.equal(state[-1], small[0]) and torch.equal(state[0], small[1])


# ---------------------------------------------------------------------- norms

WIDTHS = [1, 7, 8, 64, 513, 767, 1024, 1536, 2048, 2050, 4096, 5000, 16384]


def norm_inputs(rows, E, dtype, seed=30):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g).to(dtype)
    return [r(rows, E) for _ in range(5)], [(1 + 0.3 * r(E)).to(dtype) for _ in range(2)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("E", WIDTHS)
@pytest.mark.parametrize("rows", [1, 5, 37])
def test_norm_gated(clear, dtype, E, rows):
    step(f"norm_gated {dtype} {rows} x {E}")
    (m, x, z, du, _), (skip, w) = norm_inputs(rows, E, dtype)
    m[0], x[0] = 0.0, 0.0                       # a row of zeros
    on = [t.requires_grad_() for t in dev(m, x, z, skip, w)]
    u = clear.norm_gated(*on)
    got = torch.autograd.grad(u, on, du.cuda())
    leaves = [t.requires_grad_() for t in wide(m, x, z, skip, w)]
    want = R.gated(*leaves, 1e-5)
    check(u, want, dtype, "u")
    for n, a, b in zip(["dm", "dx", "dz", "dskip", "dw"], got,
                       torch.autograd.grad(want, leaves, du.double())):
        check(a, b, dtype, n)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("E", WIDTHS)
@pytest.mark.parametrize("rows", [1, 5, 37])
def test_norm_residual(clear, dtype, E, rows):
    step(f"norm_residual {dtype} {rows} x {E}")
    (o, r, du, dr, _), (scale, w) = norm_inputs(rows, E, dtype)
    on = [t.requires_grad_() for t in dev(o, r, scale, w)]
    out = clear.norm_residual(*on)
    leaves = [t.requires_grad_() for t in wide(o, r, scale, w)]
    want = R.residual(*leaves, 1e-5)
    check(out[0], want[0], dtype, "r_new")
    check(out[1], want[1], dtype, "u")
    # both outputs used, and each alone
    for use in ((0, 1), (0,), (1,)):
        d = [(dr, du)[k] for k in use]
        got = torch.autograd.grad([out[k] for k in use], on, dev(*d), retain_graph=True,
                                  allow_unused=True)
        ref = torch.autograd.grad([want[k] for k in use], leaves, wide(*d), retain_graph=True,
                                  allow_unused=True)
        for n, a, b in zip(["do", "dr", "dscale", "dw"], got, ref):
            check(a, torch.zeros(E, dtype=torch.float64) if b is None else b, dtype, n)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_norm_gradients_against_differences(clear, dtype):
    """In float32 directly; in bfloat16 the gradient carries two roundings."""
    step(f"norm gradients against differences {dtype}")
    (m, x, z, du, _), (skip, w) = norm_inputs(6, 40, dtype, seed=31)
    g = torch.Generator().manual_seed(32)
    for f, ref, ins in ((clear.norm_gated, R.gated, (m, x, z, skip, w)),
                        (lambda *a: clear.norm_residual(*a)[1],
                         lambda *a: R.residual(*a)[1], (m, x, skip, w))):
        on = [t.requires_grad_() for t in dev(*ins)]
        got = torch.autograd.grad(f(*on), on, du.cuda())
        for i in range(len(ins)):
            v = torch.randn(ins[i].shape, generator=g).double()
            at = []
            for sign in (1, -1):
                q = wide(*ins)
                q[i] = q[i] + sign * 1e-5 * v
                at.append((ref(*q, 1e-5) * du.double()).sum())
            want = (at[0] - at[1]).item() / 2e-5
            have = (got[i].double().cpu() * v).sum().item()
            size = (got[i].double().cpu().norm() * v.norm()).item()
            assert abs(have - want) <= TOL[dtype] * size, (i, have, want)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("gap", [8, 3])
def test_norms_on_slices(clear, dtype, gap):
    """Rows further apart than their width, aligned and not; a gradient whose
    rows do not lie evenly."""
    step(f"norm slices {dtype} gap={gap}")
    E = 96
    g = torch.Generator().manual_seed(33)
    t = torch.randn(3, 11, 3 * E + gap, generator=g).to(dtype)
    du = torch.randn(11, 3, E, generator=g).to(dtype).transpose(0, 1)
    _, (skip, w) = norm_inputs(1, E, dtype, seed=34)

    def run(t, skip, w, du, f, h):
        t.requires_grad_()
        a, b, c = t[..., gap:].split(E, -1)
        u = f(a, b, c, skip, w, 1e-5)
        r, v = h(a, c, skip, w, 1e-5)
        return u, r, v, torch.autograd.grad([u, v], t, [du, du])[0]

    got = run(*dev(t, skip, w, du), clear.norm_gated, clear.norm_residual)
    want = run(*wide(t, skip, w, du), R.gated, R.residual)
    for n, a, b in zip(["u", "r", "v", "dt"], got, want):
        # dt sums two gradients that are each rounded before
        assert R.rel(a, b) <= TOL[dtype] * (2 if n == "dt" else 1), n


def test_norms_without_rows(clear):
    step("norms of nothing")
    for dtype in (F32, BF16):
        m = torch.empty(0, 3, 40, dtype=dtype, device="cuda").requires_grad_()
        w = torch.ones(40, dtype=dtype, device="cuda").requires_grad_()
        u = clear.norm_gated(m, m, m, w, w)
        r, v = clear.norm_residual(m, m, w, w)
        assert u.shape == r.shape == v.shape == m.shape
        for d in torch.autograd.grad([u, v], [w], [u.detach(), v.detach()]):
            assert (d == 0).all()


def test_norms_keep_rows_apart(clear):
    step("norm NaN")
    (m, x, z, _, _), (skip, w) = norm_inputs(9, 100, BF16)
    clean = clear.norm_gated(*dev(m, x, z, skip, w))
    m[4, 3] = math.nan
    got = clear.norm_gated(*dev(m, x, z, skip, w))
    keep = [i for i in range(9) if i != 4]
    assert torch.equal(got[keep], clean[keep]) and got[4].isnan().all()


def test_norms_many_rows_are_deterministic(clear):
    step("norms of many rows")
    (m, x, z, du, _), (skip, w) = norm_inputs(5000, 100, F32)
    on = [t.requires_grad_() for t in dev(m, x, z, skip, w)]
    a, b = (torch.autograd.grad(clear.norm_gated(*on), on, du.cuda()) for _ in range(2))
    assert all(torch.equal(s, t) for s, t in zip(a, b))
    leaves = [t.requires_grad_() for t in wide(m, x, z, skip, w)]
    want = torch.autograd.grad(R.gated(*leaves, 1e-5), leaves, du.double())
    for n, s, t in zip(["dm", "dx", "dz", "dskip", "dw"], a, want):
        check(s, t, F32, n)


# ------------------------------------------------------------ streams, graphs

def test_other_streams(clear):
    step("other streams")
    f = dev(*R.factors(40, 2, 300, 2, 64, 1, 64, BF16))
    want = clear.scan(*f)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = clear.scan(*f, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    with torch.cuda.stream(side):
        got = clear.scan(*f)
    side.synchronize()
    assert torch.equal(got, want)


def test_graph_replays(clear):
    """The block's calls in one graph, replayed between eager work."""
    step("graph")
    b, L, H, P, N = 1, 200, 4, 32, 64
    x, la, B, C = dev(*R.factors(41, b, L, H, P, 1, N, BF16))
    E = H * P
    z, skip, w = (torch.randn(s, device="cuda").to(BF16) for s in ((b, L, E), (E,), (E,)))
    state = torch.randn(b, H, P, N, device="cuda")
    start = state.clone()

    def block():
        y, h = clear.scan(x, la, B, C, h0=state, return_state=True)
        u = clear.norm_gated(y.flatten(2), x.flatten(2), z, skip, w)
        r, v = clear.norm_residual(u, z, skip, w)
        last = clear.scan_step(x[:, 0], la[:, 0], B[:, 0], C[:, 0], state)
        return u, r, v, h, last

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        for _ in range(2):
            block()
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = block()
    for k in range(4):
        x.normal_()
        state.copy_(start)
        want = [t.clone() for t in block()]
        after = state.clone()
        state.copy_(start)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(out, want)), k
        assert torch.equal(state, after)


# ------------------------------------------------------------------- refusals

def test_refusals(clear):
    step("refusals")
    x, la, B, C = dev(*R.factors(50, 2, 10, 4, 16, 2, 32, BF16))
    h = torch.zeros(2, 4, 16, 32, device="cuda")
    bad = [
        (TypeError, lambda: clear.scan(x.cpu(), la, B, C)),
        (TypeError, lambda: clear.scan(x.half(), la, B, C)),
        (TypeError, lambda: clear.scan(x, la.float(), B, C)),
        (TypeError, lambda: clear.scan(x, la, B, C, h0=h.bfloat16())),
        (ValueError, lambda: clear.scan(x, la[:, :9], B, C)),
        (ValueError, lambda: clear.scan(x, la, B, C[..., :31])),
        (ValueError, lambda: clear.scan(x.transpose(2, 3).contiguous().transpose(2, 3), la, B, C)),
        (ValueError, lambda: clear.scan(x, la, B, C, h0=h[:1])),
        (ValueError, lambda: clear.scan(x, la, B, C, h0=h.transpose(2, 3).contiguous()
                                        .transpose(2, 3))),
        (RuntimeError, lambda: clear.scan(x[:, :, :3], la[:, :, :3], B, C)),   # 3 heads, 2 groups
        (RuntimeError, lambda: clear.scan(x, la, *[torch.zeros(2, 10, 2, 129, dtype=BF16,
                                                               device="cuda")] * 2)),
        (ValueError, lambda: clear.scan_step(x[:, 0], la[:, 0], B[:, 0], C[:, 0], h[:, :2])),
        (RuntimeError, lambda: clear.scan_step(x[:, 0], la[:, 0], B[:, 0], C[:, 0], h[:1])),
        (TypeError, lambda: clear.scan_step(x[:, 0], la[:, 0], B[:, 0], C[:, 0], h,
                                            slots=torch.zeros(2, device="cuda",
                                                              dtype=torch.int64))),
        (ValueError, lambda: clear.scan_step(x[:, 0].clone().requires_grad_(), la[:, 0], B[:, 0],
                                             C[:, 0], h)),
    ]
    m = torch.zeros(4, 24, dtype=BF16, device="cuda")
    w = torch.zeros(24, dtype=BF16, device="cuda")
    bad += [
        (ValueError, lambda: clear.norm_gated(m, m[:3], m, w, w)),
        (ValueError, lambda: clear.norm_gated(m, m, m, w, w[:20])),
        (TypeError, lambda: clear.norm_gated(m, m, m, w, w.float())),
        (RuntimeError, lambda: clear.norm_gated(m, m, m, w, w, eps=0.0)),
        (RuntimeError, lambda: clear.norm_gated(m, m, m, w, w, eps=math.nan)),
        (ValueError, lambda: clear.norm_residual(m.t().contiguous().t(), m, w, w)),
        (RuntimeError, lambda: clear.norm_residual(*[torch.zeros(1, 16385, device="cuda")] * 2,
                                                   *[torch.zeros(16385, device="cuda")] * 2)),
    ]
    for k, (error, call) in enumerate(bad):
        with pytest.raises(error):
            call()
            pytest.fail(f"call {k} was not refused")


# -------------------------------------------------------------------- example

@pytest.mark.parametrize("dtype", [F32, BF16])
def test_example_learns_and_serves(clear, dtype):
    """The example's block: its loss falls by half, and token by token it gives
    what it gives at once, to the roundings on the way: four on either side
    between the recurrence and the output, each of at most one unit (bfloat16:
    2^-8; float32, whose sums have some hundreds of terms: 2^-16), on values up
    to some five times the root mean square."""
    step(f"example {dtype}")
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                        "clear_block.py")
    spec = importlib.util.spec_from_file_location("clear_block", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    block = example.Block(dtype=dtype)
    first, last = example.train(block, 40, 4, 200)
    assert last < 0.5 * first
    unit = 2.0 ** (-8 if dtype == BF16 else -16)
    assert example.serve(block, 5, 100, 10) <= 2 * 4 * 5 * unit
