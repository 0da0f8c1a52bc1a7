"""Argument checks and workspace sizes of the block in the clear, at the C
entry points (no call here reaches a kernel)."""
import ctypes

import pytest
import torch

import clear_reference as R


@pytest.fixture(scope="module")
def clear():
    from paper_2608_17442_amd import clear
    return clear


def scan_desc(clear, **kw):
    v = dict(dtype=1, batch=2, len=100, heads=4, head_dim=64, groups=1, d_state=128)
    v.update(kw)
    return clear._ScanDesc(**v)


def norm_desc(clear, **kw):
    v = dict(dtype=1, width=100, rows=10, eps=1e-5)
    v.update(kw)
    return clear._NormDesc(**v)


def bytes_of(clear, d, backward=0):
    n = ctypes.c_size_t()
    rc = clear._lib.fesc_clear_scan_workspace(ctypes.byref(d), backward, ctypes.byref(n))
    return rc, n.value


@pytest.mark.parametrize("bad", [
    dict(dtype=2), dict(heads=0), dict(groups=0), dict(groups=3), dict(heads=5000),
    dict(head_dim=0), dict(head_dim=4097), dict(d_state=0), dict(d_state=129),
    dict(x_token=(1 << 40) + 1), dict(dy_batch=1 << 63),
])
def test_scan_descriptors_are_checked(clear, bad):
    d = scan_desc(clear, **bad)
    assert bytes_of(clear, d)[0] == -1
    lib = clear._lib
    null = [None] * 8
    assert lib.fesc_clear_scan(ctypes.byref(d), *null, 0, None) == -1
    assert lib.fesc_clear_scan_bwd(ctypes.byref(d), *[None] * 13, 0, None) == -1
    assert lib.fesc_clear_scan_step(ctypes.byref(d), *[None] * 5, 4, None, None, None) == -1


def test_null_arguments_are_refused(clear):
    lib = clear._lib
    d, n = scan_desc(clear), norm_desc(clear)
    assert lib.fesc_clear_scan_workspace(None, 0, None) == -1
    assert lib.fesc_clear_scan_workspace(ctypes.byref(d), 0, None) == -1
    assert lib.fesc_clear_scan(ctypes.byref(d), *[None] * 8, 1 << 40, None) == -1
    assert lib.fesc_clear_scan_bwd(ctypes.byref(d), *[None] * 13, 1 << 40, None) == -1
    assert lib.fesc_clear_scan_step(ctypes.byref(d), *[None] * 5, 4, None, None, None) == -1
    assert lib.fesc_clear_norm_gated(None, *[None] * 7) == -1
    assert lib.fesc_clear_norm_gated(ctypes.byref(n), *[None] * 7) == -1
    assert lib.fesc_clear_norm_residual(ctypes.byref(n), *[None] * 7) == -1
    assert lib.fesc_clear_norm_gated_bwd(ctypes.byref(n), *[None] * 12, 1 << 40, None) == -1
    assert lib.fesc_clear_norm_residual_bwd(ctypes.byref(n), *[None] * 11, 1 << 40, None) == -1
    assert b"null" in lib.fesc_last_error()


def test_small_or_unaligned_workspaces_are_refused(clear):
    """Made-up addresses: the check comes before anything is launched."""
    lib = clear._lib
    d = scan_desc(clear, batch=1, len=2000)
    rc, need = bytes_of(clear, d)
    assert rc == 0 and need > 0                    # few heads: the sequence is cut
    p = 1 << 20
    args = [p] * 4 + [None, p, None]
    assert lib.fesc_clear_scan(ctypes.byref(d), *args, p, need - 1, None) == -1
    assert b"small" in lib.fesc_last_error()
    assert lib.fesc_clear_scan(ctypes.byref(d), *args, None, need, None) == -1
    assert lib.fesc_clear_scan(ctypes.byref(d), *args, p + 8, need, None) == -1
    assert b"aligned" in lib.fesc_last_error()
    n = norm_desc(clear)
    need = ctypes.c_size_t()
    assert lib.fesc_clear_norm_workspace(ctypes.byref(n), ctypes.byref(need)) == 0
    assert lib.fesc_clear_norm_gated_bwd(ctypes.byref(n), *[p] * 11, p, need.value - 1, None) == -1


@pytest.mark.parametrize("bad", [dict(dtype=7), dict(width=0), dict(width=16385), dict(eps=0.0),
                                 dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
                                 dict(m_row=1 << 41), dict(rows=1 << 41)])
def test_norm_descriptors_are_checked(clear, bad):
    d = norm_desc(clear, **bad)
    p = 1 << 20
    assert clear._lib.fesc_clear_norm_gated(ctypes.byref(d), *[p] * 6, None) == -1
    assert clear._lib.fesc_clear_norm_residual(ctypes.byref(d), *[p] * 6, None) == -1


def test_too_large_calls_are_refused(clear):
    p = 1 << 20
    d = scan_desc(clear, batch=1 << 20, heads=4096, groups=1, len=64)
    assert clear._lib.fesc_clear_scan(ctypes.byref(d), *[p] * 4, None, p, None, p, 1 << 62,
                                      None) == -1
    d = scan_desc(clear, batch=1 << 20, heads=4096, groups=1)
    assert clear._lib.fesc_clear_scan_step(ctypes.byref(d), *[p] * 5, 1 << 20, None, p, None) == -1
    d = scan_desc(clear, batch=8)
    assert clear._lib.fesc_clear_scan_step(ctypes.byref(d), *[p] * 5, 7, None, p, None) == -1
    assert b"pool" in clear._lib.fesc_last_error()


def test_empty_calls_do_nothing(clear):
    """No rows: nothing is read, written or launched."""
    lib = clear._lib
    d = scan_desc(clear, batch=0)
    assert bytes_of(clear, d) == (0, 0)
    assert lib.fesc_clear_scan(ctypes.byref(d), *[None] * 8, 0, None) == 0
    assert lib.fesc_clear_scan_bwd(ctypes.byref(d), *[None] * 13, 0, None) == 0
    assert lib.fesc_clear_scan_step(ctypes.byref(d), *[None] * 5, 0, None, None, None) == 0
    n = norm_desc(clear, rows=0)
    assert lib.fesc_clear_norm_gated(ctypes.byref(n), *[None] * 7) == 0
    assert lib.fesc_clear_norm_residual(ctypes.byref(n), *[None] * 7) == 0


def test_tensors_on_the_cpu_are_refused(clear):
    x, la, B, C = R.factors(1, 1, 4, 2, 8, 1, 16, torch.float32)
    with pytest.raises(TypeError, match="CUDA"):
        clear.scan(x, la, B, C)
    with pytest.raises(TypeError, match="CUDA"):
        clear.scan_step(x[:, 0], la[:, 0], B[:, 0], C[:, 0], torch.zeros(1, 2, 8, 16))
    with pytest.raises(TypeError, match="CUDA"):
        clear.norm_gated(x, x, x, x[0, 0, 0], x[0, 0, 0])
    with pytest.raises(TypeError, match="CUDA"):
        clear.norm_residual(x, x, x[0, 0, 0], x[0, 0, 0])


# The reference itself, against closed forms.

def test_reference_scan_is_the_sum_over_earlier_tokens():
    x, la, B, C = (t.double() for t in R.factors(2, 1, 9, 2, 3, 1, 4, torch.float32))
    h0 = torch.randn(1, 2, 3, 4, dtype=torch.float64)
    y, h = R.scan(x, la, B, C, h0)
    for t in range(9):
        for head in range(2):
            w = torch.stack([la[0, r + 1:t + 1, head].sum().exp() for r in range(t + 1)])
            want = ((C[0, t, 0] * B[0, :t + 1, 0]).sum(-1) * w) @ x[0, :t + 1, head]
            want = want + la[0, :t + 1, head].sum().exp() * (h0[0, head] @ C[0, t, 0])
            assert torch.allclose(y[0, t, head], want, rtol=1e-12, atol=1e-12)
    w = torch.stack([la[0, r + 1:, 1].sum().exp() for r in range(9)])
    want = (x[0, :, 1] * w[:, None]).t() @ B[0, :, 0] + la[0, :, 1].sum().exp() * h0[0, 1]
    assert torch.allclose(h[0, 1], want, rtol=1e-12, atol=1e-12)


def test_reference_norms_scale_rows_to_one():
    g = torch.Generator().manual_seed(3)
    m, x, z = (torch.randn(4, 50, generator=g, dtype=torch.float64) for _ in range(3))
    one = torch.ones(50, dtype=torch.float64)
    u = R.gated(m, x, z, one, one, 1e-30)
    assert torch.allclose(u.square().mean(-1), torch.ones(4, dtype=torch.float64))
    v, u = R.residual(m, x, 2 * one, 3 * one, 1e-30)
    assert torch.allclose(v, x + 2 * m) and torch.allclose(u.square().mean(-1), 9 * one[:4])
