"""The block in the clear: the gated linear recurrence and the norms of
``include/fesc.h`` (section "The block in the clear") on torch tensors.

    scan           S_t = e^{la_t} S_{t-1} + x_t B_t^T,  y_t = S_t C_t
    scan_step      one token for each row of a batch, states in place
    norm_gated     u = v w / sqrt(mean v^2 + eps),  v = (m + skip x) silu(z)
    norm_residual  the same norm of r + scale o, which is returned too

``scan`` and the norms are differentiable.  All tensors of a call are of one
type, float32 or bfloat16, except states, which are float32.  Every
computation runs in the library's HIP kernels, on the current stream (or on
`stream`); there is no fallback path.
"""
from __future__ import annotations

import ctypes

import torch

from .fesc import _check, _lib

_u32, _u64, _vp, _sz = ctypes.c_uint32, ctypes.c_uint64, ctypes.c_void_p, ctypes.c_size_t

_TYPES = {torch.float32: 0, torch.bfloat16: 1}


class _ScanDesc(ctypes.Structure):
    _fields_ = [(n, _u32) for n in ("dtype", "batch", "len", "heads", "head_dim", "groups",
                                    "d_state")]
    _fields_ += [(n, _u64) for n in ("x_token", "x_batch", "la_token", "la_batch", "b_token",
                                     "b_batch", "c_token", "c_batch", "dy_token", "dy_batch")]


class _NormDesc(ctypes.Structure):
    _fields_ = [("dtype", _u32), ("width", _u32), ("rows", _u64), ("eps", ctypes.c_float)]
    _fields_ += [(n, _u64) for n in ("m_row", "x_row", "z_row", "o_row", "r_row", "du_row",
                                     "dr_row")]


_SIGS = {
    "fesc_clear_scan_workspace": [_vp, ctypes.c_int, _vp],
    "fesc_clear_scan": [_vp] * 9 + [_sz, _vp],
    "fesc_clear_scan_bwd": [_vp] * 14 + [_sz, _vp],
    "fesc_clear_scan_step": [_vp] * 6 + [_u32] + [_vp] * 3,
    "fesc_clear_norm_gated": [_vp] * 8,
    "fesc_clear_norm_residual": [_vp] * 8,
    "fesc_clear_norm_workspace": [_vp, _vp],
    "fesc_clear_norm_gated_bwd": [_vp] * 13 + [_sz, _vp],
    "fesc_clear_norm_residual_bwd": [_vp] * 12 + [_sz, _vp],
}
for _name, _args in _SIGS.items():
    _f = getattr(_lib, _name)
    _f.argtypes = _args
    _f.restype = ctypes.c_int


def _p(t):
    return None if t is None else t.data_ptr()


def _stream(t):
    """The current stream of t's device, as its handle."""
    return torch._C._cuda_getCurrentRawStream(t.device.index)


def _once():
    if torch.is_grad_enabled():
        raise RuntimeError("the block in the clear is differentiable once: no create_graph=True")


def _tensor(t, what, like=None, dtype=None):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{what}: expected a CUDA tensor")
    if like is None:
        if t.dtype not in _TYPES:
            raise TypeError(f"{what}: float32 or bfloat16, got {t.dtype}")
        if t.device.index != torch.cuda.current_device():
            raise ValueError(f"{what}: on {t.device}, the current device is "
                             f"cuda:{torch.cuda.current_device()}")
    else:
        if t.dtype != (dtype or like.dtype):
            raise TypeError(f"{what}: expected {dtype or like.dtype}, got {t.dtype}")
        if t.device != like.device:
            raise ValueError(f"{what}: on {t.device}, expected {like.device}")
    return t


def _shape(t, shape, what):
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{what}: shape {tuple(t.shape)}, expected {tuple(shape)}")


def _dense_tail(t, dims):
    """Whether the last `dims` dimensions are laid out without gaps."""
    step = 1
    for d in range(t.dim() - 1, t.dim() - 1 - dims, -1):
        if t.shape[d] != 1:
            if t.stride(d) != step:
                return False
            step *= t.shape[d]
    return True


def _factor(t, dims, what):
    if t.numel() and not _dense_tail(t, dims):
        raise ValueError(f"{what}: the last {dims} dimension(s) must be contiguous")
    return t


def _state(t, shape, what, like):
    _tensor(t, what, like, torch.float32)
    _shape(t, shape, what)
    if not t.is_contiguous():
        raise ValueError(f"{what}: must be contiguous")
    return t


def _space(desc, query, *args):
    need = _sz()
    _check(query(ctypes.byref(desc), *args, ctypes.byref(need)))
    return need.value


def _buffer(bytes_, like):
    return torch.empty(bytes_, dtype=torch.uint8, device=like.device) if bytes_ else None


# ---------------------------------------------------------------- recurrence

def _scan_desc(x, la, B, C):
    b, n, H, P = x.shape
    G, N = B.shape[2:]
    return _ScanDesc(_TYPES[x.dtype], b, n, H, P, G, N, x.stride(1), x.stride(0), la.stride(1),
                     la.stride(0), B.stride(1), B.stride(0), C.stride(1), C.stride(0), 0, 0)


def _scan_forward(x, la, B, C, h0, want_state):
    d = _scan_desc(x, la, B, C)
    b, n, H, P = x.shape
    y = torch.empty((b, n, H, P), dtype=x.dtype, device=x.device)
    h = None
    if want_state:
        h = torch.empty((b, H, P, B.shape[3]), dtype=torch.float32, device=x.device)
    need = _space(d, _lib.fesc_clear_scan_workspace, 0)
    w = _buffer(need, x)
    _check(_lib.fesc_clear_scan(ctypes.byref(d), _p(x), _p(la), _p(B), _p(C), _p(h0), _p(y),
                                _p(h), _p(w), need, _stream(x)))
    return y, h


class _Scan(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, la, B, C, h0, want_state):
        ctx.set_materialize_grads(False)
        ctx.save_for_backward(x, la, B, C, h0)
        y, h = _scan_forward(x, la, B, C, h0, want_state)
        return (y, h) if want_state else y

    @staticmethod
    def backward(ctx, dy, dh=None):
        _once()
        x, la, B, C, h0 = ctx.saved_tensors
        if dy is None:
            if dh is None:
                return (None,) * 6
            dy = torch.zeros_like(x, memory_format=torch.contiguous_format)
        elif not _dense_tail(dy, 2):
            dy = dy.contiguous()
        if dh is not None:
            dh = dh.contiguous()
        d = _scan_desc(x, la, B, C)
        d.dy_token, d.dy_batch = dy.stride(1), dy.stride(0)

        def like(t):
            return torch.empty(t.shape, dtype=t.dtype, device=t.device)

        dx, dla, db, dc = like(x), like(la), like(B), like(C)
        dh0 = like(h0) if h0 is not None and ctx.needs_input_grad[4] else None
        need = _space(d, _lib.fesc_clear_scan_workspace, 1)
        w = _buffer(need, x)
        _check(_lib.fesc_clear_scan_bwd(
            ctypes.byref(d), _p(x), _p(la), _p(B), _p(C), _p(h0), _p(dy), _p(dh), _p(dx), _p(dla),
            _p(db), _p(dc), _p(dh0), _p(w), need, _stream(x)))
        return dx, dla, db, dc, dh0, None


def scan(x, la, B, C, h0=None, return_state=False, stream=None):
    """Outputs y [batch, len, heads, head_dim] of the recurrence, and with
    `return_state` the final state as well.

    x [batch, len, heads, head_dim], la [batch, len, heads] (log decays, <= 0;
    -inf resets the state), B and C [batch, len, groups, d_state]; the first
    two dimensions may have any strides, so slices of a wider projection do.
    h0 and the returned state: float32 [batch, heads, head_dim, d_state].
    Differentiable with respect to all five.
    """
    if stream is not None:
        with torch.cuda.stream(stream):
            return scan(x, la, B, C, h0, return_state)
    _tensor(x, "x")
    for t, what in ((la, "la"), (B, "B"), (C, "C")):
        _tensor(t, what, x)
    if x.dim() != 4 or B.dim() != 4:
        raise ValueError("x, B: expected [batch, len, heads or groups, width]")
    _shape(la, x.shape[:3], "la")
    _shape(B, (*x.shape[:2], *B.shape[2:]), "B")
    _shape(C, B.shape, "C")
    _factor(x, 2, "x"), _factor(la, 1, "la"), _factor(B, 2, "B"), _factor(C, 2, "C")
    if h0 is not None:
        _state(h0, (x.shape[0], *x.shape[2:], B.shape[3]), "h0", x)
    if torch.is_grad_enabled() and (x.requires_grad or la.requires_grad or B.requires_grad
                                    or C.requires_grad
                                    or (h0 is not None and h0.requires_grad)):
        return _Scan.apply(x, la, B, C, h0, return_state)
    y, h = _scan_forward(x, la, B, C, h0, return_state)
    return (y, h) if return_state else y


def scan_step(x, la, B, C, state, slots=None, stream=None):
    """One token for each row: updates `state` in place and returns y
    [rows, heads, head_dim].

    x [rows, heads, head_dim], la [rows, heads], B and C [rows, groups,
    d_state]; state float32 [pool, heads, head_dim, d_state].  Row i uses state
    slots[i] (int32, None: i); a slot outside the pool (-1) marks an idle row,
    whose y is zero.  No two rows may name one slot.  Not differentiable.
    """
    if stream is not None:
        with torch.cuda.stream(stream):
            return scan_step(x, la, B, C, state, slots)
    _tensor(x, "x")
    for t, what in ((la, "la"), (B, "B"), (C, "C")):
        _tensor(t, what, x)
    if x.dim() != 3 or B.dim() != 3:
        raise ValueError("x, B: expected [rows, heads or groups, width]")
    rows, H, P = x.shape
    G, N = B.shape[1:]
    _shape(la, (rows, H), "la")
    _shape(B, (rows, G, N), "B")
    _shape(C, B.shape, "C")
    _factor(x, 2, "x"), _factor(la, 1, "la"), _factor(B, 2, "B"), _factor(C, 2, "C")
    _state(state, (state.shape[0] if state.dim() else 0, H, P, N), "state", x)
    if slots is not None:
        _tensor(slots, "slots", x, torch.int32)
        _shape(slots, (rows,), "slots")
        if not slots.is_contiguous():
            raise ValueError("slots: must be contiguous")
    if torch.is_grad_enabled() and any(t.requires_grad for t in (x, la, B, C, state)):
        raise ValueError("scan_step is not differentiable: use scan, or torch.no_grad()")
    y = torch.empty((rows, H, P), dtype=x.dtype, device=x.device)
    d = _ScanDesc(_TYPES[x.dtype], rows, 1, H, P, G, N, 0, x.stride(0), 0, la.stride(0), 0,
                  B.stride(0), 0, C.stride(0), 0, 0)
    _check(_lib.fesc_clear_scan_step(ctypes.byref(d), _p(x), _p(la), _p(B), _p(C), _p(state),
                                     state.shape[0], _p(slots), _p(y), _stream(x)))
    return y


# --------------------------------------------------------------------- norms

def _rows(t, what):
    """Row stride of [..., width] whose leading dimensions lie evenly."""
    w = t.shape[-1]
    if t.numel() == 0:
        return w
    if w != 1 and t.stride(-1) != 1:
        raise ValueError(f"{what}: the last dimension must be contiguous")
    stride, step = None, None
    for d in range(t.dim() - 2, -1, -1):
        if t.shape[d] == 1:
            continue
        if stride is None:
            stride = step = t.stride(d)
        elif t.stride(d) != step:
            raise ValueError(f"{what}: rows must lie evenly (one stride)")
        step *= t.shape[d]
    return w if stride is None else stride


def _grad_rows(t):
    """A gradient as rows that lie evenly, with their stride."""
    try:
        return t, _rows(t, "")
    except ValueError:
        t = t.contiguous()
        return t, t.shape[-1]


def _norm_desc(t, eps, **strides):
    w = t.shape[-1]
    d = _NormDesc(_TYPES[t.dtype], w, t.numel() // w if w else 0, eps)
    for k, v in strides.items():
        setattr(d, k, v)
    return d


def _norm_check(first, others, vectors):
    """Types and shapes of a norm's arrays (name, tensor) and weight vectors."""
    t = _tensor(first[1], first[0])
    if t.dim() == 0:
        raise ValueError(f"{first[0]}: expected [..., width]")
    for what, o in others:
        _shape(_tensor(o, what, t), t.shape, what)
    for what, v in vectors:
        _shape(_tensor(v, what, t), t.shape[-1:], what)
        if not v.is_contiguous():
            raise ValueError(f"{what}: must be contiguous")


def _empty(t):
    return torch.empty(t.shape, dtype=t.dtype, device=t.device)


def _gated_forward(m, x, z, skip, w, eps):
    d = _norm_desc(m, eps, m_row=_rows(m, "m"), x_row=_rows(x, "x"), z_row=_rows(z, "z"))
    u = _empty(m)
    _check(_lib.fesc_clear_norm_gated(ctypes.byref(d), _p(m), _p(x), _p(z), _p(skip), _p(w), _p(u),
                                      _stream(m)))
    return u


class _Gated(torch.autograd.Function):
    @staticmethod
    def forward(ctx, m, x, z, skip, w, eps):
        ctx.eps = eps
        ctx.save_for_backward(m, x, z, skip, w)
        return _gated_forward(m, x, z, skip, w, eps)

    @staticmethod
    def backward(ctx, du):
        _once()
        m, x, z, skip, w = ctx.saved_tensors
        du, du_row = _grad_rows(du)
        d = _norm_desc(m, ctx.eps, m_row=_rows(m, "m"), x_row=_rows(x, "x"), z_row=_rows(z, "z"),
                       du_row=du_row)
        dm, dx, dz, dskip, dw = (_empty(t) for t in (m, x, z, skip, w))
        need = _space(d, _lib.fesc_clear_norm_workspace)
        ws = _buffer(need, m)
        _check(_lib.fesc_clear_norm_gated_bwd(
            ctypes.byref(d), _p(m), _p(x), _p(z), _p(skip), _p(w), _p(du), _p(dm), _p(dx), _p(dz),
            _p(dskip), _p(dw), _p(ws), need, _stream(m)))
        return dm, dx, dz, dskip, dw, None


def norm_gated(m, x, z, skip, w, eps=1e-5, stream=None):
    """u = v w / sqrt(mean v^2 + eps) over the last dimension, with
    v = (m + skip x) silu(z): m the recurrence's output, x its input (the skip
    connection), z the gate, all [..., width] with rows of any one stride;
    skip and w [width].  Differentiable with respect to all five."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return norm_gated(m, x, z, skip, w, eps)
    _norm_check(("m", m), (("x", x), ("z", z)), (("skip", skip), ("w", w)))
    if torch.is_grad_enabled() and (m.requires_grad or x.requires_grad or z.requires_grad
                                    or skip.requires_grad or w.requires_grad):
        return _Gated.apply(m, x, z, skip, w, eps)
    return _gated_forward(m, x, z, skip, w, eps)


def _residual_forward(o, r, scale, w, eps):
    d = _norm_desc(o, eps, o_row=_rows(o, "o"), r_row=_rows(r, "r"))
    new, u = _empty(o), _empty(o)
    _check(_lib.fesc_clear_norm_residual(ctypes.byref(d), _p(o), _p(r), _p(scale), _p(w), _p(new),
                                         _p(u), _stream(o)))
    return new, u


class _Residual(torch.autograd.Function):
    @staticmethod
    def forward(ctx, o, r, scale, w, eps):
        ctx.set_materialize_grads(False)
        ctx.eps = eps
        ctx.save_for_backward(o, r, scale, w)
        return _residual_forward(o, r, scale, w, eps)

    @staticmethod
    def backward(ctx, dnew, du):
        _once()
        o, r, scale, w = ctx.saved_tensors
        if dnew is None and du is None:
            return (None,) * 5
        d = _norm_desc(o, ctx.eps, o_row=_rows(o, "o"), r_row=_rows(r, "r"))
        if du is not None:
            du, d.du_row = _grad_rows(du)
        if dnew is not None:
            dnew, d.dr_row = _grad_rows(dnew)
        do, dr, dscale, dw = (_empty(t) for t in (o, r, scale, w))
        need = _space(d, _lib.fesc_clear_norm_workspace)
        ws = _buffer(need, o)
        _check(_lib.fesc_clear_norm_residual_bwd(
            ctypes.byref(d), _p(o), _p(r), _p(scale), _p(w), _p(du), _p(dnew), _p(do), _p(dr),
            _p(dscale), _p(dw), _p(ws), need, _stream(o)))
        return do, dr, dscale, dw, None


def norm_residual(o, r, scale, w, eps=1e-5, stream=None):
    """(r_new, u): r_new = r + scale o, the residual stream after a block's
    output o, and u = r_new w / sqrt(mean r_new^2 + eps), the next block's
    input.  o and r [..., width] with rows of any one stride; scale and w
    [width].  u is formed from r_new before it is rounded.  Differentiable
    with respect to all four."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return norm_residual(o, r, scale, w, eps)
    _norm_check(("o", o), (("r", r),), (("scale", scale), ("w", w)))
    if torch.is_grad_enabled() and (o.requires_grad or r.requires_grad or scale.requires_grad
                                    or w.requires_grad):
        return _Residual.apply(o, r, scale, w, eps)
    return _residual_forward(o, r, scale, w, eps)
