"""The block in the clear: the gated linear recurrence and the norms of
``include/fesc.h`` (section "The block in the clear") on torch tensors.

    scan           S_t = e^{la_t} S_{t-1} + x_t B_t^T,  y_t = S_t C_t
    scan_step      one token for each row of a batch, states in place
    norm_gated     u = v w / sqrt(mean v^2 + eps),  v = (m + skip x) silu(z)
    norm_residual  the same norm of r + scale o, which is returned too

``scan`` and the norms are differentiable, once and in reverse; what would need
another derivative or a trace of them is refused.  All tensors of a call are of one
type, float32 or bfloat16, except states, which are float32.  Every
computation runs in the library's HIP kernels, on the current stream (or on
`stream`); there is no fallback path.  A call with `stream` is put behind what that
stream has to do, not behind work of the current one that forms its inputs, and its
outputs are ready in that stream's order: the caller orders streams that share
tensors.  Inputs may be dropped as soon as a call returns.
"""
from __future__ import annotations

import ctypes

import torch
from torch.autograd import forward_ad

from .fesc import _check, _lib

_u32, _u64, _vp, _sz = ctypes.c_uint32, ctypes.c_uint64, ctypes.c_void_p, ctypes.c_size_t

_TYPES = {torch.float32: 0, torch.bfloat16: 1}
_MOST_TOKEN_STRIDE = 1 << 22    # of the recurrence's arrays


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


def _stream(device):
    """The current stream of a device, as its handle."""
    return torch._C._cuda_getCurrentRawStream(device)


def _on(stream, call, *args):
    """A call on `stream`, which the memory of its tensors is kept for."""
    with torch.cuda.stream(stream):
        out = call(*args)
    for t in args:
        if isinstance(t, torch.Tensor):
            t.record_stream(stream)
    return out


def _once():
    if torch.is_grad_enabled():
        raise RuntimeError("the block in the clear is differentiable once: no create_graph=True")


def _unrecorded(name, *ts):
    """Refuses what a call on addresses would drop without a word: tangents of
    forward-mode differentiation, and the call itself from a trace."""
    if forward_ad._current_level >= 0:
        for t in ts:
            if t is not None and forward_ad.unpack_dual(t).tangent is not None:
                raise NotImplementedError(f"{name}: no forward-mode derivative")
    if torch._C._get_tracing_state() is not None:
        raise NotImplementedError(f"{name}: cannot be traced")


# ---------------------------------------------------------- argument checks

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


def _shape(t, shape, what):
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{what}: shape {tuple(t.shape)}, expected {tuple(shape)}")


def _counts(t, what):
    """Sizes go to the library in 32 bits."""
    if t.shape and max(t.shape) >= 1 << 32:
        raise ValueError(f"{what}: a size of 2^32 or more")


def _dense_tail(t, dims):
    """Whether the last `dims` dimensions are laid out without gaps."""
    step = 1
    for d in range(t.dim() - 1, t.dim() - 1 - dims, -1):
        if t.shape[d] != 1:
            if t.stride(d) != step:
                return False
            step *= t.shape[d]
    return True


def _steps(t):
    """Strides of the first two dimensions, [batch, len, ...]; that of a
    dimension of one entry, which may be anything, is that of a dense one."""
    step = t.shape[2:].numel()
    token = t.stride(1) if t.shape[1] > 1 else step
    return token, t.stride(0) if t.shape[0] > 1 else token * t.shape[1]


def _factor(t, dims, what):
    if t.numel() and not _dense_tail(t, dims):
        raise ValueError(f"{what}: the last {dims} dimension(s) must be contiguous")


def _state(t, shape, what, like):
    _tensor(t, what, like, torch.float32)
    _shape(t, shape, what)
    if not t.is_contiguous():
        raise ValueError(f"{what}: must be contiguous")


# A call's plan: its checked descriptor and workspace sizes, kept by what they
# follow from (types, shapes, strides, device) so that a program that makes
# the same kind of call again does not check it again.
_PLANS = {}
_MOST_PLANS = 4096


def _plan(key, make, args):
    plan = _PLANS.get(key)
    if plan is None:
        plan = make(*args)
        if len(_PLANS) >= _MOST_PLANS:
            _PLANS.clear()
        _PLANS[key] = plan
    return plan


def _key(name, *ts):
    """What a plan follows from; no plan is kept for what is not a tensor."""
    if not isinstance(ts[0], torch.Tensor) or not ts[0].is_cuda:
        raise TypeError(f"{name}: expected CUDA tensors")
    key = [name, torch.cuda.current_device()]
    for t in ts:
        if t is None:
            key.append(None)
        else:
            if not isinstance(t, torch.Tensor):
                raise TypeError(f"{name}: expected tensors, got {type(t).__name__}")
            key += (t.dtype, t.device, t.shape, t.stride())
    return tuple(key)


class _Plan:
    """ref: the descriptor's address; device; workspace sizes, forward and
    backward."""

    __slots__ = ("desc", "ref", "device", "space", "grad_space", "shapes")

    def __init__(self, desc, device):
        self.desc, self.ref, self.device = desc, ctypes.byref(desc), device


def _space(query, *args):
    need = _sz()
    _check(query(*args, ctypes.byref(need)))
    return need.value


def _buffer(size, device):
    return torch.empty(size, dtype=torch.uint8, device=device) if size else None


# ---------------------------------------------------------------- recurrence

def _scan_plan(x, la, B, C, h0, dy=None):
    _tensor(x, "x")
    for t, what in ((la, "la"), (B, "B"), (C, "C")):
        _tensor(t, what, x)
    if x.dim() != 4 or B.dim() != 4:
        raise ValueError("x, B: expected [batch, len, heads or groups, width]")
    _shape(la, x.shape[:3], "la")
    _shape(B, (*x.shape[:2], *B.shape[2:]), "B")
    _shape(C, B.shape, "C")
    _counts(x, "x"), _counts(B, "B")
    _factor(x, 2, "x"), _factor(la, 1, "la"), _factor(B, 2, "B"), _factor(C, 2, "C")
    b, n, H, P = x.shape
    G, N = B.shape[2:]
    if h0 is not None:
        _state(h0, (b, H, P, N), "h0", x)
    # without dy: the strides of a contiguous one
    d = _ScanDesc(_TYPES[x.dtype], b, n, H, P, G, N, *_steps(x), *_steps(la), *_steps(B),
                  *_steps(C), *((H * P, n * H * P) if dy is None else _steps(dy)))
    plan = _Plan(d, x.device)
    plan.space = _space(_lib.fesc_clear_scan_workspace, plan.ref, 0)
    plan.grad_space = _space(_lib.fesc_clear_scan_workspace, plan.ref, 1)
    plan.shapes = (tuple(x.shape), (b, H, P, N))
    return plan


def _scan_forward(plan, x, la, B, C, h0, want_state):
    device = plan.device
    y = torch.empty(plan.shapes[0], dtype=x.dtype, device=device)
    h = torch.empty(plan.shapes[1], dtype=torch.float32, device=device) if want_state else None
    w = _buffer(plan.space, device)
    _check(_lib.fesc_clear_scan(plan.ref, x.data_ptr(), la.data_ptr(), B.data_ptr(), C.data_ptr(),
                                _p(h0), y.data_ptr(), _p(h), _p(w), plan.space,
                                _stream(device.index)))
    return y, h


class _Scan(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, la, B, C, h0, want_state, plan):
        ctx.set_materialize_grads(False)
        ctx.plan = plan
        ctx.save_for_backward(x, la, B, C, h0)
        y, h = _scan_forward(plan, x, la, B, C, h0, want_state)
        return (y, h) if want_state else y

    @staticmethod
    def backward(ctx, dy, dh=None):
        _once()
        _unrecorded("scan", dy, dh)
        x, la, B, C, h0 = ctx.saved_tensors
        if dy is None:
            if dh is None:
                return (None,) * 7
            dy = torch.zeros_like(x, memory_format=torch.contiguous_format)
        elif not _dense_tail(dy, 2) or _steps(dy)[0] > _MOST_TOKEN_STRIDE:
            dy = dy.contiguous()
        if dh is not None:
            dh = dh.contiguous()
        plan = ctx.plan if dy.is_contiguous() else _plan(
            _key("scan gradient", x, la, B, C, h0, dy), _scan_plan, (x, la, B, C, h0, dy))
        dx, dla, db, dc = (torch.empty(t.shape, dtype=t.dtype, device=plan.device)
                           for t in (x, la, B, C))
        dh0 = torch.empty_like(h0) if h0 is not None and ctx.needs_input_grad[4] else None
        w = _buffer(plan.grad_space, plan.device)
        _check(_lib.fesc_clear_scan_bwd(
            plan.ref, x.data_ptr(), la.data_ptr(), B.data_ptr(), C.data_ptr(), _p(h0),
            dy.data_ptr(), _p(dh), dx.data_ptr(), dla.data_ptr(), db.data_ptr(), dc.data_ptr(),
            _p(dh0), _p(w), plan.grad_space, _stream(plan.device.index)))
        return dx, dla, db, dc, dh0, None, None


def scan(x, la, B, C, h0=None, return_state=False, stream=None):
    """Outputs y [batch, len, heads, head_dim] of the recurrence, and with
    `return_state` the final state as well.

    x [batch, len, heads, head_dim], la [batch, len, heads] (log decays, <= 0;
    -inf resets the state, whatever it was), B and C [batch, len, groups, d_state]; the first
    two dimensions may have any strides, so slices of a wider projection do.
    h0 and the returned state: float32 [batch, heads, head_dim, d_state].
    In bfloat16 y is rounded once; with `return_state` the states behind it are
    held to 2^-24 instead of 2^-18, so it need not be the same to the last bit.
    Differentiable (once) with respect to all five.
    """
    if stream is not None:
        return _on(stream, scan, x, la, B, C, h0, return_state)
    plan = _plan(_key("scan", x, la, B, C, h0), _scan_plan, (x, la, B, C, h0))
    if torch.is_grad_enabled() and (x.requires_grad or la.requires_grad or B.requires_grad
                                    or C.requires_grad
                                    or (h0 is not None and h0.requires_grad)):
        return _Scan.apply(x, la, B, C, h0, return_state, plan)
    _unrecorded("scan", x, la, B, C, h0)
    y, h = _scan_forward(plan, x, la, B, C, h0, return_state)
    return (y, h) if return_state else y


def _step_plan(x, la, B, C, state, slots):
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
    _counts(x, "x"), _counts(B, "B"), _counts(state, "state")
    _factor(x, 2, "x"), _factor(la, 1, "la"), _factor(B, 2, "B"), _factor(C, 2, "C")
    _state(state, (state.shape[0] if state.dim() else 0, H, P, N), "state", x)
    if slots is not None:
        _tensor(slots, "slots", x, torch.int32)
        _shape(slots, (rows,), "slots")
        if not slots.is_contiguous():
            raise ValueError("slots: must be contiguous")
    plan = _Plan(_ScanDesc(_TYPES[x.dtype], rows, 1, H, P, G, N,
                           *(s for t in (x, la, B, C) for s in _steps(t[:, None])), 0, 0), x.device)
    plan.shapes = (rows, H, P)
    return plan


def scan_step(x, la, B, C, state, slots=None, stream=None):
    """One token for each row: updates `state` in place and returns y
    [rows, heads, head_dim].

    x [rows, heads, head_dim], la [rows, heads], B and C [rows, groups,
    d_state]; state float32 [pool, heads, head_dim, d_state].  Row i uses state
    slots[i] (int32, None: i); a slot outside the pool (-1) marks an idle row,
    whose y is zero.  No two rows may name one slot.  A new sequence may take
    over a slot by a first token of la = -inf.  Not differentiable.
    """
    if stream is not None:
        return _on(stream, scan_step, x, la, B, C, state, slots)
    plan = _plan(_key("scan_step", x, la, B, C, state, slots), _step_plan,
                 (x, la, B, C, state, slots))
    if torch.is_grad_enabled() and (x.requires_grad or la.requires_grad or B.requires_grad
                                    or C.requires_grad or state.requires_grad):
        raise ValueError("scan_step is not differentiable: use scan, or torch.no_grad()")
    _unrecorded("scan_step", x, la, B, C, state)
    device = plan.device
    y = torch.empty(plan.shapes, dtype=x.dtype, device=device)
    _check(_lib.fesc_clear_scan_step(plan.ref, x.data_ptr(), la.data_ptr(), B.data_ptr(),
                                     C.data_ptr(), state.data_ptr(), state.shape[0], _p(slots),
                                     y.data_ptr(), _stream(device.index)))
    # a gradient that was to read the states as they were is refused
    torch.autograd.graph.increment_version(state)
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


def _even(t):
    """A gradient whose rows lie evenly."""
    try:
        _rows(t, "")
        return t
    except ValueError:
        return t.contiguous()


def _norm_plan(arrays, vectors, eps, grads=()):
    """From (name, tensor) pairs: the row arrays, the weight vectors, and the
    incoming gradients by the names of their strides (absent: None)."""
    what, first = arrays[0]
    _tensor(first, what)
    if first.dim() == 0:
        raise ValueError(f"{what}: expected [..., width]")
    for what, t in arrays[1:]:
        _tensor(t, what, first)
        _shape(t, first.shape, what)
    for what, v in vectors:
        _tensor(v, what, first)
        _shape(v, first.shape[-1:], what)
        if not v.is_contiguous():
            raise ValueError(f"{what}: must be contiguous")
    w = first.shape[-1]
    _counts(vectors[0][1], vectors[0][0])
    d = _NormDesc(_TYPES[first.dtype], w, first.numel() // w if w else 0, eps)
    for what, t in arrays:
        setattr(d, what + "_row", _rows(t, what))
    d.du_row = d.dr_row = w                 # of contiguous gradients, unless given
    for what, t in grads:
        setattr(d, what + "_row", _rows(t, what) if t is not None else w)
    plan = _Plan(d, first.device)
    plan.grad_space = _space(_lib.fesc_clear_norm_workspace, plan.ref)
    plan.shapes = tuple(first.shape)
    return plan


def _gated_plan(m, x, z, skip, w, eps, *du):
    return _norm_plan((("m", m), ("x", x), ("z", z)), (("skip", skip), ("w", w)), eps,
                      tuple(zip(("du",), du)))


def _gated_forward(plan, m, x, z, skip, w):
    u = torch.empty(plan.shapes, dtype=m.dtype, device=plan.device)
    _check(_lib.fesc_clear_norm_gated(plan.ref, m.data_ptr(), x.data_ptr(), z.data_ptr(),
                                      skip.data_ptr(), w.data_ptr(), u.data_ptr(),
                                      _stream(plan.device.index)))
    return u


class _Gated(torch.autograd.Function):
    @staticmethod
    def forward(ctx, m, x, z, skip, w, eps, plan):
        ctx.eps, ctx.plan = eps, plan
        ctx.save_for_backward(m, x, z, skip, w)
        return _gated_forward(plan, m, x, z, skip, w)

    @staticmethod
    def backward(ctx, du):
        _once()
        _unrecorded("norm_gated", du)
        saved = m, x, z, skip, w = ctx.saved_tensors
        if du.is_contiguous():
            plan = ctx.plan
        else:
            du = _even(du)
            plan = _plan((ctx.eps, _key("gated gradient", *saved, du)), _gated_plan,
                         (*saved, ctx.eps, du))
        dm, dx, dz, dskip, dw = (torch.empty(t.shape, dtype=t.dtype, device=plan.device)
                                 for t in saved)
        ws = _buffer(plan.grad_space, plan.device)
        _check(_lib.fesc_clear_norm_gated_bwd(
            plan.ref, m.data_ptr(), x.data_ptr(), z.data_ptr(), skip.data_ptr(), w.data_ptr(),
            du.data_ptr(), dm.data_ptr(), dx.data_ptr(), dz.data_ptr(), dskip.data_ptr(),
            dw.data_ptr(), _p(ws), plan.grad_space, _stream(plan.device.index)))
        return dm, dx, dz, dskip, dw, None, None


def norm_gated(m, x, z, skip, w, eps=1e-5, stream=None):
    """u = v w / sqrt(mean v^2 + eps) over the last dimension, with
    v = (m + skip x) silu(z): m the recurrence's output, x its input (the skip
    connection), z the gate, all [..., width] with rows of any one stride;
    skip and w [width].  Differentiable (once) with respect to all five."""
    if stream is not None:
        return _on(stream, norm_gated, m, x, z, skip, w, eps)
    eps = float(eps)                        # by its value: plans are kept by it
    plan = _plan((eps, _key("norm_gated", m, x, z, skip, w)), _gated_plan, (m, x, z, skip, w, eps))
    if torch.is_grad_enabled() and (m.requires_grad or x.requires_grad or z.requires_grad
                                    or skip.requires_grad or w.requires_grad):
        return _Gated.apply(m, x, z, skip, w, eps, plan)
    _unrecorded("norm_gated", m, x, z, skip, w)
    return _gated_forward(plan, m, x, z, skip, w)


def _residual_plan(o, r, scale, w, eps, *grads):
    return _norm_plan((("o", o), ("r", r)), (("scale", scale), ("w", w)), eps,
                      tuple(zip(("dr", "du"), grads)))


def _residual_forward(plan, o, r, scale, w):
    new = torch.empty(plan.shapes, dtype=o.dtype, device=plan.device)
    u = torch.empty(plan.shapes, dtype=o.dtype, device=plan.device)
    _check(_lib.fesc_clear_norm_residual(plan.ref, o.data_ptr(), r.data_ptr(), scale.data_ptr(),
                                         w.data_ptr(), new.data_ptr(), u.data_ptr(),
                                         _stream(plan.device.index)))
    return new, u


class _Residual(torch.autograd.Function):
    @staticmethod
    def forward(ctx, o, r, scale, w, eps, plan):
        ctx.set_materialize_grads(False)
        ctx.eps, ctx.plan = eps, plan
        ctx.save_for_backward(o, r, scale, w)
        return _residual_forward(plan, o, r, scale, w)

    @staticmethod
    def backward(ctx, dnew, du):
        _once()
        _unrecorded("norm_residual", dnew, du)
        saved = o, r, scale, w = ctx.saved_tensors
        if dnew is None and du is None:
            return (None,) * 6
        if (du is None or du.is_contiguous()) and (dnew is None or dnew.is_contiguous()):
            plan = ctx.plan
        else:
            du = _even(du) if du is not None else None
            dnew = _even(dnew) if dnew is not None else None
            plan = _plan((ctx.eps, _key("residual gradient", *saved, dnew, du)), _residual_plan,
                         (*saved, ctx.eps, dnew, du))
        do, dr, dscale, dw = (torch.empty(t.shape, dtype=t.dtype, device=plan.device)
                              for t in saved)
        ws = _buffer(plan.grad_space, plan.device)
        _check(_lib.fesc_clear_norm_residual_bwd(
            plan.ref, o.data_ptr(), r.data_ptr(), scale.data_ptr(), w.data_ptr(), _p(du),
            _p(dnew), do.data_ptr(), dr.data_ptr(), dscale.data_ptr(), dw.data_ptr(), _p(ws),
            plan.grad_space, _stream(plan.device.index)))
        return do, dr, dscale, dw, None, None


def norm_residual(o, r, scale, w, eps=1e-5, stream=None):
    """(r_new, u): r_new = r + scale o, the residual stream after a block's
    output o, and u = r_new w / sqrt(mean r_new^2 + eps), the next block's
    input.  o and r [..., width] with rows of any one stride; scale and w
    [width].  u is formed from r_new before it is rounded.  Differentiable
    (once) with respect to all four."""
    if stream is not None:
        return _on(stream, norm_residual, o, r, scale, w, eps)
    eps = float(eps)                        # by its value: plans are kept by it
    plan = _plan((eps, _key("norm_residual", o, r, scale, w)), _residual_plan,
                 (o, r, scale, w, eps))
    if torch.is_grad_enabled() and (o.requires_grad or r.requires_grad or scale.requires_grad
                                    or w.requires_grad):
        return _Residual.apply(o, r, scale, w, eps, plan)
    _unrecorded("norm_residual", o, r, scale, w)
    return _residual_forward(plan, o, r, scale, w)
