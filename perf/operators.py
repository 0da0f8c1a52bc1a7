"""The operators of the block in the clear: which calls are measured, with
their sizes, their inputs, their plain forms and what they compute in 64 bits.

One pass is one call as a user's program makes it: the recurrence over a batch
of prompts, its training step, one token for each served sequence, and the
norms before and after the block with their training steps.  The base shape is
the one that the encrypted scan runs: 24 heads of 64 channels, a state of 128,
768 features, 1536 channels.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------- cases

def listed():
    base = dict(heads=24, head_dim=64, groups=1, d_state=128)
    return [
        # one token of one served sequence: the smallest call, all latency
        dict(name="step_one", op="step", dtype="bf16", batch=1, pool=1, idle=0, **base),
        # one token for each of 250 sequences whose states lie in a pool, in
        # any order, some rows of the batch idle
        dict(name="step_pool", op="step", dtype="bf16", batch=250, pool=300, idle=6, **base),
        # short odd prompts that go on from a state, in 32 bits
        dict(name="scan_short_f32", op="scan", dtype="f32", train=False, batch=3, len=77,
             state=True, resets=0, **base),
        # one prompt of the encrypted scan's own length: few rows, a long axis
        dict(name="scan_prompt", op="scan", dtype="bf16", train=False, batch=1, len=2048,
             state=True, resets=0, **base),
        # a batch of prompts
        dict(name="scan_batch", op="scan", dtype="bf16", train=False, batch=8, len=2048,
             state=True, resets=0, **base),
        # one long packed sequence of many documents, each begun by a reset
        dict(name="scan_long", op="scan", dtype="bf16", train=False, batch=1, len=50001,
             state=False, resets=40, **base),
        # a training step on a batch
        dict(name="train_batch", op="scan", dtype="bf16", train=True, batch=8, len=2048,
             state=False, resets=0, **base),
        # a training step in 32 bits, odd length, two groups, states in and out
        dict(name="train_f32", op="scan", dtype="f32", train=True, batch=2, len=333, heads=6,
             head_dim=32, groups=2, d_state=48, state=True, resets=3),
        # skip, gate and norm of four served tokens
        dict(name="gated_rows", op="gated", dtype="bf16", train=False, rows=4, width=1536),
        # the same in a training step, one batch of 8 x 2048 tokens
        dict(name="gated_train", op="gated", dtype="bf16", train=True, rows=16384, width=1536),
        # residual and norm before the next block, an odd width in 32 bits
        dict(name="residual_odd_f32", op="residual", dtype="f32", train=False, rows=1001,
             width=767),
        # the same in a training step, one batch of 8 x 2048 tokens
        dict(name="residual_train", op="residual", dtype="bf16", train=True, rows=16384,
             width=768),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the same ranges."""
    op = rng.choice(["step", "scan", "scan", "scan", "gated", "residual"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op in ("gated", "residual"):
        width = _log_int(rng, 24, 4096)
        if rng.random() < 0.5:
            width = -(-width // 64) * 64
        rows = _log_int(rng, 1, max(1, min(16384, 6000000 // width)))
        return dict(op=op, dtype=dtype, train=rng.random() < 0.5, rows=rows, width=width)
    groups = rng.choice([1, 1, 2, 4])
    c = dict(op=op, dtype=dtype, heads=groups * rng.randint(1, 24 // groups),
             head_dim=rng.choice([16, 32, 48, 64, 64, 64, 100, 128]), groups=groups,
             d_state=rng.choice([16, 33, 48, 64, 64, 100, 128, 128, 128]))
    head = c["heads"] * c["head_dim"] * c["d_state"]
    if op == "step":
        batch = _log_int(rng, 1, max(1, min(512, 50000000 // head)))
        return dict(c, batch=batch, pool=batch + rng.randint(0, 40), idle=rng.randint(0, batch // 4))
    train = rng.random() < 0.4
    tokens = 1600000000 // head if train else 8000000000 // head
    if dtype == "f32":
        tokens //= 4
    length = _log_int(rng, 1, min(tokens, 8192 if train else 40000))
    return dict(c, train=train, batch=_log_int(rng, 1, max(1, min(32, tokens // length))),
                len=length, state=rng.random() < 0.5,
                resets=0 if rng.random() < 0.5 else rng.randint(1, 8))


# ------------------------------------------------------------------ inputs

def _factors(case, g, lead):
    """x, log decay, B and C of `lead` tokens: decays from e^-1 a token to
    long memories of some 500 tokens, head by head."""
    t = TYPES[case["dtype"]]
    H, P, G, N = (case[k] for k in ("heads", "head_dim", "groups", "d_state"))

    def normal(*s):
        return torch.randn(*lead, *s, generator=g, device=DEV)

    rate = torch.logspace(-3, 0, H, device=DEV)
    x, B, C = normal(H, P).to(t), normal(G, N).to(t), normal(G, N).to(t)
    la = (-torch.nn.functional.softplus(normal(H)) * rate).to(t)
    return x, la, B, C


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    t = TYPES[case["dtype"]]
    s = {"case": case}
    if case["op"] in ("gated", "residual"):
        rows, E = case["rows"], case["width"]

        def normal(*shape, by=1.0, at=0.0):
            return (at + by * torch.randn(*shape, generator=g, device=DEV)).to(t)

        names = ("m", "x", "z") if case["op"] == "gated" else ("o", "r")
        for k in names:
            s[k] = normal(rows, E)
        s["skip" if case["op"] == "gated" else "scale"] = normal(E, by=0.3, at=1.0)
        s["w"] = normal(E, by=0.1, at=1.0)
        if case["train"]:
            s["du"] = normal(rows, E)
            if case["op"] == "residual":
                s["dr"] = normal(rows, E)
            for k in _leaves(case):
                s[k].requires_grad_()
        return s
    H, P, N = case["heads"], case["head_dim"], case["d_state"]
    if case["op"] == "step":
        n, pool = case["batch"], case["pool"]
        s["x"], s["la"], s["B"], s["C"] = _factors(case, g, (n,))
        s["state"] = torch.randn(pool, H, P, N, generator=g, device=DEV)
        slots = torch.randperm(pool, generator=g, device=DEV)[:n]
        if case["idle"]:
            slots[torch.randperm(n, generator=g, device=DEV)[:case["idle"]]] = -1
        s["slots"] = slots.to(torch.int32)
        return s
    b, L = case["batch"], case["len"]
    s["x"], s["la"], s["B"], s["C"] = _factors(case, g, (b, L))
    if case["resets"]:
        at = torch.randint(0, L, (case["resets"],), generator=g, device=DEV)
        s["la"][:, at] = -math.inf
    s["h0"] = torch.randn(b, H, P, N, generator=g, device=DEV) if case["state"] else None
    if case["train"]:
        s["dy"] = torch.randn(b, L, H, P, generator=g, device=DEV).to(t)
        if case["state"]:
            s["dh"] = torch.randn(b, H, P, N, generator=g, device=DEV)
        for k in _leaves(case):
            s[k].requires_grad_()
    return s


def _leaves(case):
    return {"gated": ["m", "x", "z", "skip", "w"], "residual": ["o", "r", "scale", "w"],
            "scan": ["x", "la", "B", "C"] + (["h0"] if case.get("state") else [])}[case["op"]]


# ------------------------------------------------------------- plain forms

def _segment_sums(la):
    """[..., Q] -> [..., Q, Q]: entry (s, r) = sum of la over r < k <= s, -inf
    for r > s."""
    Q = la.shape[-1]
    i = torch.arange(Q, device=la.device)
    t = la[..., :, None].expand(*la.shape, Q).masked_fill(i[:, None] <= i, 0.0).cumsum(-2)
    return t.masked_fill(i[:, None] < i, -math.inf)


def _plain_scan(x, la, B, C, h0):
    """The recurrence in chunks, each a product with the matrix of decays
    between its tokens, and the chunks' states likewise."""
    t, (b, L, H, P), (G, N) = x.dtype, x.shape, B.shape[2:]
    Q = 64 if L <= 4096 else 256
    n = -(-L // Q)

    def chunks(v, to):  # [b, L, k, ...] -> [b, n, to, Q, ...]
        v = torch.nn.functional.pad(v.float(), [0, 0] * (v.dim() - 2) + [0, n * Q - L])
        return v.unflatten(1, (n, Q)).transpose(2, 3).repeat_interleave(to // v.shape[2], 2)

    xc, ac, Bc, Cc = chunks(x, H), chunks(la, H), chunks(B, G), chunks(C, G)
    D = _segment_sums(ac).exp()
    W = D * (Cc @ Bc.transpose(-1, -2)).repeat_interleave(H // G, 2)
    Bc, Cc = Bc.repeat_interleave(H // G, 2), Cc.repeat_interleave(H // G, 2)
    S = (D[..., -1, :, None] * xc).transpose(-1, -2) @ Bc
    S = torch.cat([torch.zeros_like(S[:, :1]) if h0 is None else h0[:, None], S], 1)
    total = torch.nn.functional.pad(ac.sum(-1), (0, 0, 1, 0)).transpose(1, 2)
    S = (_segment_sums(total).exp() @ S.transpose(1, 2).flatten(3)).unflatten(-1, (P, N))
    S = S.transpose(1, 2)
    y = W @ xc + ac.cumsum(-1).exp()[..., None] * (Cc @ S[:, :-1].transpose(-1, -2))
    return y.transpose(2, 3).flatten(1, 2)[:, :L].to(t), S[:, -1]


def _plain_step(x, la, B, C, state, slots):
    rep = x.shape[1] // B.shape[1]
    B, C = (v.float().repeat_interleave(rep, 1)[:, :, None] for v in (B, C))
    at = slots.long()
    S = la.float().exp()[..., None, None] * state[at] + x.float()[..., None] * B
    y = ((S * C).sum(-1) * (at >= 0)[:, None, None]).to(x.dtype)
    state[at[at >= 0]] = S[at >= 0]
    return y


def _plain_gated(m, x, z, skip, w, eps):
    m, x, z, skip, w = (v.float() for v in (m, x, z, skip, w))
    v = (m + skip * x) * z * torch.sigmoid(z)
    return v * torch.rsqrt((v * v).mean(-1, keepdim=True) + eps) * w


def _plain_residual(o, r, scale, w, eps):
    o, r, scale, w = (v.float() for v in (o, r, scale, w))
    new = r + scale * o
    return new, new * torch.rsqrt((new * new).mean(-1, keepdim=True) + eps) * w


EPS = 1e-5


def run(s):
    case = s["case"]
    t = TYPES[case["dtype"]]
    if own:
        from paper_2608_17442_amd import clear
    if case["op"] == "step":
        if own:
            y = clear.scan_step(s["x"], s["la"], s["B"], s["C"], s["state"], slots=s["slots"])
        else:
            y = _plain_step(s["x"], s["la"], s["B"], s["C"], s["state"], s["slots"])
        return {"y": y, "state": s["state"]}
    if case["op"] == "scan":
        if own:
            out = clear.scan(s["x"], s["la"], s["B"], s["C"], h0=s["h0"],
                             return_state=case["state"])
            y, h = out if case["state"] else (out, None)
        else:
            y, h = _plain_scan(s["x"], s["la"], s["B"], s["C"], s["h0"])
        out = {"y": y, "h": h} if case["state"] else {"y": y}
        down = [s["dy"], s["dh"]] if case["train"] and case["state"] else [s.get("dy")]
    elif case["op"] == "gated":
        if own:
            u = clear.norm_gated(s["m"], s["x"], s["z"], s["skip"], s["w"], eps=EPS)
        else:
            u = _plain_gated(s["m"], s["x"], s["z"], s["skip"], s["w"], EPS).to(t)
        out, down = {"u": u}, [s.get("du")]
    else:
        if own:
            r, u = clear.norm_residual(s["o"], s["r"], s["scale"], s["w"], eps=EPS)
        else:
            r, u = (v.to(t) for v in _plain_residual(s["o"], s["r"], s["scale"], s["w"], EPS))
        out, down = {"r": r, "u": u}, [s.get("dr"), s.get("du")]
    if case["train"]:
        names = _leaves(case)
        grads = torch.autograd.grad(list(out.values()), [s[k] for k in names], down)
        out.update({"d" + k: v for k, v in zip(names, grads)})
    return out


# ---------------------------------------------------------- work and right answers

def work(case):
    """Each input read once, each output written once; the products of the
    recurrence itself (two per token and state entry, five in its gradient)."""
    T = 2 if case["dtype"] == "bf16" else 4
    if case["op"] in ("gated", "residual"):
        n = case["rows"] * case["width"]
        arrays = 4
        if case["train"]:  # inputs, their gradients, outputs and the incoming gradients
            arrays = 8
        return {"bytes": n * arrays * T + 4 * case["width"] * T, "flops": 20 * n * arrays / 4}
    H, P, G, N = (case[k] for k in ("heads", "head_dim", "groups", "d_state"))
    factors = H * P + H + 2 * G * N
    if case["op"] == "step":
        rows = case["batch"] - case["idle"]
        return {"bytes": rows * (8 * H * P * N + T * factors) + case["batch"] * T * H * P,
                "flops": 5 * rows * H * P * N}
    tokens = case["batch"] * case["len"]
    state = 4 * case["batch"] * H * P * N * (2 if case["state"] else 0)
    if case["train"]:  # factors and dy in, y and the factors' gradients out
        return {"bytes": tokens * T * (2 * factors + 2 * H * P) + 2 * state,
                "flops": 14 * tokens * H * P * N}
    return {"bytes": tokens * T * (factors + H * P) + state, "flops": 4 * tokens * H * P * N}


def exact(case, seed):
    def exact_scan(s):
        """Token by token, from the definition; the gradient of a log decay from
        the difference of <dy, y> and <dx, x>, summed from the end."""
        d = {k: s[k].detach().double() for k in ("x", "la", "B", "C", "h0", "dy", "dh")
             if s.get(k) is not None}
        x, a, B, C = d["x"], d["la"].exp(), d["B"], d["C"]
        b, L, H, P = x.shape
        G, N = B.shape[2:]
        S = d["h0"].clone() if "h0" in d else x.new_zeros(b, H, P, N)
        y = torch.empty_like(x)
        dC = torch.empty_like(C)

        def heads(v):
            return v.repeat_interleave(H // G, 1)

        for t in range(L):
            S = a[:, t, :, None, None] * S + x[:, t, :, :, None] * heads(B[:, t])[:, :, None]
            y[:, t] = (S @ heads(C[:, t])[..., None])[..., 0]
            if case["train"]:
                dC[:, t] = (d["dy"][:, t, :, None] @ S)[:, :, 0].unflatten(1, (G, -1)).sum(2)
        out = {"y": y, "h": S} if case["state"] else {"y": y}
        if not case["train"]:
            return out
        R = d["dh"].clone() if "dh" in d else torch.zeros_like(S)
        run_la = (R * S).sum((-1, -2))
        dx, dla, dB = torch.empty_like(x), torch.empty_like(a), torch.empty_like(B)
        for t in reversed(range(L)):
            dy = d["dy"][:, t]
            R = R + dy[..., None] * heads(C[:, t])[:, :, None]
            dx[:, t] = (R @ heads(B[:, t])[..., None])[..., 0]
            dB[:, t] = (x[:, t, :, None] @ R)[:, :, 0].unflatten(1, (G, -1)).sum(2)
            run_la = run_la + (dy * y[:, t]).sum(-1) - (dx[:, t] * x[:, t]).sum(-1)
            dla[:, t] = run_la
            R = a[:, t, :, None, None] * R
        out.update(dx=dx, dla=dla, dB=dB, dC=dC)
        if "h0" in d:
            out["dh0"] = R
        return out

    def exact_norm(v, w, du):
        """u = v rstd w and, with du, the gradients with respect to v and w."""
        rstd = 1.0 / torch.sqrt(v.square().mean(-1, keepdim=True) + EPS)
        n = v * rstd
        if du is None:
            return n * w, None, None
        g = du * w
        return n * w, rstd * (g - n * (g * n).mean(-1, keepdim=True)), (du * n).sum(0)

    s = prepare(case, seed)
    if case["op"] == "scan":
        return exact_scan(s)
    d = {k: v.detach().double() for k, v in s.items() if torch.is_tensor(v) and k != "slots"}
    if case["op"] == "step":
        rep = case["heads"] // case["groups"]
        y = torch.zeros_like(d["x"])
        for i, at in enumerate(s["slots"].tolist()):
            if at >= 0:
                S = d["state"][at]
                S *= d["la"][i].exp()[:, None, None]
                S += d["x"][i][..., None] * d["B"][i].repeat_interleave(rep, 0)[:, None]
                y[i] = (S @ d["C"][i].repeat_interleave(rep, 0)[..., None])[..., 0]
        return {"y": y, "state": d["state"]}
    if case["op"] == "gated":
        sig = 1.0 / (1.0 + torch.exp(-d["z"]))
        q, gate = d["m"] + d["skip"] * d["x"], d["z"] * sig
        u, dv, dw = exact_norm(q * gate, d["w"], d.get("du"))
        if not case["train"]:
            return {"u": u}
        dq = dv * gate
        return {"u": u, "dm": dq, "dx": dq * d["skip"], "dz": dv * q * (sig + gate * (1.0 - sig)),
                "dskip": (dq * d["x"]).sum(0), "dw": dw}
    r = d["r"] + d["scale"] * d["o"]
    u, dv, dw = exact_norm(r, d["w"], d.get("du"))
    if not case["train"]:
        return {"r": r, "u": u}
    dv = dv + d["dr"]
    return {"r": r, "u": u, "do": dv * d["scale"], "dr": dv, "dscale": (dv * d["o"]).sum(0),
            "dw": dw}
