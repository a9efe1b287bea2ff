"""The gated recurrence, its gradients, 8-bit values and activations in 64 bits, row by row from their definitions, with bounds of
what 32-bit arithmetic may be off by.

Errors are counted in u = 2^-24, half a unit of a 32-bit float.  A bound E runs along with each value: a row's factor is off by
K u relative to itself (K counts the roundings of the gate, below), and each product and sum by u, so a value h = a h' + b with
magnitudes S = a S' + |b| is off by E = a E' + K u S.  Pieces of rows that are joined as P h + H only group the same products and sums:
a term's path through n rows meets n factors and at most 3 n + 3 products and sums in either order."""
import torch

U = 2.0 ** -24
F64 = torch.float64
CHUNK, BLOCK = 64, 32
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def roundings(dtype, g):
    """K: expf is off by 2 ulp = 4 u, its 16-bit stand-in by 2 + 1.16 |z| ulp (the documented bounds of both); 1 + e: u; the quotient 2 ulp =
    4 u; one minus it u (relative to the larger part, at least 1/2: 2 u); then the products and sums above, 4, and b = w x, 1."""
    z = min(float(g.abs().max()), 88.0) if g.numel() else 0.0
    return (4 if dtype == torch.float32 else 2 * (2 + 1.16 * z)) + 1 + 4 + 2 + 4 + 1


def tiny(dtype):
    """What a result below the type's normal numbers may be off by."""
    return {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -25}[dtype]


def eight(v, fmt):
    """The values (64 bits) that stand for v in blocks of 32 along the last dim."""
    v = v.to(F64)
    out = torch.empty_like(v)
    for lo in range(0, v.shape[-1], BLOCK):
        p = v[..., lo:lo + BLOCK]
        finite = torch.isfinite(p)
        top = torch.where(finite, p.abs(), 0.0).amax(-1, keepdim=True)
        k = torch.where(top > 0, torch.frexp(top)[1].to(F64) - 1, -1000.0)
        scale = torch.exp2((k - (6 if fmt == "int8" else 7)).clamp(min=-126))
        m = torch.where(finite, p / scale, 0.0)
        if fmt == "int8":
            q = torch.round(m).clamp(-127, 127)
        else:
            step = torch.exp2((torch.frexp(m.abs())[1].to(F64) - 1).clamp(min=-6) - 3)
            q = (torch.round(m / step) * step).clamp(-240, 240)
        out[..., lo:lo + BLOCK] = torch.where(finite, q * scale, float("nan"))
    return out


def act(kind, x):
    """f(x), f'(x)"""
    if kind == "tanh":
        return torch.tanh(x), 1.0 / torch.cosh(x) ** 2
    if kind == "silu":
        s = torch.sigmoid(x)
        return x * s, s + x * s * torch.sigmoid(-x)
    c = (2.0 / torch.pi) ** 0.5
    z = c * (x + 0.044715 * x ** 3)
    s = torch.sigmoid(2 * z)
    return x * s, s + 2 * x * s * torch.sigmoid(-2 * z) * c * (1 + 3 * 0.044715 * x ** 2)


def gate_parts(g):
    return torch.sigmoid(g), torch.sigmoid(-g)


def forward(g, x, h0, lengths, mix):
    """h, h_last, states ahead of each row, and bounds of their errors (before the last rounding)."""
    B, T, C = g.shape
    K = roundings(g.dtype, g[torch.isfinite(g)])
    g, x = g.to(F64), x.to(F64)
    n = torch.full((B,), T, device=g.device) if lengths is None else lengths.to(torch.int64).clamp(0, T)
    h = torch.zeros(B, C, dtype=F64, device=g.device) if h0 is None else h0.to(F64)
    S, E = h.abs(), torch.zeros_like(h)
    rows, errs, ahead, ahead_err = [], [], [], []
    a, w = gate_parts(g)
    b = w * x if mix else x
    for t in range(T):
        on = (n > t)[:, None]
        ahead.append(h)
        ahead_err.append(E)
        at, bt = a[:, t], b[:, t]
        S_new = at * S + bt.abs()
        E = torch.where(on, at * E + K * U * S_new, E)
        h = torch.where(on, at * h + bt, h)
        S = torch.where(on, S_new, S)
        rows.append(torch.where(on, h, 0.0))
        errs.append(torch.where(on, E, 0.0))
    stack = (lambda r: torch.stack(r, 1)) if T else (lambda r: g)
    return stack(rows), h, stack(ahead), stack(errs), E, stack(ahead_err)


def backward(g, x, h0, lengths, mix, dh, dh_last, fmt=None):
    """dg, dx, dh0 and bounds of their errors (before the last rounding)."""
    B, T, C = g.shape
    K = roundings(g.dtype, g[torch.isfinite(g)])
    _, _, ahead, _, _, ahead_err = forward(g, x, h0, lengths, mix)
    n = torch.full((B,), T, device=g.device) if lengths is None else lengths.to(torch.int64).clamp(0, T)
    if fmt is not None:
        live = (torch.arange(T, device=g.device)[None] < n[:, None])[:, :, None]
        # rows behind a sequence are not data: they take no part in anything
        g, x = torch.where(live, eight(g, "int8"), 0.0), torch.where(live, eight(x, fmt), 0.0)
    g, x = g.to(F64), x.to(F64)
    a, w = gate_parts(g)
    b = w * x if mix else x
    before, before_err = [], []
    for t in range(T):
        if fmt is None or t % CHUNK == 0:
            h, E, S = ahead[:, t], ahead_err[:, t], ahead[:, t].abs()
        before.append(h)
        before_err.append(E)
        S = a[:, t] * S + b[:, t].abs()
        E = a[:, t] * E + K * U * S
        h = a[:, t] * h + b[:, t]
    if fmt is None:                          # formed again from the state ahead of the chunk: the same sums once more
        before_err = [2 * e for e in before_err]
    zero = torch.zeros(B, C, dtype=F64, device=g.device)
    mu = zero if dh_last is None else dh_last.to(F64)
    S, E = mu.abs(), zero
    dg, dx, eg, ex = [None] * T, [None] * T, [None] * T, [None] * T
    for t in range(T - 1, -1, -1):
        on = (n > t)[:, None]
        d = zero if dh is None else dh[:, t].to(F64)
        lam, Sl = d + mu, d.abs() + S
        El = E + U * Sl
        diff = before[t] - x[:, t] if mix else before[t]
        Ed = before_err[t] + U * (before[t].abs() + x[:, t].abs())
        f = a[:, t] * w[:, t]
        dg[t] = torch.where(on, lam * f * diff, 0.0)
        eg[t] = torch.where(on, f * (El * diff.abs() + lam.abs() * Ed + El * Ed + 2 * K * U * Sl * diff.abs()), 0.0)
        wt = w[:, t] if mix else 1.0
        dx[t] = torch.where(on, lam * wt, 0.0)
        ex[t] = torch.where(on, (El + K * U * Sl) * wt, 0.0)
        mu = torch.where(on, a[:, t] * lam, mu)
        E = torch.where(on, a[:, t] * El + K * U * a[:, t] * Sl, E)
        S = torch.where(on, a[:, t] * Sl, S)
    stack = (lambda r: torch.stack(r, 1)) if T else (lambda r: g)
    return stack(dg), stack(dx), mu, stack(eg), stack(ex), E


def check(got, want, err, dtype, what=""):
    """|got - want| <= err + half a step of the type at the value, with a hundredth of slack for what is of second order."""
    assert got.dtype == dtype and got.shape == want.shape, what
    got = got.to(F64)
    assert torch.isfinite(got).all(), what
    tol = 1.01 * (err + HALF_STEP[dtype] * (want.abs() + err)) + tiny(dtype)
    over = (got - want).abs() - tol
    assert float(over.max() if over.numel() else -1.0) <= 0.0, f"{what}: {float((got - want).abs().max())} off, at the worst place allowed {float(tol.flatten()[over.argmax()])}"


def fields(B, T, C, dtype, seed, gate=(-1.0, 6.0), device="cuda"):
    """Gate (memories of one row to a few hundred, by column) and input."""
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)
    lo, hi = gate
    g = torch.randn(B, T, C, device=device, generator=gen) + lo + (hi - lo) * torch.rand(C, device=device, generator=gen)
    x = torch.randn(B, T, C, device=device, generator=gen)
    return g.to(dtype), x.to(dtype), gen
