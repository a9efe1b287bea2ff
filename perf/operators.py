"""Cases of the operators that a generator uses next to the losses: the gated linear recurrence over the rows of a field and
checkpoints in 8 bits.

A case is one pass of
  scan      the recurrence h_t = a_t h_{t-1} + w_t x_t, a = sigmoid(g), w = 1 or 1 - a: a generator run forward (one row: a step of it)
  train     the recurrence as a PyTorch op: forward, and its gradients back to gate, input and initial state
  train8    the same with the saved inputs in 8 bits
  pack      a saved tensor put into 8 bits and read back
  act8      a pointwise activation as a PyTorch op, forward and backward, whose saved input is in 8 bits
Fields are [B][T][C]: T rows (time), C columns (nodes in space, or channels).
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
CHUNK = 64                    # rows between two states that a checkpoint of the recurrence keeps in 32 bits
BLOCK = 32                    # values that share a scale
MOST_SCAN = 1 << 27           # elements of the largest listed cases: 65536 x 2048 forward, 8 x 4096 x 2048 as a training step
MOST_TRAIN = 1 << 26


def _seq(op, B, T, C, dtype, name=None, **kw):
    c = {"op": op, "B": B, "T": T, "C": C, "dtype": dtype, "mix": True, "h0": True, "ragged": False, "fused": False, "format": "int8"}
    c.update(kw)
    if name:
        c["name"] = name
    return c


def _flat(op, n, dtype, name=None, **kw):
    c = {"op": op, "n": n, "dtype": dtype, "format": "int8", "kind": "silu"}
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one row for each of 64 samples: the step of a generator that is run forward in time, where latency is what counts
        _seq("scan", 64, 1, 1024, "bf16", "scan_step_64x1024_bf16"),
        # one very long sequence with few columns
        _seq("scan", 1, 65536, 2048, "bf16", "scan_long_65536x2048_bf16", fused=True),
        # the fields of the Burgers loss at high resolution, 1024^2 x 64
        _seq("scan", 64, 1024, 1024, "f32", "scan_field_1024_b64_f32", mix=False, h0=False),
        # samples of unlike length (none and one row among them), odd sizes
        _seq("scan", 7, 1531, 777, "f16", "scan_ragged_7x1531x777_f16", ragged=True),
        # the ordinary training step; gate and input are the halves of one projection
        _seq("train", 8, 2048, 2048, "bf16", "train_8x2048x2048_bf16", fused=True),
        # odd, ragged fields in 32 bits
        _seq("train", 16, 509, 383, "f32", "train_ragged_16x509x383_f32", ragged=True, mix=False),
        # the smallest training grid, 64^2 x 8: launches and host time
        _seq("train", 8, 64, 64, "f32", "train_64_b8_f32"),
        # the largest training step, its inputs kept in 8 bits
        _seq("train8", 8, 4096, 2048, "bf16", "train8_8x4096x2048_bf16"),
        # rows that are no multiple of a block, rows that end inside a chunk
        _seq("train8", 4, 257, 100, "f32", "train8_4x257x100_f32", format="e4m3", mix=False, h0=False),
        # the gradient that a loss over 1024^2 x 64 fields saves for its backward pass
        _flat("pack", 1 << 26, "f32", "pack_1024_b64_f32"),
        # a small saved tensor of odd size
        _flat("pack", 131 * 129, "bf16", "pack_16899_bf16", format="e4m3"),
        # an activation of a 2D generator: 64 channels, 256^2, 8 samples
        _flat("act8", 64 * 256 * 256 * 8, "bf16", "act8_silu_64x256_b8_bf16"),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["scan", "scan", "train", "train8", "pack", "act8"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    fmt = rng.choice(["int8", "e4m3"])
    if op in ("pack", "act8"):
        return _flat(op, _spread(rng, 1, 1 << 26 if op == "pack" else 1 << 25), dtype, format=fmt, kind=rng.choice(["silu", "gelu", "tanh"]))
    most = MOST_SCAN if op == "scan" else MOST_TRAIN
    if dtype == "f32":
        most //= 2
    while True:
        B, T, C = _spread(rng, 1, 64), _spread(rng, 1, 65536 if op == "scan" else 16384), _spread(rng, 1, 4096)
        if B * T * C <= most:
            break
    return _seq(op, B, T, C, dtype, mix=rng.random() < 0.5, h0=rng.random() < 0.7, ragged=rng.random() < 0.4, fused=rng.random() < 0.4, format=fmt)


def _inputs(case, seed):
    dev = "cuda" if torch.cuda.is_available() else "cpu"
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(*shape, device=dev, dtype=torch.float32, generator=gen)

    if "n" in case:
        n = case["n"]
        x = normal(n)
        x = x * torch.where(torch.rand(n, device=dev, generator=gen) < 0.002, 20.0, 1.5)      # a few outliers, as activations have them
        s = {"x": x.to(dt)}
        if case["op"] == "act8":
            s["dy"] = normal(n).to(dt)
        return s
    B, T, C = case["B"], case["T"], case["C"]
    both = torch.empty(B, T, 2, C, device=dev, dtype=dt)
    for b in range(B):                                        # memories of one row to a few hundred, by column
        both[b, :, 0] = normal(T, C) + torch.rand(C, device=dev, generator=gen) * 7.0 - 1.0
        both[b, :, 1] = normal(T, C)
    s = {}
    if case["fused"]:
        s["g"], s["x"] = both[:, :, 0], both[:, :, 1]
    else:
        s["g"], s["x"] = both[:, :, 0].contiguous(), both[:, :, 1].contiguous()
    s["h0"] = normal(B, C) if case["h0"] else None
    s["lengths"] = None
    if case["ragged"]:
        n = (torch.rand(B, device=dev, generator=gen) * (T + 1)).to(torch.int32).clamp_(0, T)
        n[0] = T
        if B > 2:
            n[1], n[2] = 0, 1
        s["lengths"] = n
    if case["op"] != "scan":
        s["dh"] = torch.empty(B, T, C, device=dev, dtype=dt)
        for b in range(B):
            s["dh"][b] = normal(T, C)
        s["dhT"] = normal(B, C)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        from paper_2007_12792_b200 import autograd, binding, checkpoints
        s["autograd"], s["B"], s["checkpoints"] = autograd, binding, checkpoints
        if case["op"] == "scan":
            s["problem"] = binding.Scan(batch=case["B"], rows=case["T"], cols=case["C"], dtype=DTYPES[case["dtype"]], mix=case["mix"],
                                        lengths=s["lengths"])
    if case["op"] != "scan" and case["op"] != "pack":
        for k in ("g", "x", "h0"):
            if s.get(k) is not None:
                s[k] = s[k].detach().requires_grad_()
    return s


# ---- the framework's calls ------------------------------------------------------------------------------------------------------
def _run_own(s):
    case = s["case"]
    op = case["op"]
    if op == "scan":
        h = torch.empty(case["B"], case["T"], case["C"], dtype=DTYPES[case["dtype"]], device="cuda")
        h_last = torch.empty(case["B"], case["C"], dtype=torch.float32, device="cuda")
        s["B"].dn_scan_forward(s["problem"], s["g"], s["x"], s["h0"], h, h_last)
        return {"h": h, "h_last": h_last}
    if op in ("train", "train8"):
        leaves = [s["g"], s["x"]] + ([s["h0"]] if case["h0"] else [])
        h, h_last = s["autograd"].gated_scan(s["g"], s["x"], s["h0"], lengths=s["lengths"], mix=case["mix"],
                                             checkpoint=case["format"] if op == "train8" else None)
        grads = torch.autograd.grad((h, h_last), leaves, (s["dh"], s["dhT"]))
        return dict(zip(["h", "h_last", "dg", "dx", "dh0"], [h.detach(), h_last.detach(), *grads]))
    if op == "pack":
        return {"x": s["checkpoints"].pack(s["x"], case["format"]).unpack()}
    y = s["autograd"].activation(s["x"], case["kind"], checkpoint=case["format"])
    return {"y": y.detach(), "dx": torch.autograd.grad(y, s["x"], s["dy"])[0]}


# ---- the plain forms ------------------------------------------------------------------------------------------------------------
def _doubling(a, b, start):
    """h_t = a_t h_{t-1} + b_t along dim 1 by doubling spans, in 32 bits."""
    h, A = b.clone(), a.clone()
    if start is not None:
        h[:, 0] += a[:, 0] * start
    d = 1
    while d < h.shape[1]:
        h[:, d:] += A[:, d:] * h[:, :-d]
        A[:, d:] = A[:, d:] * A[:, :-d]
        d *= 2
    return h


def _rounded8(x, fmt):
    """The values that stand for x in 8 bits: blocks of 32 along the last dim, each with a power of two as its scale."""
    shape, n = x.shape, x.shape[-1]
    v = x.to(torch.float32)
    pad = -n % BLOCK
    if pad:
        v = torch.cat([v, v.new_zeros(*shape[:-1], pad)], -1)
    v = v.reshape(*shape[:-1], -1, BLOCK)
    finite = torch.isfinite(v)
    amax = torch.where(finite, v.abs(), 0.0).amax(-1, keepdim=True)
    k = (amax.view(torch.int32) >> 23) - 127                 # amax lies in [2^k, 2^(k+1))
    e = (k - (6 if fmt == "int8" else 7)).clamp(min=-126)
    scale, inverse = ((e + 127) << 23).view(torch.float32), ((127 - e) << 23).view(torch.float32)
    q = torch.where(finite, v * inverse, 0.0)
    if fmt == "int8":
        q = q.round().clamp(-127.0, 127.0)
    else:
        q = q.to(torch.float8_e4m3fn).to(torch.float32).clamp(-240.0, 240.0)
    v = torch.where(finite, q * scale, float("nan"))
    return v.reshape(*shape[:-1], -1)[..., :n]


def _gate(g):
    g = g.to(torch.float32)
    return torch.sigmoid(g), torch.sigmoid(-g)


def _plain_forward(case, s):
    B, T, C = case["B"], case["T"], case["C"]
    a, w = _gate(s["g"])
    x = s["x"].to(torch.float32)
    b = w * x if case["mix"] else x
    live = None
    if s["lengths"] is not None:
        live = (torch.arange(T, device=x.device)[None, :] < s["lengths"][:, None])[:, :, None]
        a, b = torch.where(live, a, 1.0), torch.where(live, b, 0.0)
    h = _doubling(a, b, s["h0"])
    return h, h[:, -1], live


def _plain_backward(case, s, h, live):
    B, T, C = case["B"], case["T"], case["C"]
    g, x = s["g"].to(torch.float32), s["x"].to(torch.float32)
    zero = torch.zeros(B, 1, C, device=h.device) if s["h0"] is None else s["h0"][:, None]
    if case["op"] == "train8":
        g, x = _rounded8(g, "int8"), _rounded8(x, case["format"])
        a, w = _gate(g)
        pad = -T % CHUNK
        n = (T + pad) // CHUNK
        start = torch.cat([zero, h[:, CHUNK - 1:T - 1:CHUNK]], 1).reshape(B * n, C)
        b = w * x if case["mix"] else x
        b, aa = (torch.cat([v, v.new_zeros(B, pad, C)], 1) for v in (b, a))
        inner = _doubling(aa.reshape(B * n, CHUNK, C), b.reshape(B * n, CHUNK, C), start)
        before = torch.cat([start[:, None], inner[:, :-1]], 1).reshape(B, T + pad, C)[:, :T]
    else:
        a, w = _gate(g)
        before = torch.cat([zero, h[:, :-1]], 1)
    d = s["dh"].to(torch.float32)
    if live is not None:
        d, a_live = torch.where(live, d, 0.0), torch.where(live, a, 1.0)
    else:
        a_live = a
    # l_t = d_t + a_{t+1} l_{t+1}; the last state's gradient enters behind the last row (rows without data pass it on)
    last = torch.cat([a_live[:, 1:], torch.ones_like(a[:, :1])], 1)
    lam = _doubling(last.flip(1), d.flip(1), s["dhT"]).flip(1)
    dx = w * lam if case["mix"] else lam
    dg = lam * (before - x if case["mix"] else before) * a * w
    if live is not None:
        dx, dg = torch.where(live, dx, 0.0), torch.where(live, dg, 0.0)
    return dg, dx, a_live[:, 0] * lam[:, 0]


def _act(kind, x):
    """Value and derivative of an activation."""
    if kind == "tanh":
        y = torch.tanh(x)
        return y, 4.0 * torch.sigmoid(2.0 * x) * torch.sigmoid(-2.0 * x)
    z, dz = (x, 1.0) if kind == "silu" else (1.5957691216057308 * (x + 0.044715 * x * x * x), 1.5957691216057308 * (1.0 + 3 * 0.044715 * x * x))
    p, q = torch.sigmoid(z), torch.sigmoid(-z)
    return x * p, p * (1.0 + x * q * dz)


def _run_plain(s):
    case = s["case"]
    dt = DTYPES[case["dtype"]]
    with torch.no_grad():
        if case["op"] == "pack":
            return {"x": _rounded8(s["x"], case["format"]).to(dt)}
        if case["op"] == "act8":
            y = _act(case["kind"], s["x"].to(torch.float32))[0]
            d = _act(case["kind"], _rounded8(s["x"], case["format"]))[1]
            return {"y": y.to(dt), "dx": (s["dy"].to(torch.float32) * d).to(dt)}
        h, h_last, live = _plain_forward(case, s)
        out = {"h": (h if live is None else torch.where(live, h, 0.0)).to(dt), "h_last": h_last.clone()}
        if case["op"] != "scan":
            dg, dx, dh0 = _plain_backward(case, s, h, live)
            out["dg"], out["dx"] = dg.to(dt), dx.to(dt)
            if case["h0"]:
                out["dh0"] = dh0
        return out


def run(state):
    return _run_own(state) if own else _run_plain(state)


def work(case):
    """Inputs read once and outputs written once by each call of the pass (forward and backward are two calls)."""
    t = 4 if case["dtype"] == "f32" else 2
    saved = 1 + 1 / BLOCK
    if "n" in case:
        n = case["n"]
        if case["op"] == "pack":
            return {"bytes": n * (2 * t + 2 * saved), "flops": 4 * n}
        return {"bytes": n * (4 * t + 2 * saved), "flops": 25 * n}
    n, edge = case["B"] * case["T"] * case["C"], 4 * case["B"] * case["C"]
    rows = n * 4 / CHUNK
    if case["op"] == "scan":
        return {"bytes": 3 * t * n + 2 * edge, "flops": 10 * n}
    if case["op"] == "train":
        return {"bytes": 8 * t * n + 2 * rows + 4 * edge, "flops": 35 * n}
    return {"bytes": (6 * t + 4 * saved) * n + 2 * rows + 4 * edge, "flops": 45 * n}


# ---- the definition in 64 bits --------------------------------------------------------------------------------------------------
def _stands_for(v, fmt):
    """The 8-bit values of v (64 bits), block by block of 32 along the last dim."""
    out = torch.empty_like(v)
    for lo in range(0, v.shape[-1], BLOCK):
        if v.shape[-1] > 4096 and v.shape[-1] - lo >= BLOCK and lo == 0:        # long rows: all whole blocks at once
            whole = v.shape[-1] // BLOCK * BLOCK
            out[..., :whole] = _stands_for(v[..., :whole].reshape(-1, BLOCK), fmt).reshape(*v.shape[:-1], whole)
            if whole < v.shape[-1]:
                out[..., whole:] = _stands_for(v[..., whole:], fmt)
            return out
        p = v[..., lo:lo + BLOCK]
        top = p.abs().amax(-1, keepdim=True)
        k = torch.frexp(top)[1].to(torch.float64) - 1
        if fmt == "int8":
            step = torch.exp2((k - 6).clamp(min=-126))
            out[..., lo:lo + BLOCK] = torch.round(p / step).clamp(-127, 127) * step
        else:
            scale = torch.exp2((k - 7).clamp(min=-126))
            m = p / scale
            step = torch.exp2((torch.frexp(m.abs())[1].to(torch.float64) - 1).clamp(min=-6) - 3)
            out[..., lo:lo + BLOCK] = (torch.round(m / step) * step).clamp(-240, 240) * scale
    return out


def _exact_act(kind, x):
    if kind == "tanh":
        return torch.tanh(x), 1.0 / torch.cosh(x) ** 2
    if kind == "silu":
        s = 1.0 / (1.0 + torch.exp(-x))
        return x * s, s + x * s * (1.0 / (1.0 + torch.exp(x)))
    c = math.sqrt(2.0 / math.pi)
    z = c * (x + 0.044715 * x ** 3)
    p = 1.0 / (1.0 + torch.exp(-2.0 * z))
    return x * p, p + 0.5 * x / torch.cosh(z) ** 2 * c * (1.0 + 3 * 0.044715 * x ** 2)


def exact(case, seed):
    s = _inputs(case, seed)
    f64 = torch.float64
    if case["op"] == "pack":
        return {"x": _stands_for(s["x"].to(f64), case["format"])}
    if case["op"] == "act8":
        x = s["x"].to(f64)
        return {"y": _exact_act(case["kind"], x)[0], "dx": s["dy"].to(f64) * _exact_act(case["kind"], _stands_for(x, case["format"]))[1]}
    B, T, C = case["B"], case["T"], case["C"]
    dev = s["g"].device
    n = torch.full((B,), T, device=dev) if s["lengths"] is None else s["lengths"].to(torch.int64)
    state = torch.zeros(B, C, dtype=f64, device=dev) if s["h0"] is None else s["h0"].to(f64)
    h = torch.zeros(B, T, C, dtype=f64, device=dev)
    before = torch.empty(B, T, C, dtype=f64, device=dev) if case["op"] != "scan" else None      # the state ahead of each row
    g8 = x8 = inner = None
    if case["op"] == "train8":
        g8, x8 = (torch.cat([_stands_for(s[k][b].to(f64), f)[None] for b in range(B)]) for k, f in (("g", "int8"), ("x", case["format"])))

    def row(state, g, x):
        a = torch.sigmoid(g)
        return a * state + (torch.sigmoid(-g) * x if case["mix"] else x)

    for t in range(T):
        on = (n > t)[:, None]
        if before is not None:
            if g8 is None:
                before[:, t] = state
            else:
                if t % CHUNK == 0:
                    inner = state
                before[:, t] = inner
                inner = row(inner, g8[:, t], x8[:, t])
        state = torch.where(on, row(state, s["g"][:, t].to(f64), s["x"][:, t].to(f64)), state)
        h[:, t] = torch.where(on, state, 0.0)
    out = {"h": h, "h_last": state}
    if before is None:
        return out
    dg, dx = torch.zeros_like(h), torch.zeros_like(h)
    mu = s["dhT"].to(f64)
    for t in range(T - 1, -1, -1):
        on = (n > t)[:, None]
        g, x = (s["g"][:, t].to(f64), s["x"][:, t].to(f64)) if g8 is None else (g8[:, t], x8[:, t])
        a, w = torch.sigmoid(g), torch.sigmoid(-g)
        lam = s["dh"][:, t].to(f64) + mu
        dx[:, t] = torch.where(on, lam * w if case["mix"] else lam, 0.0)
        dg[:, t] = torch.where(on, lam * a * w * (before[:, t] - x if case["mix"] else before[:, t]), 0.0)
        mu = torch.where(on, a * lam, mu)
    out["dg"], out["dx"] = dg, dx
    if case["h0"]:
        out["dh0"] = mu
    return out
