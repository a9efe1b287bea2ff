"""Tensors in 8 bits and the activations that keep theirs so, against 64 bits; and a generator of them all under the losses."""
import pytest
import torch

import scan_util as S
from paper_2007_12792_b200 import autograd, checkpoints
from paper_2007_12792_b200 import binding as B

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
DTYPES = [F32, BF16, F16]
FORMATS = ["int8", "e4m3"]
SIZES = [1, 2, 7, 8, 31, 32, 33, 63, 64, 100, 1023, 8191, 8192, 8193, 70001]


def values(n, dtype, seed):
    gen = torch.Generator(device="cuda"); gen.manual_seed(seed)
    x = torch.randn(n, device="cuda", generator=gen) * torch.exp2(torch.randint(-9, 9, (n,), device="cuda", generator=gen).float())
    x[::97] = 0.0
    return x.to(dtype)


def rounded(v, dtype):
    """64-bit values rounded once to the type (they have at most 8 significant bits: 32 bits hold all but the smallest exactly)."""
    return v.to(F32).to(dtype)


def same(a, b):
    return torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(torch.nan_to_num(a, nan=0.0), torch.nan_to_num(b, nan=0.0))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", DTYPES)
def test_values_bit_for_bit(dtype, fmt):
    for n in SIZES:
        x = values(n, dtype, n)
        got = checkpoints.pack(x, fmt).unpack()
        assert got.dtype == dtype and torch.equal(got, rounded(S.eight(x, fmt), dtype)), n
        y = torch.zeros(n + 3, dtype=dtype, device="cuda")[3:].copy_(x)             # off the 16 bytes of a wide access
        assert y.data_ptr() % 16 and torch.equal(checkpoints.pack(y, fmt).unpack(), got)
        p = checkpoints.pack(x, fmt)
        wide = torch.full((n + 10,), 7.0, dtype=dtype, device="cuda")
        B.dn_unpack(p.data, fmt, wide[5:n + 5])
        assert torch.equal(wide[5:n + 5], got) and bool((wide[:5] == 7).all()) and bool((wide[n + 5:] == 7).all())
        room = torch.full((B.dn_packed_bytes(n) + 9,), 77, dtype=torch.uint8, device="cuda")
        B.dn_pack(x, fmt, room)
        end = (n + 15) // 16 * 16
        assert torch.equal(room[:n], p.data[:n]) and torch.equal(room[end:-9], p.data[end:]) and bool((room[-9:] == 77).all()) and bool((room[n:end] == 77).all())


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", DTYPES)
def test_the_ends_of_the_range(dtype, fmt):
    f = torch.finfo(dtype)
    tiniest = f.smallest_normal * f.eps
    for top in (f.max, f.max / 2, f.smallest_normal, f.smallest_normal * 3.99, tiniest, 127.5, 127.4, 128.0, 247.9, 255.9, 1.0, 0.0):
        x = torch.linspace(-1.0, 1.0, 64, device="cuda").mul_(top if top < 1e38 else 1.0)
        if top >= 1e38:
            x = x * 1.6e38 * 2
        x = x.to(dtype)
        x[5], x[40] = top, -top
        got = checkpoints.pack(x, fmt).unpack()
        assert torch.isfinite(got).all()
        assert same(got, rounded(S.eight(x, fmt), dtype)), top
    x = values(320, dtype, 1)
    clean = checkpoints.pack(x, fmt).unpack()
    x[3], x[40], x[41], x[319] = float("nan"), float("inf"), float("-inf"), float("nan")
    x[64:96] = float("inf")
    got = checkpoints.pack(x, fmt).unpack()
    bad = torch.tensor([3, 40, 41, 319] + list(range(64, 96)), device="cuda")
    assert torch.isnan(got[bad]).all() and same(got, rounded(S.eight(x, fmt), dtype))
    good = torch.ones(320, dtype=torch.bool, device="cuda"); good[bad] = False
    blocks = torch.arange(320, device="cuda") // 32
    untouched = good & (blocks != 0) & (blocks != 1) & (blocks != 9)
    assert torch.equal(got[untouched], clean[untouched])


@pytest.mark.parametrize("dtype", DTYPES)
def test_error_bounds(dtype):
    """int8: half a step, 2^-7 of the block's largest power of two, a step where 127 stands for up to 128; e4m3: 2^-4 of the value (240 for up to
    256 too), or half the least step, 2^-17 of that power of two.  Rounding to the type adds nothing: its grid is finer."""
    x = values(1 << 16, dtype, 9).to(S.F64)
    top = x.view(-1, 32).abs().amax(-1, keepdim=True)
    power = torch.exp2(torch.frexp(top)[1].to(S.F64) - 1)
    for fmt in FORMATS:
        got = checkpoints.pack(x.to(dtype), fmt).unpack().to(S.F64)
        err = (got - x).view(-1, 32).abs()
        if fmt == "int8":
            allowed = torch.where(x.view(-1, 32).abs() > power * 127.5 / 64, power / 64, power / 128)
        else:
            allowed = torch.maximum(x.view(-1, 32).abs() * 2.0 ** -4, power * 2.0 ** -17)
        assert bool((err <= allowed).all()), fmt


def test_shapes_and_strides():
    x = torch.randn(6, 5, 4, 3, device="cuda")
    for v in (x, x.permute(0, 2, 3, 1), x[:, ::2], x[:0], x[0, 0, 0, 0], x.expand(2, 6, 5, 4, 3), x.to(memory_format=torch.channels_last)):
        p = checkpoints.pack(v, "int8")
        got = p.unpack()
        assert got.shape == v.shape and got.is_contiguous()
        if v.numel():
            assert torch.equal(got.flatten(), S.eight(v.contiguous().flatten(), "int8").float())
    assert checkpoints.pack(torch.randn(1024, device="cuda").requires_grad_()).data.numel() == 1024 + 32


# y: the gate's roundings (see scan_util.roundings, without the sums of the scan), its argument (gelu: 6 products and sums, whose error
# moves the gate by |z| (1 - s) times that, at most 0.3), one product; tanh: the documented 2 ulp.  dx: the slope's sum of two terms
# of either sign, each off by as much relative to itself, and the product with dy.
def slope_error(kind, x, dtype):
    u = S.U
    k = (4 if dtype == F32 else 2 * (2 + 1.16 * 88)) + 8
    z = x if kind == "silu" else 2 * x if kind == "tanh" else 2 * (2 / torch.pi) ** 0.5 * (x + 0.044715 * x ** 3)
    dz = 1.0 if kind == "silu" else 2 * (2 / torch.pi) ** 0.5 * (1 + 3 * 0.044715 * x ** 2)
    p, q = torch.sigmoid(z), torch.sigmoid(-z)
    kk = k + 8 * z.abs()                       # an argument off by 8 u relative to itself moves p and q by 8 u |z| relative to themselves at most
    if kind == "tanh":
        return u * 4 * p * q * (2 * kk + 4)
    return u * (p * kk + p * q * x.abs() * dz * (2 * kk + 14))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("kind", ["silu", "gelu", "tanh"])
@pytest.mark.parametrize("dtype", DTYPES)
def test_activations(dtype, kind, fmt):
    for n in (1, 33, 4096, 10007):
        gen = torch.Generator(device="cuda"); gen.manual_seed(n)
        x = (torch.randn(n, device="cuda", generator=gen) * 3).to(dtype)
        x[::50] *= 8
        dy = torch.randn(n, device="cuda", generator=gen).to(dtype)
        x.requires_grad_()
        y = autograd.activation(x, kind, checkpoint=fmt)
        (dx,) = torch.autograd.grad(y, x, dy)
        xd = x.detach()
        x64 = xd.to(S.F64)
        want = S.act(kind, x64)[0]
        z = x64 if kind == "silu" else 2 * (2 / torch.pi) ** 0.5 * (x64 + 0.044715 * x64 ** 3)
        k = (4 if dtype == F32 else 2 * (2 + 1.16 * 88)) + 9 + 8 * z.abs()
        err = 4 * S.U * want.abs() if kind == "tanh" else S.U * k * want.abs()
        S.check(y.detach(), want, err + 2.0 ** -140, dtype, "y")
        kept = S.eight(x64, fmt)
        slope = S.act(kind, kept)[1]
        S.check(dx, dy.to(S.F64) * slope, dy.to(S.F64).abs() * slope_error(kind, kept, dtype) + 2.0 ** -140, dtype, "dx")
        packed = torch.empty(B.dn_packed_bytes(n), dtype=torch.uint8, device="cuda")
        y2, d2 = torch.empty_like(xd), dy.clone()
        B.dn_activation_forward(kind, xd, y2, fmt, packed)
        B.dn_activation_backward(kind, packed, fmt, d2, d2)                  # in place
        assert torch.equal(y2, y) and torch.equal(d2, dx)
        with torch.no_grad():
            assert torch.equal(autograd.activation(x, kind, checkpoint=fmt), y)


@pytest.mark.parametrize("dtype", DTYPES)
def test_activations_far_out(dtype):
    big = torch.finfo(dtype).max
    x = torch.tensor([0.0, -0.0, big, -big, big / 2, -big / 2, 20.0, -20.0, 1e-6, -1e-6], device="cuda").to(dtype).repeat_interleave(32)     # a block for each
    x.requires_grad_()
    for kind in ("silu", "gelu", "tanh"):
        y = autograd.activation(x, kind)
        (dx,) = torch.autograd.grad(y, x, torch.ones_like(y))
        xs = x.detach().to(S.F64).clamp(-1e4, 1e4)
        want = S.act(kind, xs)[0]
        far = x.detach().abs() > 100
        if kind != "tanh":
            assert torch.equal(y[far], torch.where(x > 0, x, 0.0)[far])
        assert float((y.detach().to(S.F64) - want)[~far].abs().max()) <= 20 * 2 * S.HALF_STEP[dtype]
        if kind == "tanh":
            assert torch.equal(dx[far], torch.zeros_like(dx[far])) and torch.equal(y[far], torch.sign(x)[far])
        else:
            assert torch.equal(dx[far], (x > 0).to(dtype)[far])
    for bad in (float("nan"), float("inf")):
        x = torch.full((40,), 1.0, dtype=dtype, device="cuda"); x[3] = bad
        x.requires_grad_()
        (dx,) = torch.autograd.grad(autograd.activation(x, "gelu"), x, torch.ones_like(x))
        assert torch.isnan(dx[3]) and torch.isfinite(dx[4:]).all()


def test_activation_as_a_torch_op():
    x = torch.randn(3, 4, 5, device="cuda").transpose(0, 2).requires_grad_()
    y = autograd.activation(x, "tanh", checkpoint="e4m3")
    assert y.shape == x.shape
    (dx,) = torch.autograd.grad(y.sum(), x, retain_graph=True)
    assert dx.shape == x.shape
    with pytest.raises(RuntimeError, match="create_graph"):
        torch.autograd.grad(y.sum(), x, create_graph=True)
    e = torch.empty(0, 3, device="cuda", requires_grad=True)
    assert torch.autograd.grad(autograd.activation(e).sum(), e)[0].shape == (0, 3)
    for bad in (torch.zeros(3, device="cuda", dtype=torch.float64), torch.zeros(3, device="cuda", dtype=torch.int32)):
        with pytest.raises(ValueError):
            autograd.activation(bad)


def burgers_problem(Bn, nt, nx):
    return B.Burgers(nx=nx, nt=nt, batch=Bn, c=torch.linspace(3.0, 6.0, Bn, device="cuda"))


def test_the_losses_keep_their_gradient_in_8_bits():
    """A loss saves its gradient; with the context its backward pass multiplies what 8 bits hold of it."""
    Bn, nt, nx = 3, 65, 130
    p = burgers_problem(Bn, nt, nx)
    u = torch.rand(Bn, nt, nx, device="cuda").requires_grad_()
    up = torch.tensor([1.0, -2.0, 0.5], device="cuda")
    (exact,) = torch.autograd.grad(autograd.burgers_loss(u, p), u, up)
    (plain,) = torch.autograd.grad(autograd.burgers_loss(u, p), u, torch.ones(Bn, device="cuda"))
    for fmt in FORMATS:
        with checkpoints.saved_in_8_bits(fmt):
            L = autograd.burgers_loss(u, p)
        (got,) = torch.autograd.grad(L, u, up)
        assert torch.equal(got, up[:, None, None] * S.eight(plain.flatten(), fmt).float().view_as(plain))
    with checkpoints.saved_in_8_bits(min_numel=1 << 30):
        L = autograd.burgers_loss(u, p)
    assert torch.equal(torch.autograd.grad(L, u, up)[0], exact)
    q = B.Problem(dim=2, nx=66, ny=65, batch=2, kl_modes=2, kl_w=torch.randn(2, 2, 2, device="cuda"))
    v = torch.rand(2, 65, 66, device="cuda").requires_grad_()
    (plain,) = torch.autograd.grad(autograd.energy(v, q).sum(), v)
    with checkpoints.saved_in_8_bits():
        J = autograd.energy(v, q).sum()
    assert torch.equal(torch.autograd.grad(J, v)[0], S.eight(plain.flatten(), "int8").float().view_as(plain))


def test_saved_tensors_of_other_ops():
    w = torch.randn(64, 64, device="cuda", requires_grad=True)
    x = torch.randn(100, 64, device="cuda", requires_grad=True)
    dy = torch.randn(100, 64, device="cuda")
    with checkpoints.saved_in_8_bits(keep=[w]):
        y = x @ w.t()
    gx, gw = torch.autograd.grad(y, (x, w), dy)
    kept = S.eight(x.detach().flatten(), "int8").float().view_as(x)
    assert torch.equal(gx, dy @ w.detach())                       # the weight as it is, through a view of it
    assert torch.equal(gw, torch.autograd.grad(kept @ w.t(), w, dy)[0])
    # the recurrence's own checkpoint is left alone, gate and input go through the context
    g, xx, _ = S.fields(2, 130, 64, F32, 5)
    g.requires_grad_(); xx.requires_grad_()
    d = torch.randn(2, 130, 64, device="cuda")
    with checkpoints.saved_in_8_bits():
        h, _ = autograd.gated_scan(g, xx, mix=True)
        h8, _ = autograd.gated_scan(g, xx, mix=True, checkpoint="int8")
    # rows of 64 columns: the blocks of both are the same 32 values, and both give the formulas' results at these
    wg, wx, _, eg, ex, _ = S.backward(g.detach(), xx.detach(), None, None, True, d, None, "int8")
    for out in (h, h8):
        dg, dx = torch.autograd.grad(out, (g, xx), d)
        S.check(dg, wg, eg, F32, "dg")
        S.check(dx, wx, ex, F32, "dx")


@pytest.mark.parametrize("saved", [None, "int8"])
def test_a_generator_of_them_under_the_losses(saved):
    """Projection, recurrence over the time rows, activation, projection to a field, Burgers loss: value and gradients of the whole against
    64 bits, with everything that is saved kept as it is, and (the paths of the 8 bits) in 8 bits against the same chain by hand."""
    Bn, nt, nx, k = 2, 70, 66, 32
    gen = torch.Generator(device="cuda"); gen.manual_seed(1)
    r = lambda *s: torch.randn(*s, device="cuda", generator=gen)
    z, w_in, w_out, h0 = r(Bn, nt, 16), (r(16, 2 * k) * 0.5).requires_grad_(), (r(k, nx) * 0.2).requires_grad_(), (r(Bn, k) * 0.3).requires_grad_()
    p = burgers_problem(Bn, nt, nx)
    both = z @ w_in
    h, _ = autograd.gated_scan(both[..., :k], both[..., k:], h0, mix=True, checkpoint=saved)
    y = autograd.activation(h, "silu") if saved else torch.nn.functional.silu(h)
    u = y @ w_out
    L = autograd.burgers_loss(u, p).mean()
    L.backward()
    # by hand
    with torch.no_grad():
        ub = u.detach().clone().requires_grad_()
    (du,) = torch.autograd.grad(autograd.burgers_loss(ub, p).mean(), ub)
    dy = (du @ w_out.t()).detach()
    hd, bd = h.detach(), both.detach()
    slope = S.act("silu", S.eight(hd.flatten(), "int8").view_as(hd) if saved else hd.to(S.F64))[1]
    dh = (dy.to(S.F64) * slope).float()
    wg, wx, w0, eg, ex, e0 = S.backward(bd[..., :k], bd[..., k:], h0.detach(), None, True, dh, None, saved)
    # dh itself is rounded here and there (half a step each, and the slope's 40 u): the gradients are linear in it with factors below 1
    # summed over at most nt rows
    scale = float(dh.abs().max()) * 64 * S.U * nt * 4
    assert float((h0.grad.to(S.F64) - w0).abs().max()) <= float(e0.max()) + scale
    want_in = torch.cat([wg, wx], -1).to(S.F64)
    d_in = z.to(S.F64).reshape(-1, 16).t() @ want_in.reshape(-1, 2 * k)
    # sums over Bn nt rows of products that are each off by the gradients' error, and by the sum's own roundings (torch's float32 product)
    mags = z.to(S.F64).abs().reshape(-1, 16).t() @ (want_in.abs() * Bn * nt * S.U + torch.cat([eg, ex], -1) + scale * (1 + bd.to(S.F64).abs().max())).reshape(-1, 2 * k)
    assert bool(((w_in.grad.to(S.F64) - d_in).abs() <= mags).all())
    assert torch.isfinite(w_out.grad).all()
