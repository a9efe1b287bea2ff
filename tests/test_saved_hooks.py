"""What saved_in_8_bits does with the tensors that it leaves as they are (on the CPU, where these are all tensors)."""
import gc
import weakref

import pytest
import torch

import scan_util as S
from paper_2007_12792_b200 import autograd, checkpoints


def test_saved_outputs_are_let_go():
    """exp saves its result: with a hook that hands it back, result and op would hold one another and never be freed."""
    x = torch.randn(100, dtype=torch.float64, requires_grad=True)
    with checkpoints.saved_in_8_bits():
        y = torch.exp(x)
        z = (torch.tanh(y) * y).sum()
    gone = [weakref.ref(y), weakref.ref(z)]
    del y, z
    gc.collect()
    assert [r() for r in gone] == [None, None]


def test_gradients_of_what_is_kept():
    """First and second derivatives are those without the context."""
    x = torch.linspace(-1.0, 1.0, 50, dtype=torch.float64).requires_grad_()
    w = torch.randn(50, dtype=torch.float64, generator=torch.Generator().manual_seed(1)).requires_grad_()
    out = []
    for context in (checkpoints.saved_in_8_bits(keep=[w]), torch.enable_grad()):
        with context:
            y = (torch.exp(w * x) * torch.sigmoid(x)).sum()
            g = torch.autograd.grad(y, (x, w), create_graph=True)
            out.append([*g, *torch.autograd.grad((g[0] ** 2).sum() + g[1].sum(), (x, w))])
    for a, b in zip(*out):
        assert torch.equal(a, b)


def test_what_is_kept_must_not_change():
    """A weight updated between forward and backward pass, or any kept tensor written into: an error, as without the context."""
    for change in (lambda w, v: w.add_(1.0), lambda w, v: v.zero_()):
        w, x = torch.randn(5000, requires_grad=True), torch.randn(5000, requires_grad=True)
        v = torch.randn(5000)
        with checkpoints.saved_in_8_bits(keep=[w]):
            y = (w * x * v).sum()
        with torch.no_grad():
            change(w, v)
        with pytest.raises(RuntimeError, match="modified in place"):
            torch.autograd.grad(y, (w, x))


@pytest.mark.gpu
def test_what_is_kept_on_the_device_must_not_change():
    w, x = torch.randn(5000, device="cuda", requires_grad=True), torch.randn(5000, device="cuda", requires_grad=True)
    for keep in ([w], ()):
        with checkpoints.saved_in_8_bits(keep=keep):
            y = (w.view(50, 100) * x.view(50, 100)).sum()
        want = checkpoints.pack(w.detach()).unpack()
        with torch.no_grad():
            w.add_(1.0)
        if keep:
            with pytest.raises(RuntimeError, match="modified in place"):
                torch.autograd.grad(y, x)
        else:                                            # 8 bits hold a copy
            assert torch.equal(torch.autograd.grad(y, x)[0], want)


@pytest.mark.gpu
def test_expanded_views_take_no_more_memory():
    """A row that all rows share is 4 kB; a byte for each element of the view would be 8 MB."""
    row, x = torch.randn(1024, device="cuda"), torch.randn(8192, 1024, device="cuda", requires_grad=True)
    torch.cuda.synchronize()
    start = torch.cuda.memory_allocated()
    with checkpoints.saved_in_8_bits():
        y = x * row.expand(8192, 1024)
    del y
    with checkpoints.saved_in_8_bits():
        y = x * row.expand(8192, 1024)
        assert torch.cuda.memory_allocated() - start <= 4 * x.numel() + (1 << 20)           # the result alone (x wants a gradient, the row none)
    d = torch.randn_like(x)
    assert torch.equal(torch.autograd.grad(y, x, d)[0], d * row)
    # a view that is expanded a little is smaller in 8 bits
    half = torch.randn(8192, 512, device="cuda")
    with checkpoints.saved_in_8_bits():
        z = x.view(8192, 2, 512) * half[:, None].expand(8192, 2, 512)
    packed = checkpoints.pack(half[:, None].expand(8192, 2, 512)).unpack().view(8192, 1024)
    assert torch.equal(torch.autograd.grad(z.view(8192, 1024), x, d)[0], d * packed)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_gate_is_kept_as_int8(dtype):
    """gated_scan inside the context (rows of 64 columns: the blocks of 32 are those of its own checkpoint): the gradients at the gate in
    int8 and the input in the context's format, also where a gate of 12 would be off by half a unit in e4m3."""
    g, x, gen = S.fields(2, 130, 64, dtype, 5, gate=(-1.0, 12.0))
    leaves = [g.requires_grad_(), x.requires_grad_()]
    d = torch.randn(2, 130, 64, device="cuda", generator=gen).to(dtype)
    for fmt in ("e4m3", "int8"):
        with checkpoints.saved_in_8_bits(fmt):
            h, _ = autograd.gated_scan(*leaves, mix=True)
            y = torch.exp(x)                             # what is saved next is no gate
        dg, dx = torch.autograd.grad(h, leaves, d)
        wg, wx, _, eg, ex, _ = S.backward(g.detach(), x.detach(), None, None, True, d, None, fmt)
        S.check(dg, wg, eg, dtype, "dg")
        S.check(dx, wx, ex, dtype, "dx")
        assert torch.equal(torch.autograd.grad(y, x, d)[0], d * checkpoints.pack(y.detach(), fmt).unpack())
    h, _ = autograd.gated_scan(*leaves)                  # outside: nothing is left over for the context after it
    with checkpoints.saved_in_8_bits("e4m3"):
        y = torch.exp(x)
    assert torch.equal(torch.autograd.grad(y, x, d)[0], d * checkpoints.pack(y.detach(), "e4m3").unpack())
