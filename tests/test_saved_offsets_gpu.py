"""Tensors in 8 bits and activations at places that the accesses of 32 bytes do not fit, and past 2^31 elements."""
import pytest
import torch

from paper_2007_12792_b200 import autograd, checkpoints
from paper_2007_12792_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("n", [8, 40, 4096, 10007])
@pytest.mark.parametrize("off", [4, 8, 12])                            # 16, 32 and 48 bytes
def test_places_on_16_bytes(off, n, fmt):
    gen = torch.Generator(device="cuda"); gen.manual_seed(n)
    x, dy = torch.randn(n, device="cuda", generator=gen) * 3, torch.randn(n, device="cuda", generator=gen)
    def place(v=None):
        t = torch.full((n + 32,), 7.0, device="cuda")
        part = t[off:off + n]
        assert part.data_ptr() % 32 == 4 * off % 32
        return t, part if v is None else part.copy_(v)
    _, px = place(x)
    want = checkpoints.pack(x, fmt)
    got = checkpoints.pack(px, fmt)
    end = (n + 15) // 16 * 16                                          # (between the codes and the scales nothing is written)
    assert torch.equal(got.data[:n], want.data[:n]) and torch.equal(got.data[end:], want.data[end:])
    whole, part = place()
    B.dn_unpack(got.data, fmt, part)
    assert torch.equal(part, want.unpack())
    part.fill_(7.0)
    assert bool((whole == 7.0).all())
    for kind in ("silu", "gelu", "tanh"):
        packed = torch.empty(B.dn_packed_bytes(n), dtype=torch.uint8, device="cuda")
        y, d = torch.empty_like(x), torch.empty_like(x)
        B.dn_activation_forward(kind, x, y, fmt, packed)
        B.dn_activation_backward(kind, packed, fmt, dy, d)
        again = torch.empty_like(packed)
        (wy, py), (wd, pd) = place(), place()
        B.dn_activation_forward(kind, px, py, fmt, again)
        B.dn_activation_backward(kind, again, fmt, place(dy)[1], pd)
        assert torch.equal(py, y) and torch.equal(pd, d)
        for w, p in ((wy, py), (wd, pd)):
            p.fill_(7.0)
            assert bool((w == 7.0).all())


def test_past_32_bits():
    """2^31 + 12 345 values of 16 bits: the last ones are those of a small tensor."""
    n, k = (1 << 31) + 12345, 32 * 700 + 12345 % 32
    gen = torch.Generator(device="cuda"); gen.manual_seed(1)
    x = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    x[-k:] = torch.randn(k, device="cuda", generator=gen).to(torch.bfloat16)
    x[:4096] = torch.randn(4096, device="cuda", generator=gen).to(torch.bfloat16)
    tail, head = x[-k:].clone(), x[:4096].clone()
    p = checkpoints.pack(x, "int8")
    back = p.unpack()
    assert torch.equal(back[-k:], checkpoints.pack(tail, "int8").unpack()) and torch.equal(back[:4096], checkpoints.pack(head, "int8").unpack())
    assert float(back[4096:1 << 20].abs().sum()) == 0.0
    del back, p
    packed, y = torch.empty(B.dn_packed_bytes(n), dtype=torch.uint8, device="cuda"), torch.empty_like(x)
    B.dn_activation_forward("silu", x, y, "e4m3", packed)
    t8, ty = torch.empty(B.dn_packed_bytes(k), dtype=torch.uint8, device="cuda"), torch.empty_like(tail)
    B.dn_activation_forward("silu", tail, ty, "e4m3", t8)
    assert torch.equal(y[-k:], ty)
    y.fill_(1.0)
    B.dn_activation_backward("silu", packed, "e4m3", y, y)             # in place
    B.dn_activation_backward("silu", t8, "e4m3", torch.ones_like(ty), ty)
    assert torch.equal(y[-k:], ty) and bool((y[4096:1 << 20] == 0.5).all())
