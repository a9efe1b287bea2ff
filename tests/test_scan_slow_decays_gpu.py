"""Slow decays over many rows: what a constant error of the decay adds up to.

a is a 32-bit number near 1, and 1 - a of it has few digits.  16-bit types: 1 + e is rounded (u = 2^-24 at most, e = exp(-g)) and its
reciprocal is off by an ulp (the documented bound, u below 1): 2 u; 32-bit: one minus the smaller part, u / 2.  Each row adds a product and a
sum, u together with the grouping of rows another u.  A term that n rows have passed on is off by 4 n u of itself, and once by what its weight
1 - a is off by: (2 + 1.16 g) ulp of the approximate exponential, then a few roundings."""
import pytest
import torch

import scan_util as S
from paper_2007_12792_b200 import autograd

F64 = torch.float64


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T", [20000, 65536])
def test_constant_slow_gates(T, dtype):
    gates = torch.tensor([6.0, 9.0, 10.0, 10.5, 11.0, 12.0, 12.5, 13.0, 14.0, 16.0, 17.0, 20.0, 25.0, 40.0] + [8.0 + k / 16 for k in range(50)], device="cuda")
    C = len(gates)
    gen = torch.Generator(device="cuda"); gen.manual_seed(2)
    g = gates.to(dtype).expand(1, T, C).contiguous().requires_grad_()
    x = (1.0 + 0.1 * torch.randn(1, T, C, device="cuda", generator=gen)).to(dtype).requires_grad_()
    h0, dl = torch.ones(1, C, device="cuda", requires_grad=True), torch.ones(1, C, device="cuda")
    _, last = autograd.gated_scan(g, x, h0, mix=True)
    dh0, dx = torch.autograd.grad(last, (h0, x), dl)
    z = gates.to(dtype).to(F64)
    n = torch.arange(T - 1, -1, -1, device="cuda", dtype=F64)[:, None]           # rows behind
    log_a = -torch.log1p(torch.exp(-z))
    part, w = torch.exp(n * log_a), torch.sigmoid(-z)
    once = (2 * (2 + 1.16 * z) + 12) * S.U
    terms = part * w * x.detach()[0].to(F64)
    far = torch.exp(T * log_a)
    S.check(last.detach()[0], terms.sum(0) + far, (terms.abs() * (4 * n * S.U + once)).sum(0) + far * (4 * T * S.U), torch.float32, "h_last")
    S.check(dh0[0], far, far * 4 * T * S.U, torch.float32, "dh0")
    S.check(dx[0], part * w, part * w * (4 * n * S.U + once), dtype, "dx")
