"""Gates far beyond where the sigmoid is 0 or 1, infinite ones and masks among them, in checkpoints of 8 bits: held to +-63.5 they have
codes, and their neighbours keep steps of 1/2 or less."""
import pytest
import torch

import scan_util as S
from paper_2007_12792_b200 import autograd, checkpoints

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
INF = float("inf")


def far_gates(g, ends):
    big = torch.finfo(g.dtype).max
    for k, v in enumerate([100.0, -1e4, 63.5, -63.75, 64.0, -big, big, 87.5] + ([INF, -INF] if ends else [])):
        g[:, k::37, (5 * k) % g.shape[2]::41] = v
    return g


def compare(g, x, h0, dh, dl, fmt, lengths=None):
    leaves = [t.clone().requires_grad_() for t in (g, x, h0)]
    h, last = autograd.gated_scan(*leaves, lengths=lengths, mix=True, checkpoint=fmt)
    wh, wl, _, eh, el, _ = S.forward(g, x, h0, lengths, True)                    # the states do not go through 8 bits
    S.check(h.detach(), wh, eh, g.dtype, "h")
    S.check(last.detach(), wl, el, F32, "h_last")
    got = torch.autograd.grad((h, last), leaves, (dh, dl))
    # (states from held gates differ by 2^-91 of themselves)
    want = S.backward(g.clamp(-63.5, 63.5), x, h0, lengths, True, dh, dl, fmt)
    for a, w, e, t in zip(got, want[:3], want[3:], (g.dtype, g.dtype, F32)):
        S.check(a.detach(), w, e, t)


@pytest.mark.parametrize("ends", [False, True])
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("Bn,T,C", [(12, 200, 1024), (1, 1500, 96), (2, 150, 66), (2, 150, 35), (3, 13, 64), (1, 1, 40)])
def test_far_gates(Bn, T, C, dtype, fmt, ends):
    g, x, gen = S.fields(Bn, T, C, dtype, 3 * T + C)
    r = lambda *s: torch.randn(*s, device="cuda", generator=gen)
    h0, dh, dl = r(Bn, C), r(Bn, T, C).to(dtype), r(Bn, C)
    compare(far_gates(g, ends), x, h0, dh, dl, fmt)
    if Bn > 1:
        lengths = torch.randint(0, T + 1, (Bn,), device="cuda", generator=gen, dtype=torch.int32)
        compare(g, x, h0, dh, dl, fmt, lengths)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_masks_leave_their_neighbours_alone(dtype):
    """Every fourth column masked with -1e4 in every row: the other columns' gradients are those of a checkpoint without masks, bit for bit
    where the masked columns had held the largest gates anyway."""
    g, x, gen = S.fields(2, 100, 64, dtype, 4)
    dh = torch.randn(2, 100, 64, device="cuda", generator=gen).to(dtype)
    g[..., ::4] = -63.5
    out = []
    for mask in (-63.5, -1e4, -INF):
        g[..., ::4] = mask
        leaves = [t.clone().requires_grad_() for t in (g, x)]
        out.append(torch.autograd.grad(autograd.gated_scan(*leaves, mix=True, checkpoint="int8")[0], leaves, dh))
        assert torch.equal(out[-1][0], out[0][0]) and torch.equal(out[-1][1], out[0][1])


def test_far_gates_through_the_context():
    g, x, gen = S.fields(2, 130, 64, F32, 5)
    dh = torch.randn(2, 130, 64, device="cuda", generator=gen)
    for fmt in ("int8", "e4m3"):
        leaves = [far_gates(g, True).clone().requires_grad_(), x.clone().requires_grad_()]
        with checkpoints.saved_in_8_bits(fmt):
            h, _ = autograd.gated_scan(*leaves, mix=True)
        dg, dx = torch.autograd.grad(h, leaves, dh)
        wg, wx, _, eg, ex, _ = S.backward(g.clamp(-63.5, 63.5), x, None, None, True, dh, None, fmt)
        S.check(dg, wg, eg, F32, "dg")
        S.check(dx, wx, ex, F32, "dx")
