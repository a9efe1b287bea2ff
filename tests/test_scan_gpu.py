"""The gated recurrence and its gradients against their definition in 64 bits, row by row."""
import pytest
import torch

import scan_util as S
from paper_2007_12792_b200 import autograd
from paper_2007_12792_b200 import binding as B

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
DTYPES = [F32, BF16, F16]


def call_forward(g, x, h0, lengths, mix, fmt=None, keep=True, h=None, h_last=None, stream=None):
    p = B.Scan(*g.shape, dtype=g.dtype, mix=mix, checkpoint=fmt, lengths=lengths)
    h = torch.full(g.shape, 7.0, dtype=g.dtype, device="cuda") if h is None else h
    h_last = torch.full((g.shape[0], g.shape[2]), 7.0, device="cuda") if h_last is None else h_last
    ck = torch.full((B.dn_scan_checkpoint_bytes(p),), 255, dtype=torch.uint8, device="cuda") if keep else None
    B.dn_scan_forward(p, g, x, h0, h, h_last, ck, stream)
    return p, h, h_last, ck


def call_backward(p, g, x, ck, dh, dh_last, stream=None):
    new = lambda *s: torch.full(s, 7.0, dtype=p.dtype, device="cuda")
    dg, dx, dh0 = new(*p.shape), new(*p.shape), torch.full((p.batch, p.cols), 7.0, device="cuda")
    B.dn_scan_backward(p, g, x, ck, dh, dh_last, dg, dx, dh0, stream)
    return dg, dx, dh0


def compare(g, x, h0, lengths, mix, dh, dh_last, fmt):
    p, h, h_last, ck = call_forward(g, x, h0, lengths, mix, fmt)
    full = fmt is None
    dg, dx, dh0 = call_backward(p, g if full else None, x if full else None, ck, dh, dh_last)
    torch.cuda.synchronize()
    wh, wl, _, eh, el, _ = S.forward(g, x, h0, lengths, mix)
    S.check(h, wh, eh, g.dtype, "h")
    S.check(h_last, wl, el, F32, "h_last")
    wg, wx, w0, eg, ex, e0 = S.backward(g, x, h0, lengths, mix, dh, dh_last, fmt)
    S.check(dg, wg, eg, g.dtype, "dg")
    S.check(dx, wx, ex, g.dtype, "dx")
    S.check(dh0, w0, e0, F32, "dh0")


def random_case(Bn, T, C, dtype, seed, ragged=False):
    g, x, gen = S.fields(Bn, T, C, dtype, seed)
    r = lambda *s: torch.randn(*s, device="cuda", generator=gen)
    lengths = None
    if ragged:
        lengths = torch.randint(0, T + 1, (Bn,), device="cuda", generator=gen, dtype=torch.int32)
        if Bn > 3:
            lengths[:4] = torch.tensor([T, 0, 1, -5], dtype=torch.int32)
        if Bn > 4:
            lengths[4] = T + 9
    return g, x, r(Bn, C), lengths, r(Bn, T, C).to(dtype), r(Bn, C)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T", [0, 1, 2, 8, 9, 15, 16, 17, 63, 64, 65, 127, 128, 129, 511, 513, 1100])
def test_rows(T, dtype):
    for k, (C, mix, fmt) in enumerate([(33, True, None), (64, False, "int8"), (100, True, "e4m3")]):
        g, x, h0, lengths, dh, dh_last = random_case(2, T, C, dtype, 100 * T + k)
        compare(g, x, h0, lengths, mix, dh, dh_last, fmt)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("C", [1, 2, 3, 7, 8, 15, 16, 31, 32, 63, 65, 130, 257, 2050])
def test_columns(C, dtype):
    for k, (T, mix, fmt) in enumerate([(70, True, "int8"), (300, False, None), (13, True, "e4m3"), (1, False, "int8")]):
        g, x, h0, lengths, dh, dh_last = random_case(3, T, C, dtype, 100 * C + k)
        compare(g, x, h0, lengths, mix, dh, dh_last, fmt)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("fmt", [None, "int8", "e4m3"])
@pytest.mark.parametrize("Bn,T,C", [(7, 200, 37), (5, 1, 64), (6, 12, 40), (5, 64, 32), (6, 700, 96), (40, 130, 1024), (5, 2100, 18)])
def test_samples_of_unlike_length(Bn, T, C, dtype, fmt):
    g, x, h0, lengths, dh, dh_last = random_case(Bn, T, C, dtype, Bn + T + C, ragged=True)
    live = torch.arange(T, device="cuda")[None, :, None] < lengths[:, None, None]
    compare(g, x, h0, lengths, True, dh, dh_last, fmt)
    # what stands in the rows behind a sequence is not read
    for t in (g, x, dh):
        t[~live.expand_as(t)] = float("nan")
    p, h, h_last, ck = call_forward(g, x, h0, lengths, False, fmt)
    out = [h, h_last, *call_backward(p, g, x, ck, dh, dh_last)]
    for t in out:
        assert torch.isfinite(t).all()
    for t in (out[0], out[2], out[3]):
        assert float(t[~live.expand_as(t)].abs().sum()) == 0.0


@pytest.mark.parametrize("dtype", DTYPES)
def test_many_columns_and_many_strips(dtype):
    """One block per strip of columns (no cluster), and clusters of 2 to 16 blocks on the way there."""
    for Bn, T, C in [(24, 150, 1024), (9, 400, 1100), (4, 530, 640), (2, 1030, 512), (1, 2500, 256), (1, 5000, 64), (1, 9000, 8)]:
        for fmt in (None, "int8"):
            g, x, h0, lengths, dh, dh_last = random_case(Bn, T, C, dtype, T)
            compare(g, x, h0, lengths, True, dh, dh_last, fmt)


@pytest.mark.parametrize("dtype", DTYPES)
def test_missing_edges_and_gradients(dtype):
    g, x, h0, _, dh, dh_last = random_case(2, 90, 40, dtype, 5)
    for fmt in (None, "e4m3"):
        compare(g, x, None, None, True, dh, dh_last, fmt)
        compare(g, x, h0, None, False, None, dh_last, fmt)
        compare(g, x, h0, None, True, dh, None, fmt)
        compare(g, x, h0, None, True, None, None, fmt)
    p = B.Scan(*g.shape, dtype=dtype)
    h, h2 = torch.empty_like(g), torch.empty_like(g)
    B.dn_scan_forward(p, g, x, None, h, None)                       # neither a state given nor one taken, nothing kept
    B.dn_scan_forward(p, g, x, torch.zeros_like(h0), h2, torch.empty_like(h0))
    assert torch.equal(h, h2)


@pytest.mark.parametrize("dtype", DTYPES)
def test_strides(dtype):
    """Halves of one projection, time-major arrays, a gate shared by the batch or by all rows, places off 4 bytes, wide outputs."""
    Bn, T, C = 3, 77, 34
    g, x, h0, _, dh, dh_last = random_case(Bn, T, C, dtype, 11)
    both = torch.stack([g, x], 2)
    time_major = lambda t: t.transpose(0, 1).contiguous().transpose(0, 1)
    odd = torch.zeros(Bn * T * C + 1, dtype=dtype, device="cuda")[1:].view(Bn, T, C).copy_(x)
    wide_odd = torch.zeros(Bn, T, C + 1, dtype=dtype, device="cuda")[..., :C].copy_(g)
    cases = [(both[:, :, 0], both[:, :, 1], dh), (time_major(g), time_major(x), time_major(dh)), (g[:1].expand(Bn, T, C), x, dh[:, :1].expand(Bn, T, C)),
             (g[:, :1].expand(Bn, T, C), odd, dh), (wide_odd, x, dh)]
    for gg, xx, dd in cases:
        for fmt in (None, "int8"):
            compare(gg, xx, h0, None, True, dd, dh_last, fmt)
    # outputs: time-major, columns of one wider array, and nothing beside them is written
    want = call_forward(g, x, h0, None, True)
    h = torch.full((T, Bn, C), 7.0, dtype=dtype, device="cuda").transpose(0, 1)
    call_forward(g, x, h0, None, True, h=h)
    assert torch.equal(h, want[1])
    grads = call_backward(want[0], g, x, want[3], dh, dh_last)
    wide = torch.full((Bn, T + 2, 2 * C + 6), 7.0, dtype=dtype, device="cuda")
    dg, dx, dh0 = wide[:, 1:T + 1, 2:C + 2], wide[:, 1:T + 1, C + 2:2 * C + 2], torch.empty_like(h0)
    B.dn_scan_backward(want[0], g, x, want[3], dh, dh_last, dg, dx, dh0)
    assert torch.equal(dg, grads[0]) and torch.equal(dx, grads[1]) and torch.equal(dh0, grads[2])
    wide[:, 1:T + 1, 2:2 * C + 2] = 7.0
    assert bool((wide == 7.0).all())


@pytest.mark.parametrize("dtype", DTYPES)
def test_gates_at_the_ends_of_their_range(dtype):
    g, x, h0, _, dh, dh_last = random_case(2, 80, 48, dtype, 3)
    big = torch.finfo(dtype).max
    g[:, ::7] = float("-inf")                                       # forget everything
    g[:, 3::7] = float("inf")                                       # keep everything
    g[:, 5::7, ::2] = -big
    g[:, 6::7, 1::2] = big
    for mix in (False, True):
        compare(g, x, h0, None, mix, dh, dh_last, None)
    h, _ = autograd.gated_scan(g, x, h0, mix=True)
    assert torch.equal(h[:, 3], h[:, 2]) and torch.equal(h[:, 7], x[:, 7])


@pytest.mark.parametrize("dtype", DTYPES)
def test_values_that_are_not_finite_stay_in_their_column(dtype):
    g, x, h0, _, dh, dh_last = random_case(1, 150, 70, dtype, 4)
    want = call_forward(g, x, h0, None, True, "int8")
    grads = call_backward(want[0], None, None, want[3], dh, dh_last)
    g[0, 40, 5], x[0, 90, 66] = float("nan"), float("inf")
    got = call_forward(g, x, h0, None, True, "int8")
    other = [c for c in range(70) if c not in (5, 66)]
    assert torch.equal(got[1][..., other], want[1][..., other]) and torch.equal(got[1][:, :40], want[1][:, :40])
    assert torch.isnan(got[1][0, 40:, 5]).all() and not torch.isfinite(got[1][0, 90:, 66]).any()
    again = call_backward(got[0], None, None, got[3], dh, dh_last)
    for a, b in zip(grads, again):
        assert torch.equal(a[..., other], b[..., other])
    assert torch.isnan(again[0][0, 40, 5]) and torch.isnan(again[0][0, 90, 66])


def test_a_step_updates_the_state_in_place():
    for dtype in DTYPES:
        g, x, h0, _, _, _ = random_case(5, 6, 66, dtype, 9)
        state, rows = h0.clone(), []
        for t in range(6):
            p = B.Scan(5, 1, 66, dtype=dtype, mix=True)
            h = torch.empty(5, 1, 66, dtype=dtype, device="cuda")
            B.dn_scan_forward(p, g[:, t:t + 1], x[:, t:t + 1], state, h, state)
            rows.append(h)
        wh, wl, _, eh, el, _ = S.forward(g, x, h0, None, True)
        S.check(torch.cat(rows, 1), wh, eh, dtype, "h")
        S.check(state, wl, el, F32, "state")
        long = random_case(2, 3000, 24, dtype, 10)                   # a cluster of blocks, each of which reads the state
        s1, s2 = long[2].clone(), torch.empty_like(long[2])
        call_forward(long[0], long[1], long[2], None, False, h_last=s2)
        call_forward(long[0], long[1], s1, None, False, h_last=s1)
        assert torch.equal(s1, s2)


@pytest.mark.parametrize("fmt", [None, "int8", "e4m3"])
@pytest.mark.parametrize("dtype", DTYPES)
def test_as_a_torch_op(dtype, fmt):
    g, x, h0, lengths, dh, dh_last = random_case(5, 140, 50, dtype, 21, ragged=True)
    p, h, h_last, ck = call_forward(g, x, h0, lengths, True, fmt)
    want = call_backward(p, g, x, ck, dh, dh_last)
    leaves = [t.clone().requires_grad_() for t in (g, x, h0)]
    oh, ol = autograd.gated_scan(*leaves, lengths=lengths, mix=True, checkpoint=fmt)
    assert torch.equal(oh, h) and torch.equal(ol, h_last) and oh.requires_grad and ol.dtype == F32
    got = torch.autograd.grad((oh, ol), leaves, (dh, dh_last), retain_graph=True)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    # one output alone, a gradient that is one number for all places, leaves that want none
    got = torch.autograd.grad(ol.sum(), leaves, retain_graph=True)
    for a, b in zip(got, call_backward(p, g, x, ck, None, torch.ones_like(h_last))):
        assert torch.equal(a, b)
    got = torch.autograd.grad(oh.float().sum(), leaves)
    for a, b in zip(got, call_backward(p, g, x, ck, torch.ones_like(h), None)):
        assert torch.equal(a, b)
    oh, _ = autograd.gated_scan(g, leaves[1], lengths=lengths, mix=True, checkpoint=fmt)
    assert torch.isfinite(torch.autograd.grad(oh, leaves[1], dh)[0]).all()
    with torch.no_grad():
        oh, ol = autograd.gated_scan(*leaves, lengths=lengths, mix=True, checkpoint=fmt)
    assert not oh.requires_grad and torch.equal(oh, h)


def test_gradients_by_differences():
    """Central differences of the 64-bit definition (a step of 1e-6 there: their error is 1e-10 of the third derivatives, of order 1)."""
    g, x, h0, _, dh, dh_last = random_case(1, 70, 3, F32, 31)
    leaves = [t.clone().requires_grad_() for t in (g, x, h0)]
    for mix in (False, True):
        def loss(*a):
            h, l = S.forward(*a, None, mix)[:2]
            return float((h * dh.to(S.F64)).sum() + (l * dh_last.to(S.F64)).sum())
        got = torch.autograd.grad(autograd.gated_scan(*leaves, mix=mix), leaves, (dh, dh_last))
        eg, ex, e0 = S.backward(g, x, h0, None, mix, dh, dh_last)[3:]
        for k, e in enumerate((eg, ex, e0)):
            for place in [(0, 0, 0), (0, 41, 1), (0, 69, 2), (0, 63, 0), (0, 64, 1)]:
                place = place if k < 2 else (0, place[2])
                args = [t.to(S.F64).clone() for t in (g, x, h0)]
                args[k][place] += 1e-6
                up = loss(*args)
                args[k][place] -= 2e-6
                want = (up - loss(*args)) / 2e-6
                assert abs(float(got[k][place]) - want) <= float(e[place]) + 2.0 ** -24 * abs(want) + 1e-7, (mix, k, place)


def test_no_rows_as_a_torch_op():
    g = torch.empty(3, 0, 5, device="cuda", requires_grad=True)
    x, h0 = torch.empty(3, 0, 5, device="cuda", requires_grad=True), torch.randn(3, 5, device="cuda", requires_grad=True)
    for fmt in (None, "int8"):
        h, last = autograd.gated_scan(g, x, h0, checkpoint=fmt)
        assert h.shape == (3, 0, 5) and torch.equal(last, h0)
        d = torch.randn(3, 5, device="cuda")
        dg, dx, dh0 = torch.autograd.grad(last, (g, x, h0), d)
        assert dg.shape == dx.shape == (3, 0, 5) and torch.equal(dh0, d)


def test_the_first_call_of_a_process_may_be_captured():
    """A child process whose first calls stand in a graph: what they ask the device for is no work on a stream."""
    import subprocess
    import sys
    code = """
import torch
from paper_2007_12792_b200 import autograd, binding as B
g, x, d = (torch.randn(2, 1200, 64, device="cuda", dtype=torch.bfloat16) for _ in range(3))
p = B.Scan(2, 1200, 64, dtype=torch.bfloat16, mix=True, checkpoint="int8")
h, dg, dx, last, ck = torch.empty_like(g), torch.empty_like(g), torch.empty_like(g), torch.empty(2, 64, device="cuda"), B.new_scan_checkpoint(p)
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    B.dn_scan_forward(p, g, x, None, h, last, ck)
    B.dn_scan_backward(p, None, None, ck, d, None, dg, dx, None)
graph.replay()
torch.cuda.synchronize()
out = [t.clone() for t in (h, last, dg, dx)]
B.dn_scan_forward(p, g, x, None, h, last, ck)
B.dn_scan_backward(p, None, None, ck, d, None, dg, dx, None)
assert all(torch.equal(a, b) for a, b in zip(out, (h, last, dg, dx)))
print("same")
"""
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "same" in r.stdout, r.stderr[-2000:]


def test_no_second_derivative():
    g, x, _, _, dh, _ = random_case(1, 20, 8, F32, 1)
    x.requires_grad_()
    h, _ = autograd.gated_scan(g, x)
    with pytest.raises(RuntimeError, match="create_graph"):
        torch.autograd.grad(h, x, dh, create_graph=True)


def test_refused_tensors():
    g, x, h0, lengths, dh, dh_last = random_case(2, 20, 8, F32, 1)
    for bad in (lambda: autograd.gated_scan(g, x.half()), lambda: autograd.gated_scan(g, x[:, :19]), lambda: autograd.gated_scan(g[0], x[0]),
                lambda: autograd.gated_scan(g.double(), x.double()), lambda: autograd.gated_scan(g, x, h0.half()), lambda: autograd.gated_scan(g, x, h0[:1]),
                lambda: autograd.gated_scan(g, x, lengths=torch.ones(2, device="cuda")), lambda: autograd.gated_scan(g, x, lengths=torch.ones(3, device="cuda", dtype=torch.int32)),
                lambda: autograd.gated_scan(g, x, h0.cpu())):
        with pytest.raises(ValueError):
            bad()
    p = B.Scan(2, 20, 8)
    h = torch.empty_like(g)
    with pytest.raises(ValueError, match="adjacent"):
        B.dn_scan_forward(p, g.transpose(1, 2).contiguous().transpose(1, 2), x, h0, h, None)
    for empty in (torch.empty(0, 5, 4, device="cuda"), torch.empty(2, 5, 0, device="cuda")):
        with pytest.raises(B.DnError) as e:
            autograd.gated_scan(empty, empty)
        assert e.value.status == B.DN_ERR_SIZE
    for call, status in [(lambda: B.dn_scan_forward(p, g, x, h0, g, None), B.DN_ERR_ALIAS), (lambda: B.dn_scan_forward(p, g, x, h0, h[:, :1].expand_as(h), None), B.DN_ERR_LAYOUT),
                         (lambda: B.dn_scan_backward(p, g, x, torch.empty(64, dtype=torch.uint8, device="cuda"), dh, None, h, torch.empty_like(h), None), B.DN_ERR_WORKSPACE)]:
        with pytest.raises(B.DnError) as e:
            call()
        assert e.value.status == status


@pytest.mark.parametrize("fmt", [None, "int8"])
def test_streams_graphs_and_repetition(fmt):
    """Two calls at once on two streams; forward and backward captured into a graph and replayed on new data, while a graph of eager
    calls lives; the same call twice: the same bits each time."""
    a, b = random_case(4, 600, 130, BF16, 41), random_case(4, 600, 130, BF16, 42)
    one = call_forward(a[0], a[1], a[2], None, True, fmt)
    want_a = [one[1], one[2], *call_backward(one[0], a[0], a[1], one[3], a[4], a[5])]
    two = call_forward(b[0], b[1], b[2], None, True, fmt)
    want_b = [two[1], two[2], *call_backward(two[0], b[0], b[1], two[3], b[4], b[5])]
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    results = []
    for s, c in ((s1, a), (s2, b)):
        with torch.cuda.stream(s):
            r = call_forward(c[0], c[1], c[2], None, True, fmt)
            results.append([r[1], r[2], *call_backward(r[0], c[0], c[1], r[3], c[4], c[5])])
    torch.cuda.synchronize()
    for got, want in zip(results, (want_a, want_b)):
        for u, v in zip(got, want):
            assert torch.equal(u, v)
    # a stream that is named
    h = torch.empty_like(a[0]); last = torch.empty_like(a[2])
    s1.wait_stream(torch.cuda.current_stream())
    B.dn_scan_forward(one[0], a[0], a[1], a[2], h, last, one[3], stream=s1)
    s1.synchronize()
    assert torch.equal(h, want_a[0]) and torch.equal(last, want_a[1])
    # captured: the leaves of an eager graph that is still alive
    leaves = [t.clone().requires_grad_() for t in a[:3]]
    alive = autograd.gated_scan(*leaves, mix=True, checkpoint=fmt)
    static = [t.detach().clone().requires_grad_() for t in leaves]
    d, dl = a[4].clone(), a[5].clone()

    def step():
        out = autograd.gated_scan(*static, mix=True, checkpoint=fmt)
        return [*out, *torch.autograd.grad(out, static, (d, dl))]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for c, want in ((b, want_b), (a, want_a)):
        with torch.no_grad():
            for t, v in zip([*static, d, dl], [c[0], c[1], c[2], c[4], c[5]]):
                t.copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        for u, v in zip(out, want):
            assert torch.equal(u, v)
    for u, v in zip(torch.autograd.grad(alive, leaves, (a[4], a[5])), want_a[2:]):
        assert torch.equal(u, v)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("odd", [0, 1])
def test_rows_far_apart(dtype, odd):
    """Rows of one wide array, 64 MiB and more apart: offsets within a tile pass 32 bits.  odd: off the 16 bytes of a bulk copy."""
    T, C, W = 70, 8, (1 << 26) // (4 if dtype == F32 else 2) + 64
    wide = torch.empty(1, T, W, dtype=dtype, device="cuda")
    part = lambda k: wide[:, :, 16 * k + odd * 2:16 * k + odd * 2 + C]
    g, x, h0, _, dh, dh_last = random_case(1, T, C, dtype, 8)
    for k, t in enumerate((g, x, dh)):
        part(k).copy_(t)
    for fmt in (None, "int8"):
        p, h, h_last, ck = call_forward(part(0), part(1), h0, None, True, fmt, h=part(3))
        dh0 = torch.empty_like(h0)
        B.dn_scan_backward(p, part(0), part(1), ck, part(2), dh_last, part(4), part(5), dh0)
        wh, _, _, eh, _, _ = S.forward(g, x, h0, None, True)
        wg, wx, w0, eg, ex, e0 = S.backward(g, x, h0, None, True, dh, dh_last, fmt)
        for got, want, err, d in ((part(3), wh, eh, dtype), (part(4), wg, eg, dtype), (part(5), wx, ex, dtype), (dh0, w0, e0, F32)):
            S.check(got, want, err, d)


def test_negated_views():
    """Complex conjugates hand out views whose sign is only noted: the ops resolve them, the calls on buffers refuse them."""
    g, x, h0, _, dh, _ = random_case(2, 20, 8, F32, 2)
    neg = torch.complex(x, x).conj().imag
    assert neg.is_neg()
    h, _ = autograd.gated_scan(g, neg, h0)
    want, _ = autograd.gated_scan(g, -x, h0)
    assert torch.equal(h, want)
    flat = torch._neg_view(x)
    assert torch.equal(autograd.activation(flat), autograd.activation(-x))
    from paper_2007_12792_b200 import checkpoints
    assert torch.equal(checkpoints.pack(flat).unpack(), checkpoints.pack(-x).unpack())
    with pytest.raises(ValueError, match="negated"):
        B.dn_scan_forward(B.Scan(2, 20, 8), torch._neg_view(g), x, h0, torch.empty_like(g), None)


def test_offsets_beyond_32_bits():
    """2.2e9 elements: the last rows, from short memories, against a recurrence over the last 200 rows alone (2^-100 is left of what
    was before them)."""
    T, C = 1 << 20, 2100
    gen = torch.Generator(device="cuda"); gen.manual_seed(3)
    tail = lambda t: t[:, -200:].clone()
    big = lambda: torch.empty(1, T, C, dtype=BF16, device="cuda")
    g, x, dh = big(), big(), big()
    for t in (g, x, dh):
        t[:] = torch.randn(1, 4096, C, device="cuda", generator=gen).to(BF16).repeat(1, T // 4096, 1)
        t[:, -200:] = torch.randn(1, 200, C, device="cuda", generator=gen).to(BF16)
    g.clamp_(-4.0, 0.0)
    p, h, h_last, ck = call_forward(g, x, None, None, True, "int8")
    wh, wl, _, eh, el, _ = S.forward(tail(g), tail(x), None, None, True)
    S.check(h[:, -100:], wh[:, -100:], eh[:, -100:] + 1e-20, BF16, "h")
    S.check(h_last, wl, el + 1e-20, F32, "h_last")
    dl = torch.randn(1, C, device="cuda", generator=gen)
    dg, dx, dh0 = call_backward(p, None, None, ck, dh, dl)
    # the last 128 rows are the last two chunks: their states are those of the 200 rows up to 2^-72
    wg, wx, _, eg, ex, _ = S.backward(tail(g)[:, -192:], tail(x)[:, -192:], None, None, True, tail(dh)[:, -192:], dl, "int8")
    S.check(dx[:, -60:], wx[:, -60:], ex[:, -60:] + 1e-15, BF16, "dx")
    S.check(dg[:, -60:], wg[:, -60:], eg[:, -60:] + 1e-15, BF16, "dg")
    first = S.backward(g[:, :192], x[:, :192], None, None, True, dh[:, :192], None, "int8")
    S.check(dx[:, :60], first[1][:, :60], first[4][:, :60] + 1e-15, BF16, "dx of the first rows")
    S.check(dg[:, :60], first[0][:, :60], first[3][:, :60] + 1e-15, BF16, "dg of the first rows")
