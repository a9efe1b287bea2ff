"""The gated recurrence, the activations and the 8-bit tensors: what their entry points refuse, on the host (no kernel is launched)."""
import ctypes as C

import pytest
import torch

from paper_2007_12792_b200 import autograd, binding as B, checkpoints

BIG = 1 << 40          # addresses far apart; never dereferenced: validation fails first


@pytest.fixture(scope="module")
def L():
    from paper_2007_12792_b200 import build
    build.build()
    return B.lib()


def scan(**kw):
    s = B.DnScan()
    s.batch, s.rows, s.cols, s.type, s.flags, s.format = 2, 100, 48, B.DN_F32, 0, 0
    for k, v in kw.items():
        setattr(s, k, v)
    return s


def rows(at, s, **kw):
    r = B.DnRows(at * BIG, s.rows * s.cols, s.cols)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def forward(L, s, g=None, x=None, h0=None, h=None, last=None, ck=None, n=1 << 40):
    g, x, h = g or rows(1, s), x or rows(2, s), h or rows(3, s)
    return L.dn_scan_forward(C.byref(s), C.byref(g), C.byref(x), h0, C.byref(h), last, ck, n, None)


def backward(L, s, g=None, x=None, ck=6 * BIG, n=1 << 40, dh=None, dlast=None, dg=None, dx=None, dh0=None):
    g, x, dg, dx = g or rows(1, s), x or rows(2, s), dg or rows(3, s), dx or rows(4, s)
    return L.dn_scan_backward(C.byref(s), C.byref(g), C.byref(x), ck, n, C.byref(dh) if dh else None, dlast, C.byref(dg), C.byref(dx), dh0, None)


@pytest.mark.parametrize("change,status", [
    (dict(batch=0), B.DN_ERR_SIZE), (dict(cols=0), B.DN_ERR_SIZE), (dict(rows=-1), B.DN_ERR_SIZE), (dict(batch=-3), B.DN_ERR_SIZE),
    (dict(rows=(1 << 30) + 1), B.DN_ERR_SIZE), (dict(cols=(1 << 30) + 1), B.DN_ERR_SIZE), (dict(batch=1 << 30, cols=1 << 20), B.DN_ERR_SIZE),
    (dict(type=3), B.DN_ERR_MODE), (dict(type=-1), B.DN_ERR_MODE), (dict(flags=2), B.DN_ERR_MODE), (dict(format=3), B.DN_ERR_MODE), (dict(format=-1), B.DN_ERR_MODE)])
def test_scan_refuses_sizes_and_modes(L, change, status):
    s = scan(**change)
    assert L.dn_scan_checkpoint_bytes(C.byref(s)) == 0
    assert forward(L, s) == status and backward(L, s) == status


def test_scan_refuses_missing_arrays(L):
    s = scan()
    assert L.dn_scan_checkpoint_bytes(None) == 0
    assert L.dn_scan_forward(None, None, None, None, None, None, None, 0, None) == B.DN_ERR_NULL
    for k in ("g", "x", "h"):
        assert forward(L, s, **{k: rows(1, s, data=None)}) == B.DN_ERR_NULL
    for k in ("g", "x", "dg", "dx"):
        assert backward(L, s, **{k: rows(1, s, data=None)}) == B.DN_ERR_NULL
    assert backward(L, s, ck=None) == B.DN_ERR_WORKSPACE
    need = L.dn_scan_checkpoint_bytes(C.byref(s))
    assert need == 2 * 2 * 48 * 4 and need % 256 == 0
    for bad in (dict(ck=6 * BIG + 128), dict(n=need - 1)):
        assert backward(L, s, **bad) == B.DN_ERR_WORKSPACE
        assert forward(L, s, **{"ck": 6 * BIG, **bad}) == B.DN_ERR_WORKSPACE
    for fmt in (B.DN_INT8, B.DN_E4M3):       # codes of gate and input, their scales (2 blocks of columns, 128 padded rows), the states
        assert L.dn_scan_checkpoint_bytes(C.byref(scan(format=fmt))) == 2 * 9728 + 2 * 512 + 768


@pytest.mark.parametrize("change", [dict(batch_stride=-1), dict(row_stride=-48), dict(row_stride=1 << 60), dict(data=BIG + 2)])
def test_scan_refuses_layouts(L, change):
    s = scan()
    for k in ("g", "x", "h"):
        assert forward(L, s, **{k: rows(1, s, **change)}) == B.DN_ERR_LAYOUT
    for k in ("g", "x", "dh", "dg", "dx"):
        assert backward(L, s, **{k: rows(1, s, **change)}) == B.DN_ERR_LAYOUT


@pytest.mark.parametrize("change", [dict(row_stride=47), dict(row_stride=0), dict(batch_stride=0), dict(batch_stride=4799)])
def test_scan_refuses_outputs_that_meet_themselves(L, change):
    s = scan()
    assert forward(L, s, h=rows(3, s, **change)) == B.DN_ERR_LAYOUT
    assert backward(L, s, dg=rows(3, s, **change)) == B.DN_ERR_LAYOUT
    assert backward(L, s, dx=rows(4, s, **change)) == B.DN_ERR_LAYOUT


def test_scan_refuses_overlap(L):
    s = scan()
    edge = 2 * 48 * 4
    assert forward(L, s, h=rows(1, s)) == B.DN_ERR_ALIAS
    assert forward(L, s, h=rows(2, s, data=2 * BIG + 48 * 4)) == B.DN_ERR_ALIAS
    assert forward(L, s, h0=3 * BIG) == B.DN_ERR_ALIAS and forward(L, s, last=3 * BIG + 400) == B.DN_ERR_ALIAS
    assert forward(L, s, h0=7 * BIG, last=7 * BIG + 4) == B.DN_ERR_ALIAS
    assert forward(L, s, last=BIG) == B.DN_ERR_ALIAS
    assert forward(L, s, ck=3 * BIG + 256) == B.DN_ERR_ALIAS and forward(L, s, ck=BIG) == B.DN_ERR_ALIAS
    assert forward(L, scan(lengths=3 * BIG)) == B.DN_ERR_ALIAS and forward(L, scan(lengths=8 * BIG), last=8 * BIG) == B.DN_ERR_ALIAS
    assert backward(L, s, dg=rows(1, s)) == B.DN_ERR_ALIAS and backward(L, s, dx=rows(3, s)) == B.DN_ERR_ALIAS
    assert backward(L, s, dh=rows(3, s)) == B.DN_ERR_ALIAS and backward(L, s, ck=3 * BIG) == B.DN_ERR_ALIAS
    assert backward(L, s, dh0=6 * BIG) == B.DN_ERR_ALIAS and backward(L, s, dh0=7 * BIG, dlast=7 * BIG + edge - 4) == B.DN_ERR_ALIAS
    # columns of one wider array do not meet where they lie side by side
    wide = dict(batch_stride=100 * 96, row_stride=96)
    assert forward(L, s, g=rows(1, s, **wide), h=rows(1, s, data=BIG + 47 * 4, **wide)) == B.DN_ERR_ALIAS
    assert backward(L, s, dg=rows(3, s, **wide), dx=rows(3, s, data=3 * BIG + 47 * 4, **wide)) == B.DN_ERR_ALIAS


def test_scan_refuses_misaligned_edges(L):
    s = scan()
    assert forward(L, s, h0=7 * BIG + 2) == B.DN_ERR_LAYOUT and forward(L, s, last=7 * BIG + 1) == B.DN_ERR_LAYOUT
    assert forward(L, scan(lengths=8 * BIG + 2)) == B.DN_ERR_LAYOUT
    assert backward(L, s, dh0=7 * BIG + 2) == B.DN_ERR_LAYOUT and backward(L, s, dlast=7 * BIG + 2) == B.DN_ERR_LAYOUT


def test_packing_and_activations_refuse(L):
    p, q, r = BIG, 2 * BIG, 3 * BIG
    assert [L.dn_packed_bytes(n) for n in (1, 16, 32, 33, 100)] == [17, 17, 33, 50, 116]
    assert L.dn_packed_bytes(0) == 0 and L.dn_packed_bytes(-5) == 0 and L.dn_packed_bytes(1 << 50) == 0
    calls = {
        "pack": lambda n=64, t=B.DN_F32, a=p, b=q, f=B.DN_INT8: L.dn_pack(n, t, a, f, b, None),
        "unpack": lambda n=64, t=B.DN_F32, a=p, b=q, f=B.DN_INT8: L.dn_unpack(n, t, b, f, a, None),
        "forward": lambda n=64, t=B.DN_F32, a=p, b=q, f=B.DN_INT8: L.dn_activation_forward(n, t, 0, a, r, f, b, None),
        "backward": lambda n=64, t=B.DN_F32, a=p, b=q, f=B.DN_INT8: L.dn_activation_backward(n, t, 0, b, f, a, r, None)}
    for name, call in calls.items():
        assert call(n=0) == B.DN_ERR_SIZE and call(n=-1) == B.DN_ERR_SIZE and call(n=1 << 50) == B.DN_ERR_SIZE, name
        assert call(t=3) == B.DN_ERR_MODE and call(f=0) == B.DN_ERR_MODE and call(f=3) == B.DN_ERR_MODE, name
        assert call(a=None) == B.DN_ERR_NULL, name
        assert call(a=p + 2) == B.DN_ERR_LAYOUT and call(b=q + 8) == B.DN_ERR_LAYOUT, name
        if name != "backward":                                    # (dy and the packed input are both only read)
            assert call(a=p + 32, b=p) == B.DN_ERR_ALIAS, name
        if name != "forward":
            assert call(b=None) == B.DN_ERR_NULL, name
    assert L.dn_activation_forward(64, 0, 3, p, r, 1, q, None) == B.DN_ERR_MODE
    assert L.dn_activation_backward(64, 0, -1, q, 1, p, r, None) == B.DN_ERR_MODE
    assert L.dn_activation_forward(64, 0, 0, p, p + 4, 1, q, None) == B.DN_ERR_ALIAS
    assert L.dn_activation_forward(64, 0, 0, p, q, 1, q, None) == B.DN_ERR_ALIAS
    assert L.dn_activation_backward(64, 0, 0, q, 1, p, p + 4, None) == B.DN_ERR_ALIAS


def test_python_refuses(L):
    z = torch.zeros(2, 3, 4)
    for call in (lambda: autograd.gated_scan(z, z), lambda: autograd.activation(z), lambda: checkpoints.pack(z),
                 lambda: autograd.activation(z, "relu"), lambda: autograd.activation(z, checkpoint=None),
                 lambda: autograd.gated_scan(z, z, checkpoint="fp4"), lambda: checkpoints.pack(z, "int4"),
                 lambda: checkpoints.saved_in_8_bits("int4"), lambda: B.Scan(1, 1, 1, checkpoint="half")):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: autograd.gated_scan(1, 2), lambda: autograd.activation("x"), lambda: B.dn_scan_checkpoint_bytes(B.Scan(1, 1, 1, dtype="bf16"))):
        with pytest.raises(TypeError):
            call()
    assert B.dn_scan_checkpoint_bytes(B.Scan(0, 1, 1)) == 0
    with pytest.raises(ValueError):
        B.dn_scan_checkpoint_bytes(B.Scan(1, 1, 1, dtype=torch.float64))
