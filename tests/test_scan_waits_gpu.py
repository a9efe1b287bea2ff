"""The recurrence's waits have a limit.  With it at none (the flags for tests) each gives up at its first look: the kernel returns, what
was waited for and what depends on it is NaN, and the next call is as good as ever."""
import ctypes as C

import pytest
import torch

import scan_util as S
from paper_2007_12792_b200 import binding as B

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
CODE = {F32: B.DN_F32, BF16: B.DN_BF16, F16: B.DN_F16}
TILES, BLOCKS = B.DN_SCAN_GIVE_UP_TILES, B.DN_SCAN_GIVE_UP_BLOCKS


def rows(t):
    return B.DnRows(t.data_ptr(), t.stride(0), t.stride(1))


class Case:
    def __init__(self, Bn, T, Cc, dtype, fmt, ragged=False):
        self.g, self.x, gen = S.fields(Bn, T, Cc, dtype, 1)
        self.dh = torch.randn(Bn, T, Cc, device="cuda", generator=gen).to(dtype)
        self.dl = torch.randn(Bn, Cc, device="cuda", generator=gen)
        self.n = torch.full((Bn,), T, dtype=torch.int32, device="cuda")
        if ragged:
            self.n[1::2] = T // 2 + 3
        self.live = (torch.arange(T, device="cuda")[None] < self.n[:, None])[:, :, None].expand(Bn, T, Cc)
        self.s = B.DnScan(Bn, T, Cc, CODE[dtype], B.DN_SCAN_MIX, fmt, self.n.data_ptr())
        self.bytes = B.lib().dn_scan_checkpoint_bytes(C.byref(self.s))

    def forward(self, flags=0):
        self.s.flags = B.DN_SCAN_MIX | flags
        h, last = torch.full_like(self.g, 7.0), torch.full_like(self.dl, 7.0)
        ck = torch.full((self.bytes,), 255, dtype=torch.uint8, device="cuda")
        st = B.lib().dn_scan_forward(C.byref(self.s), C.byref(rows(self.g)), C.byref(rows(self.x)), None, C.byref(rows(h)), last.data_ptr(), ck.data_ptr(), self.bytes,
                                     torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert st == 0
        return h, last, ck

    def backward(self, ck, flags=0):
        self.s.flags = B.DN_SCAN_MIX | flags
        dg, dx, d0 = torch.full_like(self.g, 7.0), torch.full_like(self.g, 7.0), torch.full_like(self.dl, 7.0)
        st = B.lib().dn_scan_backward(C.byref(self.s), C.byref(rows(self.g)), C.byref(rows(self.x)), ck.data_ptr(), self.bytes, C.byref(rows(self.dh)), self.dl.data_ptr(),
                                      C.byref(rows(dg)), C.byref(rows(dx)), d0.data_ptr(), torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert st == 0
        return dg, dx, d0

    def lost(self, *fields, edge):
        for t in fields:
            assert bool(torch.isnan(t[self.live]).all()) and float(t[~self.live].abs().sum()) == 0.0
        assert bool(torch.isnan(edge).all())

    def check(self, flags):
        good = self.forward()
        grads = self.backward(good[2])
        h, last, ck = self.forward(flags)
        self.lost(h, edge=last)
        if self.s.format:                                # the states that were kept are NaN, gate and input are right: so is dx, which needs no state
            dg, dx, d0 = self.backward(ck)
            assert torch.equal(dx, grads[1]) and torch.equal(d0, grads[2]) and bool(torch.isnan(dg[:, 64:][self.live[:, 64:]]).all())
        dg, dx, d0 = self.backward(good[2], flags)
        self.lost(dg, dx, edge=d0)
        for a, b in zip(self.forward()[:2] + self.backward(good[2]), good[:2] + grads):
            assert torch.equal(a, b)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("fmt", [B.DN_SAVE_FULL, B.DN_INT8, B.DN_E4M3])
def test_tiles_that_do_not_come(dtype, fmt):
    Case(20, 300, 2048, dtype, fmt, ragged=True).check(TILES)      # a block per strip of columns
    Case(1, 8200, 1024, dtype, fmt).check(TILES)                   # clusters of blocks


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("cols", [1024, 1023, 8])                  # by bulk copies, without, few columns
def test_blocks_that_do_not_answer(dtype, cols):
    Case(1, 8200, cols, dtype, B.DN_SAVE_FULL).check(BLOCKS)
    if cols == 1024:
        Case(2, 4200, cols, dtype, B.DN_INT8, ragged=True).check(BLOCKS)
        Case(1, 8200, cols, dtype, B.DN_INT8).check(TILES | BLOCKS)


def test_the_flags_are_no_others():
    from paper_2007_12792_b200 import build
    build.build()
    size = lambda flags: B.lib().dn_scan_checkpoint_bytes(C.byref(B.DnScan(2, 100, 48, B.DN_F32, flags, 0, None)))
    assert size(0) == size(TILES) == size(BLOCKS) == size(TILES | BLOCKS | B.DN_SCAN_MIX) > 0
    assert [size(1 << k) for k in range(32) if 1 << k not in (B.DN_SCAN_MIX, TILES, BLOCKS)] == [0] * 29
