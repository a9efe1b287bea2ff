"""Saved tensors in 8 bits: what a training step keeps between forward and backward pass, in a quarter (float32) or half of its bytes.

``pack`` puts one tensor into 8 bits, ``saved_in_8_bits`` does so with what the ops inside it save for their backward pass: a
generator's layers, and the gradient that the losses of ``autograd`` compute with their value.  Blocks of 32 values share a scale
that is a power of two ("int8": errors of at most 1/128 of the block's largest magnitude, 1/64 next to it; "e4m3": of 1/16 of the value
itself, or 2^-17 of the block's largest where that is more: a small value may come back as 0); a value that is not finite comes back as NaN."""
from __future__ import annotations

import threading
from dataclasses import dataclass
from typing import Iterable

import torch

from . import binding as B

TYPES = (torch.float32, torch.bfloat16, torch.float16)


@dataclass
class Packed:
    """A tensor in 8 bits."""
    data: torch.Tensor           # uint8: the codes, then a byte per block of 32 for its scale
    format: str
    shape: torch.Size
    dtype: torch.dtype

    def unpack(self) -> torch.Tensor:
        """The values that stand for the tensor: contiguous, of its type, on its device."""
        out = B.native().unpacked(self.data, B._format(self.format), self.shape, self.dtype)
        if isinstance(out, int):
            raise B.DnError(out, "dn_unpack")
        return out


def pack(x: torch.Tensor, format: str = "int8") -> Packed:
    """x (CUDA, float32, bfloat16 or float16, any shape and strides) in 8 bits, in blocks of 32 along its elements in order."""
    data = B.native().packed(x, B._format(format))
    if isinstance(data, int):
        raise B.DnError(data, "dn_pack")
    return Packed(data, format, x.shape, x.dtype)


class _Saving(threading.local):
    """Set by gated_scan while it saves: the first tensor of numbers is its gate, which 8 bits hold as int8 in either format (an e4m3
    number is off relative to itself, and what counts of a gate of 7 is one minus its sigmoid), within +-63.5 (the sigmoid is 0 or 1
    to 2^-91 there; a mask of -1e4 would leave its neighbours steps of 64)."""
    gate = False


saving = _Saving()


class _Kept:
    """A saved tensor as it is: without its history, through which an op's saved output would hold the op and so itself, for good;
    with its version, which autograd looks at only where no hooks are."""

    def __init__(self, t: torch.Tensor):
        self.tensor, self.version = t.detach(), t._version

    def unpack(self) -> torch.Tensor:
        if self.tensor._version != self.version:
            raise RuntimeError(f"a saved tensor of shape {list(self.tensor.shape)}, kept as it is, has been modified in place: "
                               f"version {self.tensor._version} in place of {self.version}")
        return self.tensor


class saved_in_8_bits(torch.autograd.graph.saved_tensors_hooks):
    """Context in which the floating-point CUDA tensors that autograd saves are kept in 8 bits:

        with saved_in_8_bits(keep=generator.parameters()):
            loss = energy(generator(z), problem).mean()
        loss.backward()

    keep: tensors that stay as they are, views of them too (weights, which the gradient of the input multiplies with); so do
    tensors of less than ``min_numel`` elements, and expanded views whose memory is no more than 8 bits for each element.  They must not change before the backward pass, which raises RuntimeError if they
    have (an optimiser's step in between, say).  A gradient is then that of the ops at the values which 8 bits hold.  A tensor that
    several ops save is kept once for each of them.  The gate of ``autograd.gated_scan`` is kept as int8 in either format,
    held to +-63.5."""

    def __init__(self, format: str = "int8", keep: Iterable[torch.Tensor] = (), min_numel: int = 4096):
        B._format(format)
        self._keep, self._places = tuple(keep), frozenset()    # held: an address stands for its tensor only while that lives

        def put(t):
            gate = saving.gate and t.is_floating_point()
            if gate:
                saving.gate = False
            if not t.is_cuda or t.layout != torch.strided or t.dtype not in TYPES or t.numel() < min_numel:
                return _Kept(t)
            memory = t.untyped_storage()                   # of an expanded view: less than its elements
            if memory.data_ptr() in self._places or memory.nbytes() <= t.numel() + t.numel() // 32:
                return _Kept(t)
            return pack(t.detach().clamp(-63.5, 63.5), "int8") if gate else pack(t, format)

        super().__init__(put, lambda p: p.unpack())

    def __enter__(self):
        self._places = frozenset(k.untyped_storage().data_ptr() for k in self._keep if k.is_cuda)
        return super().__enter__()
