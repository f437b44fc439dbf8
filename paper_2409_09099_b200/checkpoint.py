"""Activations kept in 8 bits between the forward and the backward pass (sste_ckpt_*).

A layer that is trained keeps its input until grad_W = MVUE(grad_Z^T) X, and an MLP the inputs of its activation.  Kept in blocks of 32
elements with a shared power of two they take 8.25 bits an element, and what is restored is a bf16 number exactly, which the products
read like any other input.  This is bookkeeping only; every computation runs in libsste.
"""
from __future__ import annotations

import math

import torch

from . import binding as B

_FORMATS = {"e4m3": B.CKPT_E4M3, "int8": B.CKPT_INT8}
_ACTIVATIONS = {None: B.ACT_NONE, "gelu": B.ACT_GELU, "silu_gate": B.ACT_SILU_GATE}


class ActivationCheckpoint:
    """Room for one activation of `shape` in 8 bits: ``store`` in the forward, ``load`` or ``backward`` in the backward pass.

    ``act=None`` keeps a linear's input.  ``act="gelu"`` (tanh form) and ``act="silu_gate"`` (silu(x) * up) keep the inputs of the
    activation: ``store`` returns its output, ``backward`` the gradients and, with ``again=True``, the output once more, computed from
    the kept inputs: the next linear needs no checkpoint of its own.  ``fmt``: "int8" (error up to 1/252 of the block's maximum) or
    "e4m3" (up to 1/16 of each element).  Results go to buffers that are made once and belong to this object; the next call of the
    same method overwrites them.
    """

    def __init__(self, ctx: B.Context, shape, fmt: str = "int8", act: str | None = None, device=None):
        if fmt not in _FORMATS or act not in _ACTIVATIONS:
            raise ValueError(f"fmt is one of {sorted(_FORMATS)}, act one of {list(_ACTIVATIONS)}: got {fmt!r}, {act!r}")
        self.ctx, self.shape, self.fmt, self.act = ctx, torch.Size(shape), fmt, act
        self.n = math.prod(self.shape)
        self._fmt, self._act, self._gate = _FORMATS[fmt], _ACTIVATIONS[act], act == "silu_gate"
        self.device = torch.device(f"cuda:{ctx.device}" if device is None else device)
        blocks = (self.n + 31) // 32

        def kept():
            return (torch.empty(32 * blocks, dtype=torch.uint8, device=self.device),
                    torch.empty(blocks, dtype=torch.uint8, device=self.device))

        self.codes, self.scales = kept()
        self.up_codes, self.up_scales = kept() if self._gate else (None, None)
        self._out = {}

    @classmethod
    def of(cls, ctx: B.Context, codes, scales, shape, fmt: str):
        """A checkpoint (without activation) whose codes and scales are there already."""
        self = cls.__new__(cls)
        self.ctx, self.shape, self.fmt, self.act = ctx, torch.Size(shape), fmt, None
        self.n, self._fmt, self._act, self._gate = math.prod(self.shape), _FORMATS[fmt], B.ACT_NONE, False
        blocks = (self.n + 31) // 32
        if (codes.dtype is not torch.uint8 or scales.dtype is not torch.uint8 or codes.numel() != 32 * blocks
                or scales.numel() != blocks):
            raise ValueError(f"{self.n} elements have {32 * blocks} bytes of codes and {blocks} of scales")
        self.device, self.codes, self.scales, self.up_codes, self.up_scales = codes.device, codes, scales, None, None
        self._out = {}
        return self

    @property
    def nbytes(self) -> int:
        """Device memory that waits for the backward pass."""
        return sum(t.nbytes for t in (self.codes, self.scales, self.up_codes, self.up_scales) if t is not None)

    def _buffer(self, name):
        t = self._out.get(name)
        if t is None:
            t = self._out[name] = torch.empty(self.shape, dtype=torch.bfloat16, device=self.device)
        return t

    def _check(self, *tensors):
        for t in tensors:
            if t.shape != self.shape or t.dtype is not torch.bfloat16:
                raise ValueError(f"a bf16 tensor of {tuple(self.shape)} is wanted: got {t.dtype} {tuple(t.shape)}")

    def store(self, x, up=None, out=None):
        """Keeps x (and `up` of a gate); returns the activation's output (`out`, or a buffer), None without an activation."""
        if (up is not None) != self._gate:
            raise ValueError("`up` belongs to act='silu_gate'")
        self._check(x, *(() if up is None else (up,)), *(() if out is None else (out,)))
        if out is not None and self.act is None:
            raise ValueError("without an activation there is no output")
        y = None if self.act is None else self._buffer("y") if out is None else out
        self.ctx.ckpt_store(x, self.codes, self.scales, self._fmt, self._act, up, self.up_codes, self.up_scales, y)
        return y

    def load(self, out=None):
        """The kept values, or the activation's output computed from them."""
        y = self._buffer("loaded") if out is None else out
        self._check(y)
        self.ctx.ckpt_load(self.codes, self.scales, y, self._fmt, self._act, self.up_codes, self.up_scales)
        return y

    def backward(self, dy, again: bool = False):
        """(dx) or (dx, dup), and the activation's output once more if `again`: a tensor, or a tuple in this order."""
        if self.act is None:
            raise ValueError("without an activation there is no gradient: load()")
        self._check(dy)
        dx, dup = self._buffer("dx"), self._buffer("dup") if self._gate else None
        y = self._buffer("again") if again else None
        self.ctx.ckpt_act_bwd(dy, self.codes, self.scales, dx, self._fmt, self._act, self.up_codes, self.up_scales, dup, y)
        out = tuple(t for t in (dx, dup, y) if t is not None)
        return out if len(out) > 1 else dx
