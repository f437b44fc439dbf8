"""Activations kept in 8 bits between the forward and the backward pass (sste_ckpt_*).

A layer that is trained keeps its input until grad_W = MVUE(grad_Z^T) X, and an MLP the inputs of its activation.  Kept in blocks of 32
elements with a shared power of two they take 8.25 bits an element, and what is restored is a bf16 number exactly, which the products
read like any other input.  This is bookkeeping only; every computation runs in libsste.
"""
from __future__ import annotations

import math

import torch

from . import binding as B

_bf16, _raw_stream = torch.bfloat16, torch._C._cuda_getCurrentRawStream
_FORMATS = {"e4m3": B.CKPT_E4M3, "int8": B.CKPT_INT8}
_ACTIVATIONS = {None: B.ACT_NONE, "gelu": B.ACT_GELU, "silu_gate": B.ACT_SILU_GATE}


class ActivationCheckpoint:
    """Room for one activation of `shape` in 8 bits: ``store`` in the forward, ``load`` or ``backward`` in the backward pass.

    ``act=None`` keeps a linear's input.  ``act="gelu"`` (tanh form) and ``act="silu_gate"`` (silu(x) * up) keep the inputs of the
    activation: ``store`` returns its output, ``backward`` the gradients and, with ``again=True``, the output once more, computed from
    the kept inputs: the next linear needs no checkpoint of its own.  ``fmt``: "int8" (error up to 1/127 of the block's maximum, at
    least 2^-125) or "e4m3" (up to 1/16 of each element, for those below 2^-13 of the block's maximum 2^-17 of that).  Results go to
    buffers that are made once and belong to this object; the next call of the same method overwrites them.
    """

    def __init__(self, ctx: B.Context, shape, fmt: str = "int8", act: str | None = None, device=None):
        if fmt not in _FORMATS or act not in _ACTIVATIONS:
            raise ValueError(f"fmt is one of {sorted(_FORMATS)}, act one of {list(_ACTIVATIONS)}: got {fmt!r}, {act!r}")
        self.ctx, self.shape, self.fmt, self.act = ctx, torch.Size(shape), fmt, act
        self.n = math.prod(self.shape)
        self._fmt, self._act, self._gate = _FORMATS[fmt], _ACTIVATIONS[act], act == "silu_gate"
        self.device = torch.device("cuda", ctx.device)
        if device is not None and torch.device(device) not in (self.device, torch.device("cuda")):
            raise ValueError(f"the context is on cuda:{ctx.device}, not on {device}")
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
        if fmt not in _FORMATS:
            raise ValueError(f"fmt is one of {sorted(_FORMATS)}: got {fmt!r}")
        self = cls.__new__(cls)
        self.ctx, self.shape, self.fmt, self.act = ctx, torch.Size(shape), fmt, None
        self.n, self._fmt, self._act, self._gate = math.prod(self.shape), _FORMATS[fmt], B.ACT_NONE, False
        blocks = (self.n + 31) // 32
        if (codes.dtype is not torch.uint8 or scales.dtype is not torch.uint8 or codes.numel() != 32 * blocks
                or scales.numel() != blocks or not (codes.is_contiguous() and scales.is_contiguous())
                or codes.get_device() != ctx.device or scales.get_device() != ctx.device):
            raise ValueError(f"{self.n} elements have {32 * blocks} bytes of codes and {blocks} of scales, contiguous on cuda:{ctx.device}")
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

    def _at(self, t):
        """Address of a caller's tensor, which has to be one of these activations.  (A small layer's calls are host time: the library is
        called from here, without the binding's marshalling.)"""
        if t.dtype is not _bf16 or t.shape != self.shape:
            raise ValueError(f"a bf16 tensor of {tuple(self.shape)} is wanted: got {t.dtype} {tuple(t.shape)}")
        if t.get_device() != self.ctx.device or not t.is_contiguous():
            raise ValueError(f"contiguous tensors on cuda:{self.ctx.device} only")
        return t.data_ptr()

    def _result(self, given, name):
        """A result's tensor and its address: the caller's, or a buffer, which needs no check."""
        if given is None:
            given = self._buffer(name)
            return given, given.data_ptr()
        return given, self._at(given)

    def _kept(self):
        if self._gate:
            return self.codes.data_ptr(), self.scales.data_ptr(), self.up_codes.data_ptr(), self.up_scales.data_ptr()
        return self.codes.data_ptr(), self.scales.data_ptr(), None, None

    def store(self, x, up=None, out=None):
        """Keeps x (and `up` of a gate); returns the activation's output (`out`, or a buffer), None without an activation."""
        if (up is not None) != self._gate:
            raise ValueError("`up` belongs to act='silu_gate'")
        if self._act == B.ACT_NONE:
            if out is not None:
                raise ValueError("without an activation there is no output")
            y_at = None
        else:
            if out is None:
                out = self._buffer("y")
            y_at = self._at(out)
        ctx = self.ctx
        st = ctx.lib.sste_ckpt_store(ctx.handle, self._at(x), None if up is None else self._at(up), self.n, B.BF16, self._fmt, self._act,
                                     *self._kept(), y_at, _raw_stream(ctx.device))
        if st:
            ctx._check(st)
        return out

    def load(self, out=None):
        """The kept values, or the activation's output computed from them."""
        if out is None:
            out = self._buffer("loaded")
        ctx = self.ctx
        st = ctx.lib.sste_ckpt_load(ctx.handle, *self._kept(), self.n, self._fmt, self._act, self._at(out), B.BF16, _raw_stream(ctx.device))
        if st:
            ctx._check(st)
        return out

    def backward(self, dy, again: bool = False, dx=None, dup=None, y=None):
        """(dx) or (dx, dup), and the activation's output once more if `again`: a tensor, or a tuple in this order.  They go to the tensors
        given (dx may be dy), or to buffers of this object."""
        if self._act == B.ACT_NONE:
            raise ValueError("without an activation there is no gradient: load()")
        if (dup is not None and not self._gate) or (y is not None and not again):
            raise ValueError("`dup` belongs to act='silu_gate', `y` to again=True")
        ctx, (dx, dx_at) = self.ctx, self._result(dx, "dx")
        dup, dup_at = self._result(dup, "dup") if self._gate else (None, None)
        y, y_at = self._result(y, "again") if again else (None, None)
        st = ctx.lib.sste_ckpt_act_bwd(ctx.handle, self._at(dy), *self._kept(), self.n, B.BF16, self._fmt, self._act, dx_at, dup_at, y_at,
                                       _raw_stream(ctx.device))
        if st:
            ctx._check(st)
        if self._gate:
            return (dx, dup, y) if again else (dx, dup)
        return (dx, y) if again else dx
