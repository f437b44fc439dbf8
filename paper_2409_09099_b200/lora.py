"""Low-rank adapters of many requests beside a shared linear (sste_lora_*): Y[t] += scale[a] B_a (A_a x_t), a the adapter of row t.

``LoraPlan`` says which rows of a batch use which adapter; it is made once per batch and serves every layer.  ``LoraAdapters`` holds the
adapters of one linear, an S-STE layer or any other, and the buffers of their forward and backward pass.  This is bookkeeping only;
every computation runs in libsste.
"""
from __future__ import annotations

import ctypes

import torch

from . import binding as B
from .checkpoint import ActivationCheckpoint

_bf16, _raw_stream = torch.bfloat16, torch._C._cuda_getCurrentRawStream
# attributes that the calls go by: setting one makes the next call look at all of them again
_HELD = frozenset(("ctx", "A", "B", "scale", "V"))


def _whole(v):
    i = int(v)
    if i != v:
        raise ValueError(f"{v!r} is not a whole number")
    return i


class LoraPlan:
    """The requests of a batch of T rows: rows offsets[i] .. offsets[i + 1] - 1 use adapters[i] (-1: none).

    ``offsets`` and ``adapters`` are host sequences (a scheduler has them there); rows outside them are padding, which reaches no result and
    is not written (it may be read).  ``replace`` puts another batch's requests in the place of these, for a graph that was captured with this plan: T, the rows
    per tile and the number of tiles (``min_tiles`` leaves room for more requests) stay, or it raises.  The new table is copied on the
    current stream: calls on other streams that still read the old one come before.
    """

    def __init__(self, offsets, adapters, T: int, n_adapters: int, device=0, tile_rows: int = 0, min_tiles: int = 0):
        self.T, self.n_adapters = T, n_adapters
        self.struct, table = self._build(offsets, adapters, tile_rows, min_tiles)
        self.tile_rows, self.n_tiles = self.struct.tile_rows, self.struct.n_tiles
        self.table = table.to(torch.device("cuda", device) if isinstance(device, int) else device)
        self.device = self.table.get_device()
        self.struct.table = self.table.data_ptr()
        self.at = ctypes.addressof(self.struct)

    def _build(self, offsets, adapters, tile_rows, min_tiles):
        offsets, adapters = [_whole(v) for v in offsets], [_whole(v) for v in adapters]
        return B.lora_plan_build(offsets, adapters, self.T, self.n_adapters, tile_rows, min_tiles)

    def replace(self, offsets, adapters):
        struct, table = self._build(offsets, adapters, self.tile_rows, self.n_tiles)
        if struct.n_tiles != self.n_tiles:
            raise ValueError(f"{struct.n_tiles} tiles do not fit the plan's {self.n_tiles}: make it with a larger min_tiles")
        self.table.copy_(table)


class LoraScratch:
    """Device scratch of adapters whose calls are stream-ordered among each other (the linears of one model): as large as the largest needs.

    It grows by half or more; a smaller one stays with those that have met it, for the graphs that were captured with it."""

    def __init__(self):
        self.room = None

    def at_least(self, n: int, device):
        """(a scratch of n bytes or more, whether it is there for other calls too)"""
        if self.room is not None and self.room.device != device:
            raise ValueError(f"the scratch is on {self.room.device}, the adapters are on {device}")
        if self.room is None or self.room.nbytes < n:
            with torch.cuda.device(-1 if device.index is None else device.index):        # (the stream of the adapters' device)
                capturing = torch.cuda.is_current_stream_capturing()
            if capturing:
                # zeros in a capture are recorded, not there: the call gets a scratch that only its graph has and empties at each replay
                return torch.zeros(n, dtype=torch.uint8, device=device), False
            self.room = torch.zeros(n if self.room is None else max(n, 3 * self.room.nbytes // 2), dtype=torch.uint8, device=device)
        return self.room, True


class LoraAdapters:
    """A [n, rank, I] and B [n, O, rank] (bf16) beside a linear of T rows, scale [n] (fp32, on the device).

    ``forward(X, Y, plan)`` adds the adapters' part to Y, the linear's output.  ``backward(dY, X, dX, plan)`` adds their part to dX, the
    linear's input gradient, and returns (dX, dA, dB); X is the forward's input or the ActivationCheckpoint that kept it.  ``V`` is what
    the forward leaves for the backward (``train=False``: nothing is left, for serving).  The calls of one object are stream-ordered:
    they share its scratch and result buffers; objects that are given one ``scratch`` share that, and all their calls are stream-ordered.
    After a call has timed out on the device the object, and a scratch that it shares, are to be made anew.
    """

    def __init__(self, ctx: B.Context, A: torch.Tensor, Bw: torch.Tensor, scale: torch.Tensor, T: int,
                 grad_dtype: torch.dtype = torch.float32, scratch: LoraScratch | None = None):
        n, r, I = A.shape
        if Bw.shape[0] != n or Bw.shape[2] != r or scale.shape != (n,):
            raise ValueError(f"A [n, rank, I], B [n, O, rank], scale [n]: got {tuple(A.shape)}, {tuple(Bw.shape)}, {tuple(scale.shape)}")
        if grad_dtype not in (torch.float32, torch.bfloat16):
            raise ValueError(f"gradients are fp32 or bf16: got {grad_dtype}")
        self.ctx, self.A, self.B, self.scale = ctx, A, Bw, scale
        self.n, self.rank, self.I, self.O, self.T = n, r, I, Bw.shape[1], T
        self.V = torch.empty((T, r), dtype=torch.float32, device=A.device)
        self._grad_dtype, self._grads = grad_dtype, None
        self._scratch, self._shared = {}, LoraScratch() if scratch is None else scratch
        self._x_shape, self._y_shape = torch.Size((T, I)), torch.Size((T, self.O))
        self.struct = B.LoraStruct(n, r, I, self.O)
        self.at = ctypes.addressof(self.struct)
        self._look()

    def __setattr__(self, name, value):
        d = self.__dict__
        if name in _HELD:
            d["_looked"] = False
        d[name] = value

    def _look(self):
        """Checks the weights and V and describes where they are.  (By the address alone another view of the same storage, or what the
        allocator has put in a freed one's place, would pass for the tensor that was there.)"""
        for t, shape, dtype in ((self.A, (self.n, self.rank, self.I), _bf16), (self.B, (self.n, self.O, self.rank), _bf16),
                                (self.scale, (self.n,), torch.float32), (self.V, (self.T, self.rank), torch.float32)):
            if t.shape != shape or t.dtype is not dtype or t.get_device() != self.ctx.device or not t.is_contiguous():
                raise ValueError(f"a contiguous {dtype} tensor of {shape} on cuda:{self.ctx.device} is wanted: got {t.dtype} {tuple(t.shape)} on {t.device}")
        s = self.struct
        s.A, s.B, s.scale, self._v_at = (t.data_ptr() for t in (self.A, self.B, self.scale, self.V))
        self._looked = True

    # (a few rows' calls are host time: the library is called from here, without the binding's marshalling)
    def _ready(self, plan):
        if plan.T != self.T or plan.n_adapters != self.n or plan.device != self.ctx.device:
            raise ValueError(f"the plan is for {plan.T} rows and {plan.n_adapters} adapters on cuda:{plan.device}, the adapters are for {self.T} "
                             f"and {self.n} on cuda:{self.ctx.device}")
        s = self.struct
        if (not self._looked or s.A != self.A.data_ptr() or s.B != self.B.data_ptr() or s.scale != self.scale.data_ptr()
                or self._v_at != self.V.data_ptr()):
            self._look()

    def _at(self, t, shape):
        """Address and row distance of a caller's tensor."""
        if t.dtype is not _bf16 or t.shape != shape:
            raise ValueError(f"a bf16 tensor of {tuple(shape)} is wanted: got {t.dtype} {tuple(t.shape)}")
        rows, step = t.stride()
        if t.get_device() != self.ctx.device or step != 1:
            raise ValueError(f"tensors of contiguous rows on cuda:{self.ctx.device} only")
        return t.data_ptr(), rows if self.T > 1 else shape[1]

    def _pair(self, base, out, shape):
        """Addresses of what is added to (None: zeros) and of the result, and their row distance."""
        at, ld = self._at(out, shape)
        if base is out or base is None:
            return at if base is out else None, at, ld
        base_at, base_ld = self._at(base, shape)
        if base_ld != ld:
            raise ValueError(f"the rows of the result are {ld} elements apart, those of what it is added to {base_ld}")
        return base_at, at, ld

    def _scratch_of(self, plan):
        # the calls of this object are stream-ordered, so that batches of all sizes share one
        key = plan.tile_rows, plan.n_tiles
        t = self._scratch.get(key)
        if t is None:
            t, there = self._shared.at_least(self.ctx.lib.sste_lora_scratch_bytes(self.at, plan.at), self.A.device)
            if there:
                self._scratch[key] = t
        return t

    @property
    def _room(self):
        return self._shared.room

    def forward(self, X, Y, plan: LoraPlan, out=None, train: bool = True):
        """Y (None: zeros) plus the adapters' part, in `out` (default: Y itself)."""
        out = Y if out is None else out
        if out is None:
            raise ValueError("without Y an `out` is wanted")
        self._ready(plan)
        x, ldx = self._at(X, self._x_shape)
        y_in, y, ldy = self._pair(Y, out, self._y_shape)
        ctx, scratch = self.ctx, self._scratch_of(plan)
        st = ctx.lib.sste_lora_fwd(ctx.handle, self.at, plan.at, x, ldx, y_in, y, ldy, self._v_at if train else None,
                                   scratch.data_ptr(), scratch.nbytes, _raw_stream(ctx.device))
        if st:
            ctx._check(st)
        return out

    def _grad_buffers(self):
        if self._grads is None:
            dev, dt = self.A.device, self._grad_dtype
            self._grads = torch.empty(self.A.shape, dtype=dt, device=dev), torch.empty(self.B.shape, dtype=dt, device=dev)
        return self._grads

    def backward(self, dY, X, dX, plan: LoraPlan, out=None):
        """(dX plus the adapters' part in `out` (default: dX itself), dA, dB).  dX None and out None: no input gradient."""
        dA, dB = self._grad_buffers()
        out = dX if out is None else out
        self._ready(plan)
        y, ldy = self._at(dY, self._y_shape)
        x, ldx, codes, scales, fmt = None, 0, None, None, 0
        if isinstance(X, ActivationCheckpoint):
            if X.shape != self._x_shape or X.act is not None:
                raise ValueError(f"a checkpoint of {tuple(self._x_shape)} without an activation is wanted: got {tuple(X.shape)}, {X.act}")
            if not X.ctx.device == X.codes.get_device() == X.scales.get_device() == self.ctx.device:
                raise ValueError(f"the checkpoint is of cuda:{X.ctx.device}, its codes on {X.codes.get_device()}, the adapters are on cuda:{self.ctx.device}")
            codes, scales, fmt = X.codes.data_ptr(), X.scales.data_ptr(), X._fmt
        else:
            x, ldx = self._at(X, self._x_shape)
        dx_in, dx, lddx = (None, None, 0) if out is None else self._pair(dX, out, self._x_shape)
        ctx, scratch = self.ctx, self._scratch_of(plan)
        st = ctx.lib.sste_lora_bwd(ctx.handle, self.at, plan.at, x, ldx, codes, scales, fmt, y, ldy, self._v_at, dx_in, dx, lddx,
                                   dA.data_ptr(), dB.data_ptr(), B._CODE_OF[self._grad_dtype], scratch.data_ptr(), scratch.nbytes,
                                   _raw_stream(ctx.device))
        if st:
            ctx._check(st)
        return out, dA, dB
