"""What LoraAdapters holds its tensors to, on the host: nothing here is launched, the library is replaced by a stand-in that counts calls.

The tensors lie in host memory, whose device index is -1, and so does the context's.
"""
import types

import pytest
import torch

from paper_2409_09099_b200 import binding as B, build

T, I, O, R, N = 20, 64, 96, 16, 3


class _Library:
    """As far as LoraAdapters looks: a scratch size, and calls that do nothing."""

    def __init__(self):
        self.calls = []

    def sste_lora_scratch_bytes(self, lora, plan):
        return 4096

    def sste_lora_fwd(self, *args):
        self.calls.append(args)
        return 0

    sste_lora_bwd = sste_lora_fwd


@pytest.fixture(autouse=True)
def stand_in(monkeypatch):
    build.build()
    from paper_2409_09099_b200 import lora
    monkeypatch.setattr(lora, "_raw_stream", lambda device: 0)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    return lora


def _context():
    ctx = types.SimpleNamespace(device=-1, lib=_Library(), handle=None)
    ctx._check = lambda st: pytest.fail(f"status {st}")
    return ctx


def _bf16(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def _adapters(lora, ctx=None):
    lo = lora.LoraAdapters(ctx or _context(), _bf16(N, R, I), _bf16(N, O, R), torch.ones(N), T)
    return lo, lora.LoraPlan([0, T], [0], T, N, device="cpu")


def test_other_views_of_the_same_storage_are_refused(stand_in):
    """Same address, other layout, shape or type: none of it is computed with the old layout."""
    for name in ("A", "B", "scale", "V"):
        lo, plan = _adapters(stand_in)
        old = getattr(lo, name)
        wide = torch.zeros((2,) + tuple(old.shape), dtype=old.dtype).flatten()
        views = [old[:2], old.view(torch.float16 if old.dtype is torch.bfloat16 else torch.int32), old[None],
                 torch.as_strided(wide, old.shape, [2 * s for s in old.stride()])]
        if old.dim() == 3:
            views += [old.transpose(1, 2), old[:, :, ::2], old[:, ::2], old.view(torch.float32)]
        for t in views:
            setattr(lo, name, t)
            with pytest.raises(ValueError):
                lo.forward(_bf16(T, I), _bf16(T, O), plan)
            with pytest.raises(ValueError):
                lo.backward(_bf16(T, O), _bf16(T, I), _bf16(T, I), plan)
        assert not lo.ctx.lib.calls
        setattr(lo, name, old)                                  # the right one again
        lo.forward(_bf16(T, I), _bf16(T, O), plan)
        setattr(lo, name, old.clone())                          # another of the same kind
        lo.forward(_bf16(T, I), _bf16(T, O), plan)
        lo.backward(_bf16(T, O), _bf16(T, I), _bf16(T, I), plan)
        assert len(lo.ctx.lib.calls) == 3
        assert (lo.struct.A, lo.struct.B, lo.struct.scale) == (lo.A.data_ptr(), lo.B.data_ptr(), lo.scale.data_ptr())
        assert lo.ctx.lib.calls[-1][10] == lo.V.data_ptr()


def test_weights_whose_storage_moves_are_looked_at_again(stand_in):
    lo, plan = _adapters(stand_in)
    lo.A.data = torch.ones(N, R, I).bfloat16()                  # the tensor object stays
    lo.forward(_bf16(T, I), _bf16(T, O), plan)
    assert lo.struct.A == lo.A.data_ptr()
    lo.A.data = torch.ones(N, R, I + 8).bfloat16()
    with pytest.raises(ValueError):
        lo.forward(_bf16(T, I), _bf16(T, O), plan)


def test_a_scratch_first_met_in_a_capture_is_its_graphs_own(stand_in, monkeypatch):
    """What is zeroed inside a capture is not zero outside of it: nothing of it is kept for other calls."""
    lo, plan = _adapters(stand_in)
    x, y = _bf16(T, I), _bf16(T, O)
    scratch = lambda: lo.ctx.lib.calls[-1][9:11]
    capturing = [True]
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: capturing[0])
    lo.forward(x, y, plan)
    assert scratch()[1] == 4096 and not lo._scratch and lo._room is None
    capturing[0] = False
    lo.forward(x, y, plan)
    own, room = scratch(), lo._room
    assert room is not None and not bool(room.any()) and own == (room.data_ptr(), 4096)
    capturing[0] = True
    lo.forward(x, y, plan)                                      # one that is there already serves a capture as well
    assert scratch() == own
    lo.ctx.lib.sste_lora_scratch_bytes = lambda lora, plan: 100000
    larger = stand_in.LoraPlan([0, T], [0], T, N, device="cpu", tile_rows=128)
    lo.forward(x, y, larger)                                    # and stays when a capture needs a larger one
    assert scratch()[1] == 100000 and lo._room is room and list(lo._scratch) == [(plan.tile_rows, plan.n_tiles)]


def test_a_checkpoint_of_another_device_is_refused(stand_in):
    """Its codes are addresses there: nothing here may read through them."""
    from paper_2409_09099_b200.checkpoint import ActivationCheckpoint
    lo, plan = _adapters(stand_in)
    here = ActivationCheckpoint.of(lo.ctx, torch.zeros(T * I, dtype=torch.uint8), torch.zeros(T * I // 32, dtype=torch.uint8), (T, I), "int8")
    lo.backward(_bf16(T, O), here, _bf16(T, I), plan)
    there = ActivationCheckpoint.of(lo.ctx, here.codes, here.scales, (T, I), "int8")
    there.ctx = types.SimpleNamespace(device=1)
    with pytest.raises(ValueError):
        lo.backward(_bf16(T, O), there, _bf16(T, I), plan)
    there.ctx = lo.ctx
    for name in ("codes", "scales"):
        moved = ActivationCheckpoint.of(lo.ctx, here.codes, here.scales, (T, I), "int8")
        setattr(moved, name, types.SimpleNamespace(get_device=lambda: 1, data_ptr=lambda: 1 << 20))
        with pytest.raises(ValueError):
            lo.backward(_bf16(T, O), moved, _bf16(T, I), plan)
    assert len(lo.ctx.lib.calls) == 1


def test_a_shared_scratch_of_another_device_is_refused(stand_in):
    shared = stand_in.LoraScratch()
    shared.room = torch.zeros(1 << 20, dtype=torch.uint8, device="meta")
    lo, plan = _adapters(stand_in)
    lo._shared = shared
    with pytest.raises(ValueError):
        lo.forward(_bf16(T, I), _bf16(T, O), plan)
    assert not lo.ctx.lib.calls


def test_objects_that_share_a_scratch(stand_in):
    ctx, shared = _context(), stand_in.LoraScratch()
    plan = stand_in.LoraPlan([0, T], [0], T, N, device="cpu")
    objects = [stand_in.LoraAdapters(ctx, _bf16(N, R, I), _bf16(N, O, R), torch.ones(N), T, scratch=shared) for _ in range(3)]
    for size, lo in zip((4096, 2048, 5000), objects):
        ctx.lib.sste_lora_scratch_bytes = lambda lora, plan, size=size: size
        lo.forward(_bf16(T, I), _bf16(T, O), plan)
    for lo in objects:
        lo.forward(_bf16(T, I), _bf16(T, O), plan)
    at = [c[9:11] for c in ctx.lib.calls]
    assert at[:3] == at[3:] and at[0] == at[1] and at[2] == (shared.room.data_ptr(), 6144)


def test_the_capture_is_that_of_the_adapters_device(stand_in, monkeypatch):
    """Another device may be current, whose stream is not captured."""
    current = [0]

    class Device:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            self.was, current[0] = current[0], self.index

        def __exit__(self, *args):
            current[0] = self.was

    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: current[0] == 1)
    monkeypatch.setattr(torch, "zeros", lambda n, dtype, device: types.SimpleNamespace(nbytes=n, device=device))
    scratch = stand_in.LoraScratch()
    assert scratch.at_least(512, torch.device("cuda", 1))[1] is False and scratch.room is None
    assert scratch.at_least(512, torch.device("cuda", 0))[1] is True and scratch.room.nbytes == 512
