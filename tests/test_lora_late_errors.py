"""A backward call that is refused is refused before anything is launched: dX, which may be its own input, is as it was."""
import ctypes

import pytest
import torch

from paper_2409_09099_b200 import binding as B, build
from tests.test_ckpt_lora_checks import _call, _lora, _plan, lib, no_gpu  # noqa: F401


def test_more_steps_than_can_be_counted(lib, no_gpu):  # noqa: F811
    """2 (I + O) / 128 steps for each tile of 128 rows, counted in 31 bits; with the input's gradient alone there are none."""
    tiles, huge = (1 << 24) - 1, 1 << 24
    plan = _plan(T=2 ** 31 - 1, tile_rows=128, n_tiles=tiles)
    args = dict(ldx=huge, ldy=huge, lddx=huge, bytes=1 << 62)
    for rank, gdt in ((8, B.F32), (64, B.BF16), (64, B.F32)):
        lora = _lora(I=huge, O=huge, rank=rank)
        assert _call(lib, "bwd", lora, plan, gdt=gdt, **args) == B.ERR_SHAPE
        assert _call(lib, "bwd", lora, plan, dA=None, dB=None, **args) == B.ERR_CUDA          # as far as the device
        assert _call(lib, "fwd", lora, plan, **args) == B.ERR_CUDA
    # the last that can be: 2 (1 + 1) steps a tile, 2^24 - 1 tiles; at 64 blocks of features there are as many steps as 31 bits hold
    assert _call(lib, "bwd", _lora(I=128, O=128), plan, gdt=B.BF16, **args) == B.ERR_CUDA
    blocks = (2 ** 31 - 1) // (2 * tiles)
    for features, st in ((128 * (blocks - 1), B.ERR_CUDA), (128 * (blocks - 1) + 8, B.ERR_SHAPE)):
        assert _call(lib, "bwd", _lora(I=features, O=64), plan, **args) == st, features


@pytest.mark.gpu
def test_a_row_distance_that_no_copy_takes():
    """One row, so that nothing lies at the distance given: the call is refused for it or served, never half done."""
    dev = "cuda:0"
    ctx = B.Context(0)
    bf = lambda *shape: torch.ones(shape, dtype=torch.bfloat16, device=dev)
    A, Bw, scale = bf(1, 16, 128), bf(1, 64, 16), torch.ones(1, device=dev)
    plan, table = B.lora_plan_build([0, 1], [0], 1, 1, 128)
    table = table.to(dev)
    plan.table = table.data_ptr()
    lora = B.LoraStruct(1, 16, 128, 64, A.data_ptr(), Bw.data_ptr(), scale.data_ptr())
    l, p = ctypes.byref(lora), ctypes.byref(plan)
    scratch = torch.zeros(ctx.lib.sste_lora_scratch_bytes(l, p), dtype=torch.uint8, device=dev)
    X, dY, dX, V = bf(1, 128), bf(1, 64), bf(1, 128), torch.ones((1, 16), device=dev)
    dA, dB = torch.full((1, 16, 128), 7.0, device=dev), torch.full((1, 64, 16), 7.0, device=dev)
    for far in ((1 << 40, 64, 128), (128, 1 << 40, 128), (128, 64, 1 << 40)):
        dX.fill_(3.0)
        st = ctx.lib.sste_lora_bwd(ctx.handle, l, p, X.data_ptr(), far[0], None, None, 0, dY.data_ptr(), far[1], V.data_ptr(), dX.data_ptr(),
                                   dX.data_ptr(), far[2], dA.data_ptr(), dB.data_ptr(), B.F32, scratch.data_ptr(), scratch.nbytes, B._stream())
        torch.cuda.synchronize()
        if st == B.OK:
            assert bool((dX == torch.tensor(3.0 + 64 * 16).bfloat16().to(dev)).all()) and bool((dA == 64.0).all()) and bool((dB == 1.0).all())
        else:
            assert bool((dX == 3.0).all()) and bool((dA == 7.0).all()) and bool((dB == 7.0).all()), far
    ctx.close()
