"""The calls beside the linear allocate nothing on the device: what they need is the caller's."""
import pytest
import torch

from tests.test_gpu_lora import _adapters, _problem, ctx  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tile_rows", [16, 128])
def test_nothing_is_allocated(ctx, tile_rows):  # noqa: F811
    from paper_2409_09099_b200.checkpoint import ActivationCheckpoint
    p = _problem(1100, 1032, 520, 24, 3, 5, 9, seed=3, none=False)
    lo, plan = _adapters(ctx, p, tile_rows=tile_rows)
    kept, gate = (ActivationCheckpoint(ctx, p["X"].shape, "int8", act=a) for a in (None, "silu_gate"))
    y, d = torch.empty_like(p["Y"]), torch.empty_like(p["dX"])

    def calls():
        kept.store(p["X"]), kept.load()
        gate.store(p["X"], p["dX"]), gate.load(), gate.backward(p["dX"], again=True)
        lo.forward(p["X"], p["Y"], plan, out=y)
        lo.backward(p["dY"], p["X"], p["dX"], plan, out=d)
        lo.backward(p["dY"], kept, None, plan)

    calls()                                 # the first makes the driver load the kernels, and the objects their buffers
    torch.cuda.synchronize()
    free, held = torch.cuda.mem_get_info()[0], torch.cuda.memory_stats()["allocation.all.allocated"]
    for _ in range(3):
        calls()
    torch.cuda.synchronize()
    # free memory may rise if another process on a shared GPU releases some; it must not fall
    assert torch.cuda.mem_get_info()[0] >= free and torch.cuda.memory_stats()["allocation.all.allocated"] == held
