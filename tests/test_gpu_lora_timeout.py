"""A bounded wait of the adapters' kernels that runs out: the call returns, the status word says so, and the next calls are right.

The hook leaves the last step of each block unloaded, a barrier that nothing completes, and limits the waits to a millisecond.  Nothing here
faults, traps or spins.
"""
import pytest
import torch

from tests.test_gpu_lora import _problem

pytestmark = pytest.mark.gpu

# blocks alone, in pairs and in fours; one step of K and more than the ring holds; part tiles
SIZES = [(9600, 64, 72, 16), (9600, 1280, 200, 64), (1500, 1280, 520, 32), (300, 2056, 1288, 64)]


@pytest.mark.parametrize("kept", [None, "int8", "e4m3"])
@pytest.mark.parametrize("kernel", [1, 2])
@pytest.mark.parametrize("T,I,O,r", SIZES)
def test_expired_waits(T, I, O, r, kernel, kept):
    from paper_2409_09099_b200 import binding as B
    from paper_2409_09099_b200.checkpoint import ActivationCheckpoint
    from paper_2409_09099_b200.lora import LoraAdapters, LoraPlan
    ctx = B.Context(0)
    p = _problem(T, I, O, r, 3, 5, 9, seed=r, none=False)
    X = p["X"]
    if kept:
        X = ActivationCheckpoint(ctx, (T, I), kept)
        X.store(p["X"])
    plan = LoraPlan(p["bounds"], p["adapters"], T, 3, tile_rows=128)

    def run(dtype, forward=True):
        lo = LoraAdapters(ctx, p["A"], p["B"], p["scale"], T, grad_dtype=dtype)      # (with a scratch that is zero)
        lo.V.fill_(1.0)
        y = lo.forward(p["X"], p["Y"], plan, out=torch.zeros_like(p["Y"])) if forward else None
        return [t.clone() for t in (y, *lo.backward(p["dY"], X, p["dX"], plan, out=torch.zeros_like(p["dX"]))) if t is not None]

    for dtype in (torch.float32, torch.bfloat16):
        want = run(dtype)
        torch.cuda.synchronize()
        assert ctx.poll_device_status() == B.OK
        ctx.debug_lora_stall(kernel)
        try:
            run(dtype, forward=kernel == 1)
            torch.cuda.synchronize()                             # the kernels have returned
        finally:
            ctx.debug_lora_stall(0)
        assert ctx.poll_device_status() == B.ERR_TIMEOUT
        assert ctx.poll_device_status() == B.OK
        assert all(torch.equal(a, b) for a, b in zip(run(dtype), want))
    assert ctx.poll_device_status() == B.OK
    ctx.close()


def test_the_hook_knows_two_kernels():
    from paper_2409_09099_b200 import binding as B
    lib = B.load()
    assert lib.sste_debug_lora_stall(3) == B.ERR_INVALID_ARG and lib.sste_debug_lora_stall(-1) == B.ERR_INVALID_ARG
    assert lib.sste_debug_lora_stall(0) == B.OK
