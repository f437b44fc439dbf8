"""The adapters' calls of Context itself: the weights that the object has now, and tensors of the sizes that the kernels go by."""
import pytest
import torch

from tests.gpu_util import DEV
from tests.test_gpu_lora import _adapters, _problem, ctx  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tile_rows", [16, 128])
def test_as_the_class(ctx, tile_rows):  # noqa: F811
    p = _problem(200, 72, 136, 16, 3, 4, 7, seed=1, none=False)
    lo, plan = _adapters(ctx, p, tile_rows=tile_rows)
    old = lo.A, lo.B, lo.scale
    for change in (lambda: None, lambda: [setattr(lo, k, getattr(lo, k) * 2) for k in ("A", "B", "scale")]):
        change()
        want = lo.forward(p["X"], p["Y"], plan, out=torch.zeros_like(p["Y"])).clone(), lo.V.clone()
        want += tuple(t.clone() for t in lo.backward(p["dY"], p["X"], p["dX"], plan, out=torch.zeros_like(p["dX"])))
    lo.A, lo.B, lo.scale = old
    lo._ready(plan)
    for k, t in zip(("A", "B", "scale"), old):
        setattr(lo, k, t * 2)
    y, dx, V, scratch = torch.zeros_like(p["Y"]), torch.zeros_like(p["dX"]), torch.full_like(lo.V, 7.0), lo._scratch_of(plan)
    dA, dB = (torch.empty_like(t, dtype=torch.float32) for t in (lo.A, lo.B))
    ctx.lora_fwd(lo, plan, p["X"], p["Y"], y, V, scratch)
    ctx.lora_bwd(lo, plan, p["X"], None, p["dY"], V, p["dX"], dx, dA, dB, scratch)
    assert all(torch.equal(a, b) for a, b in zip((y, V, dx, dA, dB), want))


def test_refusals(ctx):  # noqa: F811
    from paper_2409_09099_b200.checkpoint import ActivationCheckpoint
    p = _problem(200, 72, 136, 16, 3, 4, 7, seed=1, none=False)
    lo, plan = _adapters(ctx, p)
    scratch, X, Y, dY, dX, V = lo._scratch_of(plan), p["X"], p["Y"], p["dY"], p["dX"], lo.V
    dA, dB = lo._grad_buffers()
    launches = __import__("paper_2409_09099_b200.binding", fromlist=["launch_count"]).launch_count
    before = launches()
    for args in ((X[:100], Y, Y, V), (X, Y[:100], Y, V), (X, None, Y[:, :72], V), (X.float(), Y, Y, V), (X, Y, Y, V[:100]), (X, Y, Y, V[:, :8].contiguous()),
                 (X, Y, Y, V.bfloat16())):
        with pytest.raises(AssertionError):
            ctx.lora_fwd(lo, plan, *args, scratch)
    act, wide = ActivationCheckpoint(ctx, (200, 72), "int8", act="gelu"), ActivationCheckpoint(ctx, (200, 136), "int8")
    good = dict(X=X, kept=None, dY=dY, V=V, dX_in=dX, dX_out=dX, dA=dA, dB=dB)
    for name, bad in (("X", X[:, :64]), ("dY", dY[:100]), ("V", V[:100]), ("dX_in", dX[:100]), ("dA", dA[:2]), ("dB", dB.bfloat16()), ("dA", None),
                      ("kept", act), ("kept", wide)):
        with pytest.raises(AssertionError):
            ctx.lora_bwd(lo, plan, **{**good, name: bad, **({"X": None} if name == "kept" else {})}, scratch=scratch)
    lo.A = torch.empty((3, 16, 64), dtype=torch.bfloat16, device=DEV)
    with pytest.raises(ValueError):
        ctx.lora_fwd(lo, plan, X, Y, Y, V, scratch)
    assert launches() == before
