"""Adapters whose first call of a kind is captured: calls outside of the graph before its first replay, and the replay, are right."""
import pytest
import torch

from tests.gpu_util import DEV
from tests.test_gpu_lora import _adapters, _close, _problem, _reference, ctx  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [16, 128])
def test_first_call_captured_then_others(ctx, rows):  # noqa: F811
    from paper_2409_09099_b200.lora import LoraPlan
    p = _problem(1500, 2056, 320, 16, 3, 4, 20, seed=6, none=False)
    p["split"] = 2.0 ** -25
    want, room = _reference(p)
    lo, plan = _adapters(ctx, p, tile_rows=rows)
    small = LoraPlan([0, 40], [1], 1500, 3, tile_rows=rows)
    dirty = torch.full((1 << 26,), 0x55, dtype=torch.uint8, device=DEV)           # what fresh memory may hold
    del dirty
    y, d = torch.zeros_like(p["Y"]), torch.zeros_like(p["dX"])
    lo._grad_buffers()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        lo.forward(p["X"], p["Y"], plan, out=y)
        _, dA, dB = lo.backward(p["dY"], p["X"], p["dX"], plan, out=d)
    q = {**p, "ids": torch.full((1500,), -2, device=DEV)}
    q["ids"][:40] = 1
    few, few_room = _reference(q)
    for _ in range(2):
        out = lo.forward(p["X"], p["Y"], small, out=torch.zeros_like(y))           # outside, before the replay and after it
        _close(out[:40], few["Y"][:40], few_room["Y"][:40], "Y")
        _, a, b = lo.backward(p["dY"], p["X"], None, small)
        _close(a, few["dA"], few_room["dA"], "dA", 2.0 ** -24)
        _close(b, few["dB"], few_room["dB"], "dB", 2.0 ** -24)
        for _ in range(2):
            y.zero_(), d.zero_(), lo.V.zero_(), dA.fill_(7.0), dB.fill_(7.0)
            graph.replay()
            torch.cuda.synchronize()
            inside = p["ids"] > -2
            _close(y[inside], want["Y"][inside], room["Y"][inside], "Y")
            _close(d[inside], want["dX"][inside], room["dX"][inside], "dX")
            _close(dA, want["dA"], room["dA"], "dA", 2.0 ** -24)
            _close(dB, want["dB"], room["dB"], "dB", 2.0 ** -24)
