"""ActivationCheckpoint.backward into tensors of the caller's: the same values as in its own buffers, none of which is made."""
import pytest
import torch

from tests.gpu_util import DEV
from tests.test_gpu_ckpt import _act_inputs, ctx  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("n", [33, 10007])
def test_given_tensors(ctx, n, fmt):  # noqa: F811
    from paper_2409_09099_b200.checkpoint import ActivationCheckpoint
    x, dy = _act_inputs(n, n, False)
    u = _act_inputs(n, n + 1, False)[0]
    new = lambda: torch.full_like(x, 7.0)
    for act, up in (("gelu", None), ("silu_gate", u)):
        own, k = (ActivationCheckpoint(ctx, x.shape, fmt, act=act) for _ in range(2))
        own.store(x, up), k.store(x, up, out=new())
        want = [t.clone() for t in own.backward(dy, again=True)]
        given = dict(dx=new(), y=new(), **(dict(dup=new()) if up is not None else {}))
        got = k.backward(dy, again=True, **given)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert got[0] is given["dx"] and got[-1] is given["y"] and (up is None or got[1] is given["dup"]) and not k._out
        g = dy.clone()                                          # in the gradient's place
        got = k.backward(g, dx=g, **(dict(dup=new()) if up is not None else {}))
        assert torch.equal(g, want[0]) and not k._out


def test_refusals(ctx):  # noqa: F811
    from paper_2409_09099_b200.checkpoint import ActivationCheckpoint
    x, dy = _act_inputs(256, 1, False)
    k, g = ActivationCheckpoint(ctx, x.shape, "int8", act="gelu"), ActivationCheckpoint(ctx, x.shape, "int8", act="silu_gate")
    k.store(x), g.store(x, x)
    for call in (lambda: k.backward(dy, dup=torch.empty_like(x)), lambda: k.backward(dy, y=torch.empty_like(x)),
                 lambda: k.backward(dy, dx=x[:128]), lambda: k.backward(dy, dx=x.float()), lambda: k.backward(dy, dx=x.cpu()),
                 lambda: g.backward(dy, dup=x[:3]), lambda: g.backward(dy, again=True, y=torch.empty((512,), dtype=x.dtype, device=DEV)[::2])):
        with pytest.raises(ValueError):
            call()


def test_calls_of_the_context_look_at_sizes(ctx):  # noqa: F811
    """Codes, scales and outputs that are too short, or of another type, are not written past."""
    from paper_2409_09099_b200 import binding as B
    from paper_2409_09099_b200.checkpoint import ActivationCheckpoint
    x, dy = _act_inputs(257, 1, False)
    g = ActivationCheckpoint(ctx, x.shape, "int8", act="silu_gate")
    y, dx, dup = (torch.empty_like(x) for _ in range(3))
    store = dict(x=x, codes=g.codes, scales=g.scales, fmt=g._fmt, act=g._act, up=x, up_codes=g.up_codes, up_scales=g.up_scales, y=y)
    load = dict(codes=g.codes, scales=g.scales, y=y, fmt=g._fmt, act=g._act, up_codes=g.up_codes, up_scales=g.up_scales)
    back = dict(dy=dy, codes=g.codes, scales=g.scales, dx=dx, fmt=g._fmt, act=g._act, up_codes=g.up_codes, up_scales=g.up_scales, dup=dup, y=y)
    for call, args in ((ctx.ckpt_store, store), (ctx.ckpt_load, load), (ctx.ckpt_act_bwd, back)):
        call(**args)
        before = B.launch_count()
        for name, short in (("codes", g.codes[:256]), ("scales", g.scales[:8]), ("up_codes", g.up_codes[:256]), ("up_scales", g.up_scales[:8])) + (
                (("up", x[:256]), ("y", y[:256]), ("y", y.float())) if call == ctx.ckpt_store else
                (("dx", dx[:256]), ("dup", dup[:256]), ("y", y.float())) if call == ctx.ckpt_act_bwd else ()):
            with pytest.raises(AssertionError):
                call(**{**args, name: short})
        assert B.launch_count() == before
