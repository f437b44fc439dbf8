"""The decoder with its activations kept in 8 bits and with low-rank adapters: what each linear's backward works on, and its gradients."""
import math

import pytest
import torch

from tests.gpu_util import DEV

pytestmark = pytest.mark.gpu

SMALL = dict(n_layer=2, d=128, n_head=2, d_ff=512, seq=128, batch=2, vocab=640)


def _model(ctx, **kw):
    from paper_2409_09099_b200.model import SsteGpt2, synthetic_batch
    m = SsteGpt2(ctx, **SMALL, **kw)
    return m, synthetic_batch(m, 4)


@pytest.fixture(scope="module")
def ctx():
    from paper_2409_09099_b200 import binding as B
    c = B.Context(0)
    yield c
    assert c.poll_device_status() == 0
    c.close()


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_kept_activations_in_training(ctx, fmt, monkeypatch):
    """Same forward; each linear's weight gradient is the product of its sparsified gradient with the kept form of its input."""
    from paper_2409_09099_b200.checkpoint import ActivationCheckpoint
    plain, batch = _model(ctx)
    want, _ = plain.train_step(*batch)
    m, _ = _model(ctx, checkpoint=fmt)
    stored, store = {}, ActivationCheckpoint.store
    monkeypatch.setattr(ActivationCheckpoint, "store", lambda self, x, up=None, out=None: (stored.__setitem__(id(self), x.clone()),
                                                                                          store(self, x, up, out))[1])
    seen = set()

    def check(index, step, lin, x, dy):
        seen.add(index)
        owner = m.linears[index]
        again = ActivationCheckpoint(ctx, owner.kept.shape, fmt, act=owner.kept.act)
        store(again, stored[id(owner.kept)], None, None)
        assert torch.equal(again.load(), x) and owner.x is None
        dw = torch.empty_like(lin.dW)
        ctx.linear_bwd_weight(lin.gvals, lin.gmeta, x, dw)
        off = (dw.float() - lin.dW.float()).norm() / dw.float().norm()
        assert off <= 2.0 ** -7                                       # one launch for both products may split the sum otherwise

    m.on_call = check
    loss, _ = m.train_step(*batch)
    assert seen == set(range(8))
    # the forward does not look at the kept values (GELU here is one bf16 rounding of fp32, as torch's)
    assert abs(float(loss) - float(want)) <= 2.0 ** -8 * float(want)
    assert sum(s.kept.nbytes for s in m.linears) < 0.52 * sum(2 * s.lin.T * s.lin.I for s in m.linears)
    loss, _ = m.train_step(*batch)
    assert math.isfinite(float(loss))


@pytest.mark.parametrize("checkpoint", [None, "int8"])
def test_adapters_in_training(ctx, checkpoint):
    """The adapters' gradients against 64 bits on the tensors that the model fed them; their B starts at zero, so the first forward is the plain one."""
    plain, batch = _model(ctx)
    want, _ = plain.train_step(*batch)
    m, _ = _model(ctx, checkpoint=checkpoint, adapter_rank=8)
    # (the adapters' random numbers come between the others: the same masters for the comparison)
    with torch.no_grad():
        for a, b in zip(m.linears, _model(ctx)[0].linears):
            a.w.copy_(b.w)
        fresh = _model(ctx)[0]
        m.wte.copy_(fresh.wte)
        m.wpe.copy_(fresh.wpe)
    loss, _ = m.train_step(*batch)
    assert abs(float(loss) - float(want)) <= 2.0 ** -8 * float(want)
    calls = {}
    m.on_call = lambda index, step, lin, x, dy: calls.__setitem__(index, (x.clone(), dy.clone()))
    loss, _ = m.train_step(*batch)
    assert math.isfinite(float(loss)) and set(calls) == set(range(8))
    for index, (x, dy) in calls.items():
        s = m.linears[index]
        A, Bw, X, dY = s.lora.A[0].double(), s.lora.B[0].double(), x.double(), dy.double()
        T, O, I = s.lin.T, s.lin.O, s.lin.I
        # V is of the input itself, X of dA may be the kept form: V from the adapter's own record
        V = s.lora.V.double()
        dA, dB = 2 * (dY @ Bw).t() @ X, dY.t() @ V
        room = 2.0 ** -16 + (T + O) * 2.0 ** -23
        mA, mB = 2 * (dY.abs() @ Bw.abs()).t() @ X.abs(), dY.abs().t() @ V.abs()
        assert bool(((s.a.grad[0].double() - dA).abs() <= room * mA + 1e-30).all()), index
        assert bool(((s.bt.grad[0].double() - dB).abs() <= room * mB + 1e-30).all()), index
        assert bool(s.bt.grad.any()) and bool(s.a.grad.any())
