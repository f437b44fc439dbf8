"""The operators beside the linear, each input written by a kernel of the library right in front of the call, with the queue backed up.

The adapters' expansion of few rows reads its weights, its table and what it adds to before the projection in front of it is done: that
started behind everything before it.  So these are the inputs that must not be read too early.
"""
import pytest
import torch

from paper_2409_09099_b200 import binding as B
from paper_2409_09099_b200.layer import SsteLinear
from paper_2409_09099_b200.lora import LoraAdapters, LoraPlan
from tests.test_gpu_kernel_order import BF, U8, _Tail, _empty, ctx  # noqa: F401

pytestmark = pytest.mark.gpu

N, R = 3, 16


def _adapter_calls(ctx, T, I, O, tile_rows, grad_dtype):
    """name -> (inputs, stale inputs, call)"""
    gen = torch.Generator(device="cuda").manual_seed(T)
    rnd = lambda *shape, s=1.0: _empty(shape, BF).normal_(0.0, s, generator=gen)
    bounds = [0, T // 3, T // 2, T - 8]
    plan, other = (LoraPlan(bounds, a, T, N, tile_rows=tile_rows) for a in ([1, 0, 2], [2, 1, 0]))
    assert plan.n_tiles == other.n_tiles
    weights = dict(A=rnd(N, R, I, s=I ** -0.5), B=rnd(N, O, R, s=0.1), scale=torch.tensor([1.5, 0.5, 2.0], device="cuda"), table=plan.table)
    objects = {}

    def lora_of(d):
        key = tuple(t.data_ptr() for t in d.values())
        if key not in objects:
            lo = LoraAdapters(ctx, d["A"], d["B"], d["scale"], T, grad_dtype=grad_dtype)
            p = LoraPlan(bounds, [1, 0, 2], T, N, tile_rows=tile_rows)
            p.table = d["table"]
            p.struct.table = d["table"].data_ptr()
            if "V" in d:
                lo.V = d["V"]
            lo._scratch_of(p), lo._grad_buffers()
            objects[key] = lo, p, _empty((T, O), BF), _empty((T, I), BF)
        return objects[key]

    def forward(d):
        lo, p, out, _ = lora_of(d)
        lo.forward(d["X"], d["Y"], p, out=out)
        return out[:T - 8], lo.V[:T - 8]

    def in_place(d):
        lo, p, _, _ = lora_of(d)
        lo.forward(d["X"], d["Y"], p, train=False)
        return (d["Y"],)

    def backward(d):
        lo, p, _, out = lora_of(d)
        return (lo.backward(d["dY"], d["X"], d["dX"], p, out=out)[0][:T - 8], *lo._grad_buffers())

    X, Y, dY, dX = rnd(T, I), rnd(T, O), rnd(T, O, s=0.01), rnd(T, I, s=0.01)
    V = torch.randn((T, R), device="cuda", generator=gen)
    tag = f"{tile_rows} rows, {grad_dtype}: "
    return {tag + "forward": (dict(weights, X=X, Y=Y), dict(table=other.table), forward),
            tag + "in place": (dict(weights, X=X, Y=Y), dict(table=other.table), in_place),
            tag + "backward": (dict(weights, X=X, dY=dY, dX=dX, V=V), dict(table=other.table), backward)}


def _kept_calls(ctx, fmt):
    n = 1 << 20
    gen = torch.Generator(device="cuda").manual_seed(fmt)
    x, up, dy = (_empty((n,), BF).normal_(0.0, 1.0, generator=gen) for _ in range(3))
    new = lambda: (_empty((n,), U8), _empty((n // 32,), U8))
    (codes, scales), (uc, us) = new(), new()
    ctx.ckpt_store(x, codes, scales, fmt)
    ctx.ckpt_store(up, uc, us, fmt)

    def store(d):
        (c, s), (e, t), y = new(), new(), _empty((n,), BF)
        ctx.ckpt_store(d["x"], c, s, fmt, B.ACT_SILU_GATE, d["up"], e, t, y)
        return c, s, e, t, y

    def load(d):
        y = _empty((n,), BF)
        ctx.ckpt_load(d["codes"], d["scales"], y, fmt, B.ACT_SILU_GATE, d["uc"], d["us"])
        return (y,)

    def backward(d):
        dx, dup, y = (_empty((n,), BF) for _ in range(3))
        ctx.ckpt_act_bwd(d["dy"], d["codes"], d["scales"], dx, fmt, B.ACT_SILU_GATE, d["uc"], d["us"], dup, y)
        return dx, dup, y

    kept = dict(codes=codes, scales=scales, uc=uc, us=us)
    tag = f"format {fmt}: "
    return {tag + "store": (dict(x=x, up=up), {}, store), tag + "load": (kept, {}, load), tag + "backward": (dict(kept, dy=dy), {}, backward)}


def _all_calls(ctx):
    calls = {}
    for tile_rows, T in ((16, 64), (32, 640), (64, 1024), (128, 2048)):
        for grad_dtype in (torch.float32, BF):
            calls.update(_adapter_calls(ctx, T, 512, 1024, tile_rows, grad_dtype))
    calls.update(_adapter_calls(ctx, 128, 2048, 4096, 16, BF))
    for fmt in (B.CKPT_E4M3, B.CKPT_INT8):
        calls.update(_kept_calls(ctx, fmt))
    return calls


def test_inputs_that_the_kernel_in_front_writes(ctx):  # noqa: F811
    bad = set()
    for name, (new, stale, call) in _all_calls(ctx).items():
        new = {n: _Tail(t) for n, t in new.items()}
        mine = {n: _Tail(s.t) for n, s in new.items()}
        given = {n: s.t for n, s in mine.items()}
        reset = [n for n in ("Y",) if "in place" in name]
        torch.cuda.synchronize()
        want = [t.clone() for t in call(given)]
        for last in new:
            t = new[last].t
            for rep in range(8):
                for n in reset:
                    mine[n].t.copy_(new[n].t)
                mine[last].t.copy_(stale[last] if last in stale else torch.zeros_like(t) if rep % 2 else t.flip(0))
                torch.cuda.synchronize()
                torch.cuda._sleep(400000)
                ctx.pad_2d(new[last].whole.view(BF).view(-1, 128), mine[last].whole.view(BF).view(-1, 128))
                got = call(given)
                torch.cuda.synchronize()
                if not all(torch.equal(a.reshape(-1).view(U8), b.reshape(-1).view(U8)) for a, b in zip(got, want)):
                    bad.add((name, last))
    assert not bad, sorted(bad)


@pytest.mark.parametrize("tile_rows", [16, 32, 64, 128])
def test_an_adapter_in_place_right_behind_its_product(ctx, tile_rows):  # noqa: F811
    """Y of the sparse product with an adapter (B not zero) added in place, and dX of the backward product with the adapter's part: as one at a time."""
    O, I, T = 1024, 2048, 1024
    gen = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda *shape, s: _empty(shape, BF).normal_(0.0, s, generator=gen)
    lin = SsteLinear(ctx, rnd(O, I, s=0.02), T, seed=5)
    X, dY = rnd(T, I, s=1.0), rnd(T, O, s=1e-2)
    lo = LoraAdapters(ctx, rnd(1, R, I, s=I ** -0.5), rnd(1, O, R, s=0.3), torch.full((1,), 2.0, device="cuda"), T)
    plan = LoraPlan([0, T], [0], T, 1, tile_rows=tile_rows)
    lin.init_beta(); lin.prune()
    plain = lin.forward(X).clone()
    want = lo.forward(X, plain, plan, out=torch.empty_like(plain)).clone()
    assert not torch.equal(want, plain)
    # against 64 bits: rounded to bf16 twice (the product, then the sum), V as two bf16 numbers
    part = 2.0 * (X.double() @ lo.A[0].double().t()) @ lo.B[0].double().t()
    room = (plain.double() + part).abs() * 2.0 ** -8 + 2.0 * (X.double().abs() @ lo.A[0].double().abs().t()) @ lo.B[0].double().abs().t() * 2.0 ** -11
    assert bool(((want.double() - plain.double() - part).abs() <= room + 1e-30).all())
    dx0, dw0 = (t.clone() for t in lin.backward(dY, step=3))
    dx1, dA1, dB1 = (t.clone() for t in lo.backward(dY, X, dx0, plan, out=torch.empty_like(dx0)))
    for _ in range(20):
        lin.Y.zero_(), lin.dX.zero_()
        torch.cuda.synchronize()
        torch.cuda._sleep(400000)
        y = lo.forward(X, lin.forward(X), plan)
        dx, dw = lin.backward(dY, step=3)
        dx, dA, dB = lo.backward(dY, X, dx, plan)
        assert y is lin.Y and dx is lin.dX
        torch.cuda.synchronize()
        assert torch.equal(y, want) and torch.equal(dw, dw0) and torch.equal(dx, dx1) and torch.equal(dA, dA1) and torch.equal(dB, dB1)


@pytest.mark.parametrize("tile_rows", [16, 32, 64, 128])
def test_chains_without_a_pause(ctx, tile_rows):  # noqa: F811
    """Product, adapter in place, the weights written anew, product of another input into the same Y, and so on, with nothing else in between: no
    call finds anything of the ones before it, in whatever cache."""
    O, I, T = 512, 1024, 512
    gen = torch.Generator(device="cuda").manual_seed(2)
    rnd = lambda *shape, s: _empty(shape, BF).normal_(0.0, s, generator=gen)
    lin = SsteLinear(ctx, rnd(O, I, s=0.02), T, seed=5)
    Xs, dYs = [rnd(T, I, s=1.0) for _ in range(3)], [rnd(T, O, s=1e-2) for _ in range(3)]
    As, Bs = [rnd(R * I // 128, 128, s=I ** -0.5) for _ in range(3)], [rnd(O * R // 128, 128, s=0.3) for _ in range(3)]
    A, Bw = torch.empty_like(As[0]), torch.empty_like(Bs[0])
    lo = LoraAdapters(ctx, A.view(1, R, I), Bw.view(1, O, R), torch.full((1,), 2.0, device="cuda"), T)
    plan = LoraPlan([0, T], [0], T, 1, tile_rows=tile_rows)
    lin.init_beta(); lin.prune()

    def step(i, pause):
        out = []
        for call in (lambda: ctx.pad_2d(As[i], A), lambda: ctx.pad_2d(Bs[i], Bw), lambda: lin.forward(Xs[i]), lambda: lo.forward(Xs[i], lin.Y, plan),
                     lambda: lin.backward(dYs[i], step=3), lambda: lo.backward(dYs[i], Xs[i], lin.dX, plan)):
            out = call()
            if pause:
                torch.cuda.synchronize()
        return lin.Y, *out

    want = [[t.clone() for t in step(i, True)] for i in range(3)]
    assert not torch.equal(want[0][0], want[1][0]) and not torch.equal(want[0][1], want[1][1])
    for n in range(1, 13):
        torch.cuda.synchronize()
        torch.cuda._sleep(400000)
        for k in range(n):
            got = step(k * k % 3 if n % 2 else k % 3, False)
        last = (n - 1) ** 2 % 3 if n % 2 else (n - 1) % 3
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want[last])), n
