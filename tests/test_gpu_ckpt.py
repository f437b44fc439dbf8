"""Activations kept in 8 bits (sste_ckpt_*): codes, scales and restored values bit for bit, activations and gradients against 64 bits."""
import math

import numpy as np
import pytest
import torch

from tests.gpu_util import DEV

pytestmark = pytest.mark.gpu

SIZES = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 1000, 4096, 8191, 8192 * 3 + 40, 203 * 71, 512 * 256]
FORMATS = ["int8", "e4m3"]


@pytest.fixture(scope="module")
def ctx():
    from paper_2409_09099_b200 import binding as B
    c = B.Context(0)
    yield c
    c.close()


def _values(n, seed=0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn(n, device=DEV, generator=gen)
    x *= torch.exp2(torch.randint(-20, 20, (n // 50 + 1,), device=DEV, generator=gen).float()).repeat_interleave(50)[:n]
    return x.bfloat16()


def _reference(x, fmt):
    """(codes, scales, values) of the rule in numpy's 64 bits: the least exponent found by trying all."""
    e4m3 = fmt == "e4m3"
    full, limit = (448.0, 1.875 * 2.0 ** 127) if e4m3 else (127.0, 1.96875 * 2.0 ** 127)
    v = x.float().cpu().numpy().astype(np.float64).ravel()
    v = np.concatenate([v, np.zeros(-v.size % 32)]).reshape(-1, 32)
    fine = np.isfinite(v)
    v = np.where(fine, np.clip(v, -limit, limit), 0.0)
    high = np.abs(v).max(1)
    tries = np.arange(-124, 128)
    e = tries[np.argmax(high[:, None] <= full * np.exp2(tries.astype(np.float64))[None], axis=1)]
    u = v * np.exp2(-e.astype(np.float64))[:, None]
    if e4m3:
        grid = np.exp2(np.maximum(np.floor(np.log2(np.maximum(np.abs(u), 1e-300))), -6.0) - 3)
        q = np.rint(u / grid) * grid
        mag = np.abs(q)
        ex = np.floor(np.log2(np.maximum(mag, 2.0 ** -9)))
        normal = ex >= -6
        codes = np.where(normal, (ex + 7) * 8 + mag / np.exp2(ex) * 8 - 8, mag * 512).astype(np.int64)
        codes = np.where(mag == 0, 0, codes) | np.where(np.signbit(u), 0x80, 0)
        codes = np.where(fine, codes, 0x7f)
    else:
        q = np.rint(u)
        codes = np.where(fine, q.astype(np.int64) & 0xff, 0x80)
    values = np.where(fine, q * np.exp2(e.astype(np.float64))[:, None], np.nan)
    return codes.astype(np.uint8).ravel(), (e + 127).astype(np.uint8), values.ravel()[:x.numel()]


def _check_kept(ctx, x, fmt):
    from paper_2409_09099_b200.checkpoint import ActivationCheckpoint
    k = ActivationCheckpoint(ctx, x.shape, fmt)
    assert k.store(x) is None
    back = k.load()
    codes, scales, values = _reference(x, fmt)
    assert np.array_equal(k.codes.cpu().numpy(), codes)
    assert np.array_equal(k.scales.cpu().numpy(), scales)
    got = back.float().cpu().numpy().astype(np.float64).ravel()
    assert np.array_equal(got, values, equal_nan=True)            # exactly: a kept value is a bf16 number


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("n", SIZES)
def test_kept_values(ctx, n, fmt):
    _check_kept(ctx, _values(n, n), fmt)


@pytest.mark.parametrize("fmt", FORMATS)
def test_every_value_as_a_blocks_maximum(ctx, fmt):
    """Each of the 65536 bf16 patterns in a block of its own, beside values from zero up to its own magnitude."""
    p = torch.arange(65536, device=DEV, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    frac = torch.linspace(-1, 1, 32, device=DEV)
    x = (p.float()[:, None] * frac).bfloat16()
    x[:, 7] = p
    _check_kept(ctx, x, fmt)
    # a finite value never becomes infinite, and is off by at most half a step of the block's grid
    from paper_2409_09099_b200.checkpoint import ActivationCheckpoint
    k = ActivationCheckpoint(ctx, x.shape, fmt)
    k.store(x)
    back = k.load().double()
    fine = torch.isfinite(x)
    assert torch.equal(torch.isfinite(back), fine) and bool(torch.isnan(back[~fine]).all())
    high = torch.where(fine, x.double().abs(), 0.0).amax(1, keepdim=True).expand_as(back)
    room = (x.double().abs() * 2.0 ** -4 + high * 2.0 ** -17 if fmt == "e4m3" else high / 126) + 2.0 ** -124
    room = room + torch.where(high > 1.9 * 2.0 ** 127, 0.1 * high, 0.0)                    # clamped
    assert bool(((back - x.double()).abs() <= room)[fine].all())


@pytest.mark.parametrize("fmt", FORMATS)
def test_special_values_leave_their_neighbours_alone(ctx, fmt):
    x = _values(4096, 3)
    for i, v in ((5, math.inf), (37, -math.inf), (70, math.nan), (71, -math.inf), (129, 3.3e38), (160, -3.38e38), (200, 1e-39), (300, -0.0)):
        x[i] = v
    x[512:544] = math.nan
    x[544:576] = 0.0
    x[576:608] = 1e-40
    x[608:640] = math.inf
    _check_kept(ctx, x, fmt)


def _phi(h):
    return 0.5 * (1 + torch.tanh(math.sqrt(2 / math.pi) * (h + 0.044715 * h ** 3)))


def _slope(h):
    # d/dh of h * phi(h); beyond 12 phi is 0 or 1 to the last bit of 64
    c = h.clamp(-12, 12)
    t = torch.tanh(math.sqrt(2 / math.pi) * (c + 0.044715 * c ** 3))
    return 0.5 * (1 + t) + 0.5 * c * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * c * c)


def _logistic_form(z):
    # h * phi(h) without the cancellation of 1 + tanh for negative h
    return torch.sigmoid(z)


def _near(got, want, scale, name):
    """bf16 rounding (half a step, 2^-8) plus the fp32 arithmetic: exponent arguments below 2^8 are off by 2^-15 at most, which an
    exponential turns into a relative 2^-15; sums that cancel are off by 2^-20 of `scale`; ftz below 2^-120."""
    got, want = got.double(), want.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want)), name
    off = (got - want).abs() - (want.abs() * (2.0 ** -8 + 2.0 ** -13) + scale.abs() * 2.0 ** -20 + 2.0 ** -120)
    ok = torch.isnan(want) | (off <= 0) | (got == want)
    assert bool(ok.all()), (name, got[~ok][:4], want[~ok][:4])


def _act_inputs(n, seed, wide):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn(n, device=DEV, generator=gen) * 2
    if wide:
        x = torch.linspace(-40, 40, n, device=DEV)
        x[:: 7] *= 1e-3
        x[3::101] = torch.linspace(-1e30, 1e30, len(x[3::101]), device=DEV)
    return x.bfloat16(), (torch.randn(n, device=DEV, generator=gen) * 0.01).bfloat16()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("n", [1, 31, 33, 4096, 10007])
def test_gelu(ctx, n, wide, fmt):
    from paper_2409_09099_b200.checkpoint import ActivationCheckpoint
    x, dy = _act_inputs(n, n, wide)
    k = ActivationCheckpoint(ctx, x.shape, fmt, act="gelu")
    y = k.store(x)
    h = x.double()
    sig = lambda h: h * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (h + 0.044715 * h ** 3))
    _near(y, sig(h), h * 0, "y")
    hk = torch.from_numpy(_reference(x, fmt)[2]).to(DEV)
    dx, again = k.backward(dy, again=True)
    _near(again, sig(hk), hk * 0, "again")
    _near(dx, dy.double() * _slope(hk), dy.double(), "dx")
    assert torch.equal(k.load(), again)                           # the same from either call
    assert torch.equal(k.backward(dy), dx)
    a, _, v = _reference(x, fmt)
    assert np.array_equal(k.codes.cpu().numpy(), a)               # kept as without an activation


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("n", [1, 31, 33, 4096, 10007])
def test_silu_gate(ctx, n, wide, fmt):
    from paper_2409_09099_b200.checkpoint import ActivationCheckpoint
    g, dy = _act_inputs(n, n, wide)
    u = _act_inputs(n, n + 1, False)[0]
    k = ActivationCheckpoint(ctx, g.shape, fmt, act="silu_gate")
    y = k.store(g, u)
    _near(y, g.double() * torch.sigmoid(g.double()) * u.double(), u * 0, "y")
    gk, uk = (torch.from_numpy(_reference(t, fmt)[2]).to(DEV) for t in (g, u))
    dx, dup, again = k.backward(dy, again=True)
    p = torch.sigmoid(gk)
    _near(again, gk * p * uk, u * 0, "again")
    _near(dup, dy.double() * gk * p, u * 0, "dup")
    _near(dx, dy.double() * uk * p * (1 + gk * (1 - p)), dy.double() * uk * p * (1 + gk.abs() * (1 - p)), "dx")
    assert torch.equal(k.load(), again)
    got = k.backward(dy)
    assert torch.equal(got[0], dx) and torch.equal(got[1], dup)
    assert np.array_equal(k.up_codes.cpu().numpy(), _reference(u, fmt)[0])


@pytest.mark.parametrize("act", ["gelu", "silu_gate"])
def test_gradients_against_differences(ctx, act):
    """dy d(act)/dx at the kept values against central differences of the activation in 64 bits (step 2^-12: error below 2^-20)."""
    from paper_2409_09099_b200.checkpoint import ActivationCheckpoint
    n, step = 2048, 2.0 ** -12
    gen = torch.Generator(device=DEV).manual_seed(1)
    x, u, dy = ((torch.randn(n, device=DEV, generator=gen) * s).bfloat16() for s in (2.0, 1.0, 1.0))
    k = ActivationCheckpoint(ctx, x.shape, "int8", act=act)
    k.store(x, u if act == "silu_gate" else None)
    hk, uk = (torch.from_numpy(_reference(t, "int8")[2]).to(DEV) for t in (x, u))
    f = (lambda h, w: h * _phi(h)) if act == "gelu" else (lambda h, w: h * torch.sigmoid(h) * w)
    slope = (f(hk + step, uk) - f(hk - step, uk)) / (2 * step)
    got = k.backward(dy)
    dx = got if act == "gelu" else got[0]
    room = (dy.double() * slope).abs() * 2.0 ** -8 + dy.double().abs() * (1 + uk.abs()) * 2.0 ** -18
    assert bool(((dx.double() - dy.double() * slope).abs() <= room).all())
    if act == "silu_gate":
        s = (f(hk, uk + step) - f(hk, uk - step)) / (2 * step)
        assert bool(((got[1].double() - dy.double() * s).abs() <= (dy.double() * s).abs() * (2.0 ** -8 + 2.0 ** -13) + 2.0 ** -40).all())


@pytest.mark.parametrize("act", [None, "gelu", "silu_gate"])
@pytest.mark.parametrize("n", [1, 17, 4099])
def test_nothing_is_written_behind_the_end(ctx, n, act):
    from paper_2409_09099_b200 import binding as B
    x = _values(n, 9)
    gate = act == "silu_gate"
    code_bytes, scale_bytes = B.load().sste_ckpt_code_bytes(n), B.load().sste_ckpt_scale_bytes(n)
    guard = lambda size, dt: torch.full((size + 64,), 77, dtype=dt, device=DEV)
    codes, scales, uc, us = (guard(s, torch.uint8) for s in (code_bytes, scale_bytes, code_bytes, scale_bytes))
    y, dx, dup, again, loaded = (guard(n, torch.bfloat16) for _ in range(5))
    a = {None: B.ACT_NONE, "gelu": B.ACT_GELU, "silu_gate": B.ACT_SILU_GATE}[act]
    up = (x, uc, us) if gate else (None, None, None)
    lib, h, s, dt = ctx.lib, ctx.handle, B._stream(), B.BF16
    ptr = lambda t: None if t is None else t.data_ptr()
    for fmt in (0, 1):
        assert lib.sste_ckpt_store(h, ptr(x), ptr(up[0]), n, dt, fmt, a, ptr(codes), ptr(scales), ptr(up[1]), ptr(up[2]),
                                   None if act is None else ptr(y), s) == 0
        assert lib.sste_ckpt_load(h, ptr(codes), ptr(scales), ptr(up[1]), ptr(up[2]), n, fmt, a, ptr(loaded), dt, s) == 0
        if act is not None:
            assert lib.sste_ckpt_act_bwd(h, ptr(x), ptr(codes), ptr(scales), ptr(up[1]), ptr(up[2]), n, dt, fmt, a, ptr(dx),
                                         ptr(dup) if gate else None, ptr(again), s) == 0
    for t, size in ((codes, code_bytes), (scales, scale_bytes), (uc, code_bytes), (us, scale_bytes), (y, n), (dx, n), (dup, n), (again, n),
                    (loaded, n)):
        assert bool((t[size:] == 77).all())


def test_in_place(ctx):
    from paper_2409_09099_b200.checkpoint import ActivationCheckpoint
    x, dy = _act_inputs(5000, 2, False)
    k = ActivationCheckpoint(ctx, x.shape, "int8", act="gelu")
    want = k.store(x).clone()
    dx = k.backward(dy).clone()
    k.store(x, out=x)
    assert torch.equal(x, want)
    g = dy.clone()
    ctx.ckpt_act_bwd(g, k.codes, k.scales, g, k._fmt, k._act)
    assert torch.equal(g, dx)


def test_empty(ctx):
    from paper_2409_09099_b200.checkpoint import ActivationCheckpoint
    k = ActivationCheckpoint(ctx, (0, 64), "int8", act="gelu")
    x = torch.empty((0, 64), dtype=torch.bfloat16, device=DEV)
    assert k.store(x).shape == (0, 64) and k.backward(x).shape == (0, 64) and k.load().shape == (0, 64)


def test_another_stream_and_a_captured_graph(ctx):
    from paper_2409_09099_b200.checkpoint import ActivationCheckpoint
    x, dy = _act_inputs(100_001, 4, False)
    k = ActivationCheckpoint(ctx, x.shape, "e4m3", act="gelu")
    want = [t.clone() for t in (k.store(x), *k.backward(dy, again=True))]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = [t.clone() for t in (k.store(x), *k.backward(dy, again=True))]
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = k.store(x)
        dx, again = k.backward(dy, again=True)
    x.neg_()
    want = [t.clone() for t in (k.store(x), *k.backward(dy, again=True))]
    for t in (y, dx, again, k.codes):
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, want[0]) and torch.equal(dx, want[1]) and torch.equal(again, want[2])


@pytest.mark.parametrize("fmt", FORMATS)
def test_offsets_past_32_bits(ctx, fmt):
    """2^31 + 40 elements: the last blocks lie behind 2^32 bytes of x and 2^31 of codes."""
    from paper_2409_09099_b200.checkpoint import ActivationCheckpoint
    n = 2 ** 31 + 40
    x = torch.empty(n, dtype=torch.bfloat16, device=DEV)
    x[: 2 ** 20] = _values(2 ** 20, 1)
    for at in range(2 ** 20, n, 2 ** 20):
        m = min(2 ** 20, n - at)
        x[at:at + m] = x[:m]
    k = ActivationCheckpoint(ctx, x.shape, fmt)
    k.store(x)
    back = k.load()
    for at in (0, 2 ** 30 - 64, 2 ** 31 - 2 ** 20, 2 ** 31 - 32, 2 ** 31):
        m = min(2 ** 20, n - at)
        codes, _, values = _reference(x[at:at + m], fmt)
        assert np.array_equal(back[at:at + m].float().cpu().numpy().astype(np.float64), values, equal_nan=True)
        assert np.array_equal(k.codes[at:at + codes.size].cpu().numpy(), codes)


def test_refusals(ctx):
    from paper_2409_09099_b200 import binding as B
    from paper_2409_09099_b200.checkpoint import ActivationCheckpoint
    x = _values(256, 1)
    with pytest.raises(ValueError):
        ActivationCheckpoint(ctx, (256,), "int4")
    with pytest.raises(ValueError):
        ActivationCheckpoint(ctx, (256,), "int8", act="relu")
    k, g = ActivationCheckpoint(ctx, (256,), "int8"), ActivationCheckpoint(ctx, (256,), "int8", act="silu_gate")
    for call in (lambda: k.store(x[:128]), lambda: k.store(x.float()), lambda: k.store(x, x), lambda: g.store(x), lambda: k.backward(x),
                 lambda: k.store(x, out=x), lambda: g.backward(x[:3]), lambda: k.load(x[:5]),
                 lambda: ActivationCheckpoint.of(ctx, k.codes, k.scales, (257,), "int8"), lambda: k.store(x.cpu()), lambda: k.load(x.cpu()),
                 lambda: ActivationCheckpoint.of(ctx, k.codes, k.scales, (256,), "int4"),
                 lambda: ActivationCheckpoint.of(ctx, k.codes.cpu(), k.scales, (256,), "int8"),
                 lambda: ActivationCheckpoint.of(ctx, k.codes.view(16, 16).t(), k.scales, (256,), "int8"),
                 lambda: ActivationCheckpoint(ctx, (256,), "int8", device="cpu")):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(B.SsteError) as e:
        ctx.ckpt_store(_values(300, 1)[1:257], k.codes, k.scales, 1)       # not on a 32-byte boundary
    assert e.value.code == B.ERR_ALIGN
