"""Low-rank adapters of many requests (sste_lora_*) against 64 bits, element by element.

Bounds: a product of bf16 numbers is exact in fp32; a sum of n of them is off by at most n steps of 2^-23 of the sum of their magnitudes (the
tensor cores' sums may round towards zero, hence not 2^-24).  V and U meet the second product as two bf16 numbers, off by 2^-17 of their
value at most; the gradients' sums take three for fp32 results (2^-25).  bf16 results are rounded once, by half a step, 2^-8; fp32 ones by 2^-24.
"""
import math
import random

import pytest
import torch

from tests.gpu_util import DEV

pytestmark = pytest.mark.gpu

STEP, SPLIT = 2.0 ** -23, 2.0 ** -17


@pytest.fixture(scope="module")
def ctx():
    from paper_2409_09099_b200 import binding as B
    c = B.Context(0)
    yield c
    assert c.poll_device_status() == 0
    c.close()


def _problem(T, I, O, r, n, S, tail=0, seed=0, pad=0, none=True):
    rng = random.Random(seed)
    gen = torch.Generator(device=DEV).manual_seed(seed)
    gaussian = lambda *shape, s=1.0: (torch.randn(shape, device=DEV, generator=gen) * s).bfloat16()
    rows = T - tail
    bounds = list(range(S + 1)) if S == T else [0] + sorted(rng.randint(0, rows) for _ in range(S - 1)) + [rows]
    adapters = [rng.randrange(-1 if none and S > 1 else 0, n) for _ in range(S)]
    ids = torch.full((T,), -2)
    for (b, e), a in zip(zip(bounds, bounds[1:]), adapters):
        ids[b:e] = a
    wide = lambda rows, cols, s: gaussian(rows, cols + pad, s=s)[:, :cols]          # rows `pad` elements further apart
    return dict(T=T, I=I, O=O, r=r, n=n, bounds=bounds, adapters=adapters, ids=ids.to(DEV), A=gaussian(n, r, I, s=I ** -0.5),
                B=gaussian(n, O, r, s=0.1), scale=torch.rand(n, device=DEV, generator=gen) + 0.5, X=wide(T, I, 1.0), Y=wide(T, O, 0.5),
                dY=wide(T, O, 0.02), dX=wide(T, I, 0.02))


def _rows_of(p, a):
    return torch.nonzero(p["ids"] == a).view(-1)


def _reference(p):
    """V, Y, U, dX, dA, dB in 64 bits, each with its bound."""
    T, I, O, r, n = (p[k] for k in ("T", "I", "O", "r", "n"))
    d = dict(dtype=torch.float64, device=DEV)
    out = {k: torch.zeros(s, **d) for k, s in (("V", (T, r)), ("U", (T, r)), ("dA", (n, r, I)), ("dB", (n, O, r)))}
    out["Y"], out["dX"] = p["Y"].double(), p["dX"].double()
    room = {k: torch.zeros_like(v) for k, v in out.items()}
    for a in range(n):
        rows = _rows_of(p, a)
        X, dY, A, Bw, s = p["X"][rows].double(), p["dY"][rows].double(), p["A"][a].double(), p["B"][a].double(), p["scale"][a].double()
        V, U = s * X @ A.t(), s * dY @ Bw
        Vm, Um = s * X.abs() @ A.abs().t(), s * dY.abs() @ Bw.abs()                 # magnitudes
        Ve, Ue = Vm * (I + 2) * STEP, Um * (O + 2) * STEP
        out["V"][rows], out["U"][rows], room["V"][rows], room["U"][rows] = V, U, Ve, Ue
        out["Y"][rows] += V @ Bw.t()
        out["dX"][rows] += U @ A
        # (the sum starts from Y: its magnitude is in each step)
        room["Y"][rows] = (Ve + V.abs() * SPLIT) @ Bw.abs().t() + (2 * r + 2) * STEP * (p["Y"][rows].double().abs() + (V.abs() + Ve) @ Bw.abs().t())
        room["dX"][rows] = (Ue + U.abs() * SPLIT) @ A.abs() + (2 * r + 2) * STEP * (p["dX"][rows].double().abs() + (U.abs() + Ue) @ A.abs())
        Xk = p["Xk"][rows].double() if "Xk" in p else X
        out["dA"][a], out["dB"][a] = U.t() @ Xk, dY.t() @ V
        steps, split = (3 * len(rows) + 64) * STEP, p.get("split", SPLIT)
        room["dA"][a] = (Ue + U.abs() * split).t() @ Xk.abs() + steps * (U.abs() + Ue).t() @ Xk.abs()
        room["dB"][a] = dY.abs().t() @ (Ve + V.abs() * split) + steps * dY.abs().t() @ (V.abs() + Ve)
    for k in ("Y", "dX"):
        room[k] += out[k].abs() * 2.0 ** -8 + room[k] * 2.0 ** -8
    return out, room


def _close(got, want, room, name, half=0.0):
    got = got.double()
    bad = ~((got - want).abs() <= room * (1 + half) + want.abs() * half + 1e-30)
    assert not bool(bad.any()), (name, int(bad.sum()), torch.nonzero(bad)[:3].tolist(), got[bad][:3].tolist(), want[bad][:3].tolist())


def _adapters(ctx, p, grad_dtype=torch.float32, **plan):
    from paper_2409_09099_b200.lora import LoraAdapters, LoraPlan
    lo = LoraAdapters(ctx, p["A"], p["B"], p["scale"], p["T"], grad_dtype=grad_dtype)
    lo.V.fill_(7.0)
    return lo, LoraPlan(p["bounds"], p["adapters"], p["T"], p["n"], **plan)


def _check(ctx, p, kept=None, grad_dtype=torch.float32, **plan):
    from paper_2409_09099_b200.checkpoint import ActivationCheckpoint
    lo, pl = _adapters(ctx, p, grad_dtype, **plan)
    X = p["X"]
    if kept:
        X = ActivationCheckpoint(ctx, p["X"].shape, kept)
        X.store(p["X"].contiguous())
        p["Xk"] = X.load().clone()
    p["split"] = 2.0 ** -25 if grad_dtype is torch.float32 else SPLIT
    want, room = _reference(p)
    out = torch.full_like(p["Y"], 3.0) if p["Y"].is_contiguous() else p["Y"].clone(memory_format=torch.preserve_format)
    if out.stride() != p["Y"].stride():
        out = torch.full((p["T"], p["Y"].stride(0)), 3.0, dtype=torch.bfloat16, device=DEV)[:, :p["O"]]
    dout = torch.full((p["T"], p["dX"].stride(0) if p["T"] > 1 else p["I"]), 3.0, dtype=torch.bfloat16, device=DEV)[:, :p["I"]]
    out.fill_(3.0)
    y = lo.forward(p["X"], p["Y"], pl, out=out)
    assert y is out
    dx, dA, dB = lo.backward(p["dY"], X, p["dX"], pl, out=dout)
    inside, mine = p["ids"] > -2, p["ids"] >= 0
    _close(y[inside], want["Y"][inside], room["Y"][inside], "Y")
    _close(dx[inside], want["dX"][inside], room["dX"][inside], "dX")
    _close(lo.V[mine], want["V"][mine], room["V"][mine], "V")
    none = p["ids"] == -1
    assert torch.equal(y[none], p["Y"][none]) and torch.equal(dx[none], p["dX"][none])     # no adapter: as they were
    assert bool((y[~inside] == 3).all()) and bool((dx[~inside] == 3).all()) and bool((lo.V[~mine] == 7).all())   # padding: not touched
    half = 2.0 ** -8 if grad_dtype is torch.bfloat16 else 2.0 ** -24
    _close(dA, want["dA"], room["dA"], "dA", half)
    _close(dB, want["dB"], room["dB"], "dB", half)
    for a in range(p["n"]):
        if not len(_rows_of(p, a)):
            assert not bool(dA[a].any()) and not bool(dB[a].any())
    # the same calls give the same bits
    first = [t.clone() for t in (y, dx, dA, dB)]
    again = (lo.forward(p["X"], p["Y"], pl, out=out), *lo.backward(p["dY"], X, p["dX"], pl, out=dout))
    assert all(torch.equal(a, b) for a, b in zip(first, again))


SHAPES = [
    # T, I, O, r, n, S, tail
    (1, 8, 8, 8, 1, 1, 0), (1, 768, 768, 8, 1, 1, 0), (2, 40, 72, 16, 1, 1, 0), (3, 128, 64, 64, 2, 3, 0), (17, 64, 8, 24, 1, 1, 1),
    (15, 72, 136, 40, 3, 4, 2), (64, 1280, 648, 16, 64, 64, 0), (64, 256, 256, 48, 5, 64, 0), (129, 136, 200, 32, 2, 5, 7),
    (500, 320, 1000, 56, 4, 9, 33), (1000, 768, 264, 64, 1, 1, 0), (1037, 392, 520, 16, 7, 15, 100), (4099, 768, 1280, 8, 1, 1, 0),
    (2500, 1032, 96, 32, 3, 4, 11),
]


@pytest.mark.parametrize("tile_rows", [0, 128])
@pytest.mark.parametrize("T,I,O,r,n,S,tail", SHAPES)
def test_forward_and_backward(ctx, T, I, O, r, n, S, tail, tile_rows):
    _check(ctx, _problem(T, I, O, r, n, S, tail, seed=T + r), tile_rows=tile_rows)


@pytest.mark.parametrize("tile_rows", [16, 32, 64, 128])
@pytest.mark.parametrize("r", [8, 16, 32, 40, 64])
def test_every_tile_height(ctx, r, tile_rows):
    _check(ctx, _problem(700, 200, 328, r, 3, 7, 5, seed=r), tile_rows=tile_rows)
    _check(ctx, _problem(37, 1544, 88, r, 1, 1, 0, seed=r), tile_rows=tile_rows)


@pytest.mark.parametrize("T,r", [(90, 16), (90, 64), (1500, 16), (1500, 32), (1500, 64)])
def test_fp32_gradients_are_fp32(ctx, T, r):
    """fp32 gradients are as near to 64 bits as fp32 sums are: rounding errors of T sums and of U and V, far below two bf16 numbers' 2^-17."""
    p = _problem(T, 192, 200, r, 1, 1, seed=r, none=False)
    lo, pl = _adapters(ctx, p)
    lo.forward(p["X"], p["Y"].clone(), pl)
    _, dA, dB = lo.backward(p["dY"], p["X"], None, pl)
    want, _ = _reference(p)
    for got, name in ((dA, "dA"), (dB, "dB")):
        # a random walk of T (and 200) steps of 2^-24 of the terms: sqrt(1700) * 2^-24 = 2.5e-6 of the terms' size at most, which the sums
        # exceed sqrt(T)-fold
        assert float((got.double() - want[name]).norm() / want[name].norm()) < 1e-6, name


@pytest.mark.parametrize("kept", ["int8", "e4m3"])
@pytest.mark.parametrize("grad_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tile_rows", [0, 128])
@pytest.mark.parametrize("T,I,O,r,n,S,tail", [(1, 8, 16, 8, 1, 1, 0), (333, 72, 64, 16, 2, 3, 4), (1500, 520, 264, 64, 1, 1, 0),
                                             (900, 128, 128, 24, 5, 11, 50), (700, 400, 72, 40, 2, 4, 3)])
def test_kept_input(ctx, T, I, O, r, n, S, tail, grad_dtype, kept, tile_rows):
    _check(ctx, _problem(T, I, O, r, n, S, tail, seed=I), kept, grad_dtype, tile_rows=tile_rows)


@pytest.mark.parametrize("grad_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tile_rows", [32, 128])
def test_many_adapters_of_which_few_are_used(ctx, tile_rows, grad_dtype):
    """The others' gradients are zeros, whatever was there."""
    p = _problem(1100, 1032, 136, 24, 200, 3, 9, seed=12, none=False)
    _check(ctx, p, None, grad_dtype, tile_rows=tile_rows)
    lo, pl = _adapters(ctx, p, grad_dtype, tile_rows=tile_rows)
    lo.forward(p["X"], p["Y"].clone(), pl)
    for g in lo._grad_buffers():
        g.fill_(math.nan)
    _, dA, dB = lo.backward(p["dY"], p["X"], p["dX"].clone(), pl)
    unused = torch.tensor([a not in p["adapters"] for a in range(200)], device=DEV)
    assert not bool(dA[unused].any()) and not bool(dB[unused].any()) and bool(dA.isfinite().all()) and bool(dB.isfinite().all())


@pytest.mark.parametrize("r", [8, 24, 64])
def test_long_sums_of_few_rows(ctx, r):
    """Features in the thousands and few tiles of 128 rows, both ways: their blocks share the sums."""
    _check(ctx, _problem(300, 2056, 1288, r, 2, 3, 7, seed=r), tile_rows=128)
    _check(ctx, _problem(1200, 4104, 72, r, 1, 1, seed=r + 1), "int8", torch.bfloat16, tile_rows=128)


@pytest.mark.parametrize("tile_rows", [0, 128])
@pytest.mark.parametrize("pad", [8, 24, 256])
def test_rows_further_apart(ctx, pad, tile_rows):
    _check(ctx, _problem(301, 136, 200, 16, 2, 3, 5, seed=pad, pad=pad), tile_rows=tile_rows)


def test_gradients_against_differences(ctx):
    """The gradients of sum(G * (Y + s X A^T B^T)) in X, A and B by central differences of that sum in 64 bits (it is linear in each)."""
    p = _problem(200, 64, 96, 16, 2, 3, 0, seed=5, none=False)
    lo, pl = _adapters(ctx, p)
    lo.forward(p["X"], p["Y"].clone(), pl)
    dx, dA, dB = lo.backward(p["dY"], p["X"], torch.zeros_like(p["dX"]), pl)

    def loss(X, A, Bw):
        y = torch.zeros((p["T"], p["O"]), dtype=torch.float64, device=DEV)
        for a in range(p["n"]):
            rows = _rows_of(p, a)
            y[rows] = p["scale"][a].double() * (X[rows] @ A[a].t()) @ Bw[a].t()
        return float((y * p["dY"].double()).sum())

    at = [p[k].double() for k in ("X", "A", "B")]
    _, room = _reference({**p, "dX": torch.zeros_like(p["dX"])})
    rng = random.Random(1)
    for i, (got, allowed) in enumerate(((dx, room["dX"]), (dA, room["dA"]), (dB, room["dB"]))):
        for _ in range(12):
            where = tuple(rng.randrange(s) for s in got.shape)
            hi, lo_ = [t.clone() for t in at], [t.clone() for t in at]
            hi[i][where] += 0.5
            lo_[i][where] -= 0.5
            diff = loss(*hi) - loss(*lo_)
            # dX is bf16: half a step; the difference of two sums of 64 bits: 2^-40 of them
            assert abs(float(got[where]) - diff) <= float(allowed[where]) + abs(diff) * 2.0 ** -8 + 1e-9, (i, where)


@pytest.mark.parametrize("tile_rows", [0, 128])
def test_in_place_and_without_a_base(ctx, tile_rows):
    p = _problem(333, 128, 192, 16, 2, 3, 4, seed=2)
    lo, pl = _adapters(ctx, p, tile_rows=tile_rows)
    out = torch.empty_like(p["Y"])
    want = lo.forward(p["X"], p["Y"], pl, out=out)[:329].clone()
    y = p["Y"].clone()
    assert lo.forward(p["X"], y, pl, train=False) is y
    assert torch.equal(y[:329], want) and torch.equal(y[329:], p["Y"][329:])
    zero = lo.forward(p["X"], torch.zeros_like(y), pl, out=torch.zeros_like(y)).clone()
    assert torch.equal(lo.forward(p["X"], None, pl, out=torch.zeros_like(y)), zero)
    dx, dA, dB = lo.backward(p["dY"], p["X"], p["dX"], pl, out=torch.zeros_like(p["dX"]))
    want, dA0, dB0 = dx[:329].clone(), dA.clone(), dB.clone()
    d = p["dX"].clone()
    assert lo.backward(p["dY"], p["X"], d, pl)[0] is d and torch.equal(d[:329], want)
    none, dA, dB = lo.backward(p["dY"], p["X"], None, pl)
    assert none is None and torch.equal(dA, dA0) and torch.equal(dB, dB0)


@pytest.mark.parametrize("tile_rows", [0, 128])
def test_serving_leaves_nothing_behind(ctx, tile_rows):
    p = _problem(64, 256, 512, 16, 9, 64, seed=3)
    lo, pl = _adapters(ctx, p, tile_rows=tile_rows)
    lo.forward(p["X"], p["Y"], pl, train=False)
    assert bool((lo.V == 7).all())


@pytest.mark.parametrize("tile_rows", [0, 128])
def test_values_that_are_not_finite_stay_in_their_row(ctx, tile_rows):
    """A row with an infinity, a NaN or values that overflow touches no other; rows of padding may hold anything."""
    for r in (8, 24, 64):
        p = _problem(100, 128, 136, r, 1, 1, 10, seed=8, none=False)
        lo, pl = _adapters(ctx, p, tile_rows=tile_rows)
        want = lo.forward(p["X"], p["Y"], pl, out=torch.zeros_like(p["Y"])).clone()
        wx = lo.backward(p["dY"], p["X"], p["dX"], pl, out=torch.zeros_like(p["dX"]))[0].clone()
        p["X"][3, 5], p["X"][40, 100], p["X"][55, 0] = math.inf, math.nan, 3e38
        p["dY"][3, 5], p["dY"][40, 100] = -math.inf, math.nan
        p["X"][90:], p["dY"][90:], p["Y"][90:], p["dX"][90:] = math.nan, math.inf, math.nan, math.nan
        got = lo.forward(p["X"], p["Y"], pl, out=torch.zeros_like(p["Y"]))
        gx, dA, dB = lo.backward(p["dY"], p["X"], p["dX"], pl, out=torch.zeros_like(p["dX"]))
        rest = torch.tensor([t for t in range(100) if t not in (3, 40, 55)], device=DEV)
        assert torch.equal(got[rest], want[rest])
        assert not bool(torch.isfinite(got[3]).any()) and bool(torch.isnan(got[40]).all())
        rest = torch.tensor([t for t in range(100) if t not in (3, 40)], device=DEV)
        assert torch.equal(gx[rest], wx[rest])
        # an infinity in one row of V gives infinities where 64 bits do, not NaNs
        v = lo.V[3].double()
        exact = p["Y"][3].double() + v @ p["B"][0].double().t()
        assert torch.equal(torch.isnan(got[3]), torch.isnan(exact)) and torch.equal(torch.isinf(got[3]), torch.isinf(exact))


@pytest.mark.parametrize("tile_rows", [0, 128])
def test_empty_batches(ctx, tile_rows):
    from paper_2409_09099_b200.lora import LoraAdapters, LoraPlan
    p = _problem(20, 64, 64, 16, 3, 3, seed=1)
    lo, _ = _adapters(ctx, p)
    for bounds, adapters in (([0], []), ([5, 5], [1]), ([0, 0, 0], [0, 2])):
        pl = LoraPlan(bounds, adapters, 20, 3, tile_rows=tile_rows)
        y, d = p["Y"].clone(), p["dX"].clone()
        lo.forward(p["X"], y, pl)
        _, dA, dB = lo.backward(p["dY"], p["X"], d, pl)
        assert torch.equal(y, p["Y"]) and torch.equal(d, p["dX"]) and not bool(dA.any()) and not bool(dB.any())
    e = LoraAdapters(ctx, p["A"], p["B"], p["scale"], 0)
    none = torch.empty((0, 64), dtype=torch.bfloat16, device=DEV)
    pl = LoraPlan([0], [], 0, 3)
    e.forward(none, none, pl)
    _, dA, dB = e.backward(none, none, none, pl)
    assert not bool(dA.any()) and not bool(dB.any())


@pytest.mark.parametrize("rows", [16, 128])
def test_a_table_that_leads_nowhere_is_not_followed(ctx, rows):
    """Tiles outside the batch, too high, or of adapters that there are none of are left out: nothing is read or written for them."""
    p = _problem(4 * rows, 64, 64, 16, 2, 1, seed=4, none=False)
    p["adapters"] = [0]
    lo, pl = _adapters(ctx, p, tile_rows=rows)
    at = (p["n"] + 1 + 3) // 4 * 4
    table = pl.table.cpu()
    bad = [[4 * rows - 4, rows, 0, 0], [-16, rows, 0, 0], [0, rows + 1, 0, 0], [0, rows, 2, 0]]
    table[at:at + 16] = torch.tensor(bad, dtype=torch.int32).view(-1)
    groups = at + 16 + at                                            # of 16 rows: the same
    table[groups:].view(-1, 4)[:4] = torch.tensor([[4 * rows - 4, 16, 0, 0], [-16, 16, 0, 0], [0, 17, 0, 0], [0, 16, 0, 1 << 20]], dtype=torch.int32)
    table[groups:].view(-1, 4)[4:, 2] = 1
    pl.table.copy_(table)
    y = p["Y"].clone()
    lo.forward(p["X"], y, pl)
    _, dA, dB = lo.backward(p["dY"], p["X"], p["dX"].clone(), pl)
    assert torch.equal(y, p["Y"]) and not bool(dA.any()) and not bool(dB.any()) and bool((lo.V == 7).all())
    table[0], table[1] = 0, 1 << 30                                  # more tiles than the plan has
    pl.table.copy_(table)
    _, dA, _ = lo.backward(p["dY"], p["X"], p["dX"].clone(), pl)
    assert not bool(dA.any())


def test_captured_graph_with_other_requests(ctx):
    """A decode step captured once and replayed with other requests in the plan's table."""
    from paper_2409_09099_b200.lora import LoraAdapters, LoraPlan
    p = _problem(48, 256, 320, 16, 6, 48, seed=6)
    lo = LoraAdapters(ctx, p["A"], p["B"], p["scale"], 48)
    pl = LoraPlan(p["bounds"], p["adapters"], 48, 6, tile_rows=16, min_tiles=50)
    out = torch.zeros_like(p["Y"])
    lo.forward(p["X"], p["Y"], pl, out=out, train=False)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lo.forward(p["X"], p["Y"], pl, out=out, train=False)
    for bounds, adapters in ((list(range(49)), [i % 6 for i in range(48)]), ([0, 20, 31], [3, -1]), ([4, 4, 48], [0, 5])):
        pl.replace(bounds, adapters)
        out.zero_()
        graph.replay()
        fresh = LoraPlan(bounds, adapters, 48, 6)
        want = lo.forward(p["X"], p["Y"], fresh, out=torch.zeros_like(out), train=False)
        torch.cuda.synchronize()
        q = {**p, "ids": torch.full((48,), -2, device=DEV)}
        for (b, e), a in zip(zip(bounds, bounds[1:]), adapters):
            q["ids"][b:e] = a
        ref, room = _reference(q)
        inside = q["ids"] > -2
        _close(out[inside], ref["Y"][inside], room["Y"][inside], "Y")
        _close(want[inside], ref["Y"][inside], room["Y"][inside], "Y")
        assert not bool(out[~inside].any())
    with pytest.raises(ValueError):
        LoraPlan([0, 48], [0], 48, 6, tile_rows=16).replace(list(range(49)), [i % 6 for i in range(48)])


@pytest.mark.parametrize("tile_rows", [32, 128])
def test_two_at_once_on_two_streams(ctx, tile_rows):
    """No workspace is shared: two layers' calls may run side by side on one context."""
    ps = [_problem(1000, 256, 512, 16, 2, 3, seed=s) for s in (1, 2)]
    los = [_adapters(ctx, p, tile_rows=tile_rows) for p in ps]
    want = []
    for p, (lo, pl) in zip(ps, los):
        y = lo.forward(p["X"], p["Y"], pl, out=torch.zeros_like(p["Y"])).clone()
        want.append((y, *[t.clone() for t in lo.backward(p["dY"], p["X"], p["dX"], pl, out=torch.zeros_like(p["dX"]))]))
    streams = [torch.cuda.Stream() for _ in ps]
    for _ in range(5):
        got = []
        for p, (lo, pl), s in zip(ps, los, streams):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                y = lo.forward(p["X"], p["Y"], pl, out=torch.zeros_like(p["Y"]))
                got.append((y, *lo.backward(p["dY"], p["X"], p["dX"], pl, out=torch.zeros_like(p["dX"]))))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for w, g in zip(want, got) for a, b in zip(w, g))


def test_offsets_past_32_bits(ctx):
    """70000 rows 32768 elements apart: the last ones lie behind 2^32 bytes and 2^31 elements of X and Y."""
    T, I, O, ld = 70000, 64, 72, 32768
    p = _problem(T, I, O, 16, 2, 3, 40, seed=3)
    big = [torch.zeros((T, ld), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    for t, name, at in ((big[0], "X", 64), (big[1], "Y", 512), (big[1], "dY", 1024), (big[0], "dX", 2048)):
        cols = p[name].shape[1]
        t[:, at:at + cols] = p[name]
        p[name] = t[:, at:at + cols]
    want, room = _reference(p)
    lo, pl = _adapters(ctx, p)
    y = lo.forward(p["X"], p["Y"], pl)
    dx, dA, dB = lo.backward(p["dY"], p["X"], p["dX"], pl)
    inside = p["ids"] > -2
    _close(y[inside], want["Y"][inside], room["Y"][inside], "Y")
    _close(dx[inside], want["dX"][inside], room["dX"][inside], "dX")
    _close(dA, want["dA"], room["dA"], "dA")
    _close(dB, want["dB"], room["dB"], "dB")


def test_captured_training_step_of_large_tiles(ctx):
    """Forward and backward captured and replayed with new inputs and with other requests, tiles of 128 rows."""
    from paper_2409_09099_b200.lora import LoraPlan
    p = _problem(1500, 256, 320, 16, 3, 4, 20, seed=6, none=False)
    lo, _ = _adapters(ctx, p)
    pl = LoraPlan(p["bounds"], p["adapters"], 1500, 3, min_tiles=20)
    assert pl.tile_rows == 128
    y, d = torch.zeros_like(p["Y"]), torch.zeros_like(p["dX"])
    run = lambda: (lo.forward(p["X"], p["Y"], pl, out=y), *lo.backward(p["dY"], p["X"], p["dX"], pl, out=d))
    run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _, _, dA, dB = run()
    for bounds, adapters in ((p["bounds"], p["adapters"]), ([3, 300, 300, 1480], [2, 0, 2]), ([0, 1], [1])):
        pl.replace(bounds, adapters)
        p["X"].neg_()
        y.zero_(), d.zero_(), dA.fill_(7.0), dB.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        q = {**p, "ids": torch.full((1500,), -2, device=DEV), "split": 2.0 ** -25}
        for (b, e), a in zip(zip(bounds, bounds[1:]), adapters):
            q["ids"][b:e] = a
        want, room = _reference(q)
        inside = q["ids"] > -2
        _close(y[inside], want["Y"][inside], room["Y"][inside], "Y")
        _close(d[inside], want["dX"][inside], room["dX"][inside], "dX")
        _close(dA, want["dA"], room["dA"], "dA", 2.0 ** -24)
        _close(dB, want["dB"], room["dB"], "dB", 2.0 ** -24)
        assert not bool(y[~inside].any()) and not bool(d[~inside].any())


def test_refusals(ctx):
    from paper_2409_09099_b200 import binding as B
    from paper_2409_09099_b200.checkpoint import ActivationCheckpoint
    from paper_2409_09099_b200.lora import LoraAdapters, LoraPlan
    p = _problem(20, 64, 96, 16, 3, 3, seed=1)
    lo, pl = _adapters(ctx, p)
    for call in (lambda: LoraAdapters(ctx, p["A"], p["B"][:2], p["scale"], 20), lambda: LoraAdapters(ctx, p["A"].float(), p["B"], p["scale"], 20),
                 lambda: LoraAdapters(ctx, p["A"], p["B"], p["scale"], 20, grad_dtype=torch.float16),
                 lambda: LoraPlan([0, 20], [0, 1], 20, 3), lambda: lo.forward(p["X"][:10], p["Y"], pl), lambda: lo.forward(p["Y"], p["Y"], pl),
                 lambda: lo.forward(p["X"].float(), p["Y"], pl), lambda: lo.forward(p["X"], p["Y"], LoraPlan([0, 20], [0], 20, 4)),
                 lambda: lo.forward(p["X"], p["Y"], LoraPlan([0, 20], [0], 21, 3)),
                 lambda: lo.backward(p["dY"], ActivationCheckpoint(ctx, (20, 96), "int8"), p["dX"], pl),
                 lambda: lo.backward(p["dY"], ActivationCheckpoint(ctx, (20, 64), "int8", act="gelu"), p["dX"], pl),
                 lambda: lo.forward(p["X"].cpu(), p["Y"], pl), lambda: lo.forward(p["X"], None, pl),
                 lambda: lo.forward(p["X"], p["Y"], LoraPlan([0, 20], [0], 20, 3, device="cpu")),
                 lambda: lo.forward(p["X"], p["Y"], pl, out=torch.zeros((20, 104), dtype=torch.bfloat16, device=DEV)[:, :96])):
        with pytest.raises(ValueError):
            call()
    for bounds, adapters in (([0, 21], [0]), ([0, 20], [3]), ([5, 4], [0])):
        with pytest.raises(B.SsteError):
            LoraPlan(bounds, adapters, 20, 3)
    odd = torch.zeros((20, 65), dtype=torch.bfloat16, device=DEV)
    with pytest.raises(B.SsteError) as e:
        lo.forward(odd[:, :64], p["Y"], pl)
    assert e.value.code == B.ERR_SHAPE
    with pytest.raises(B.SsteError) as e:
        lo.forward(torch.zeros((20, 72), dtype=torch.bfloat16, device=DEV)[:, 4:68], p["Y"], pl)
    assert e.value.code == B.ERR_ALIGN


def test_weights_in_the_place_of_others(ctx):
    p = _problem(20, 64, 96, 16, 3, 3, seed=1)
    lo, pl = _adapters(ctx, p)
    y = lo.forward(p["X"], p["Y"], pl, out=torch.zeros_like(p["Y"])).clone()
    lo.A, lo.B = p["A"].clone(), p["B"] * 2
    want = LoraAdapters_of(ctx, lo).forward(p["X"], p["Y"], pl, out=torch.zeros_like(p["Y"]))
    again = lo.forward(p["X"], p["Y"], pl, out=torch.zeros_like(p["Y"]))
    assert torch.equal(again, want) and not torch.equal(again, y)
    for A in (p["A"][:2], p["A"].float(), p["A"].cpu(), torch.zeros((3, 16, 128), dtype=torch.bfloat16, device=DEV)[:, :, :64]):
        lo.A = A
        with pytest.raises(ValueError):
            lo.forward(p["X"], p["Y"], pl)


def LoraAdapters_of(ctx, lo):
    from paper_2409_09099_b200.lora import LoraAdapters
    return LoraAdapters(ctx, lo.A, lo.B, lo.scale, lo.T)


@pytest.mark.parametrize("grad_dtype", [torch.float32, torch.bfloat16])
def test_batches_of_many_sizes_share_one_scratch(ctx, grad_dtype):
    """Plans of all kinds in turn on one object; what a batch of NaNs leaves in the scratch reaches no later one."""
    from paper_2409_09099_b200.lora import LoraPlan
    T = 1500
    p = _problem(T, 264, 320, 40, 3, 6, 20, seed=8, none=False)
    lo, _ = _adapters(ctx, p, grad_dtype)
    p["split"] = 2.0 ** -25 if grad_dtype is torch.float32 else SPLIT
    bad = {k: torch.full_like(p[k], math.nan) for k in ("X", "Y", "dY", "dX")}
    y, d = torch.empty_like(p["Y"]), torch.empty_like(p["dX"])
    cases = [(p["bounds"], p["adapters"]), ([0, 7], [1]), ([0, 1499], [2]), ([3, 20, 900, 1100], [0, 0, 1])]
    for rows in (128, 16, 64, 128, 32):
        for bounds, adapters in cases:
            full = LoraPlan([0, T], [rows % 3], T, 3, tile_rows=rows)
            lo.forward(bad["X"], bad["Y"], full, out=y)
            lo.backward(bad["dY"], bad["X"], bad["dX"], full, out=d)
            lo.V.zero_()
            pl = LoraPlan(bounds, adapters, T, 3, tile_rows=rows)
            lo.forward(p["X"], p["Y"], pl, out=y)
            _, dA, dB = lo.backward(p["dY"], p["X"], p["dX"], pl, out=d)
            ids = torch.full((T,), -2, device=DEV)
            for (b, e), a in zip(zip(bounds, bounds[1:]), adapters):
                ids[b:e] = a
            want, room = _reference({**p, "ids": ids})
            inside = ids > -2
            _close(y[inside], want["Y"][inside], room["Y"][inside], "Y")
            _close(d[inside], want["dX"][inside], room["dX"][inside], "dX")
            half = 2.0 ** -8 if grad_dtype is torch.bfloat16 else 2.0 ** -24
            _close(dA, want["dA"], room["dA"], "dA", half)
            _close(dB, want["dB"], room["dB"], "dB", half)
    assert len({t.data_ptr() for t in lo._scratch.values()}) < len(lo._scratch)


@pytest.mark.parametrize("kept", ["int8", "e4m3"])
@pytest.mark.parametrize("T", [40, 700])
def test_kept_values_of_every_size(ctx, T, kept):
    """Kept inputs from 2^-120 to 2^120, zeros, and elements that are not finite: those make NaNs of their columns of dA and of nothing else."""
    from paper_2409_09099_b200.checkpoint import ActivationCheckpoint
    p = _problem(T, 72, 64, 16, 1, 1, seed=T, none=False)
    for extreme in (1.0, 2.0 ** 100, 2.0 ** -100):
        X = (p["X"].float() * torch.linspace(0, 1, 72, device=DEV) * extreme).bfloat16()
        X[5, 8], X[T - 1, 70] = math.nan, -math.inf
        k = ActivationCheckpoint(ctx, X.shape, kept)
        k.store(X)
        lo, pl = _adapters(ctx, p)
        lo.forward(p["X"], p["Y"].clone(), pl)
        _, dA, dB = lo.backward(p["dY"], k, None, pl)
        bad = torch.zeros(72, dtype=torch.bool, device=DEV)
        bad[[8, 70]] = True
        assert bool(torch.isnan(dA[0][:, bad]).all()) and bool(torch.isfinite(dA[0][:, ~bad]).all()) and bool(torch.isfinite(dB).all())
        want, room = _reference({**p, "Xk": k.load()})
        _close(dA[0][:, ~bad], want["dA"][0][:, ~bad], room["dA"][0][:, ~bad], "dA", 2.0 ** -24)
