"""The projections' sums over many features on tiles of 128 rows: what they lose does not grow with the number of features.

An accumulator of the tensor core takes 32 instructions at most, each of which rounds towards zero and loses about 2^-27 of the sum
(2.4e-7 in all); the accumulators are added up in fp32, whose roundings (2^-25 of the sum on average) make a random walk: 128 additions for 65536
features, 3.4e-7.  Together 6e-7 of V.  A gradient in fp32 has its own 32 instructions and additions on top.
"""
import pytest
import torch

from tests.test_gpu_lora import _adapters, _problem, _rows_of, ctx  # noqa: F401

pytestmark = pytest.mark.gpu

T = 75 * 128                            # so many tiles that none shares its sums with another block


def _off(got, want):
    return float((got.double() - want).norm() / want.norm())


@pytest.mark.parametrize("r,K", [(64, 3080), (64, 11008), (64, 65536), (32, 40000), (16, 65536)])
def test_v_and_fp32_gradients(ctx, r, K):  # noqa: F811
    p = _problem(T, K, 64, r, 1, 1, seed=r, none=False)
    lo, plan = _adapters(ctx, p)
    assert plan.tile_rows == 128
    lo.forward(p["X"], p["Y"], plan)
    V = p["scale"][0].double() * (p["X"].double() @ p["A"][0].double().t())
    off = _off(lo.V, V)
    print(f"V, K = {K}, rank {r}: {off:.2e}")
    assert off < 7e-7
    del p, lo, V
    p = _problem(T, 64, K, r, 1, 1, seed=r + 1, none=False)
    lo, plan = _adapters(ctx, p)
    lo.V.zero_()
    _, dA, _ = lo.backward(p["dY"], p["X"], None, plan)
    U = p["scale"][0].double() * (p["dY"].double() @ p["B"][0].double())
    off = _off(dA[0], U.t() @ p["X"].double())
    print(f"dA, K = {K}, rank {r}: {off:.2e}")
    assert off < 1e-6


def test_each_round_of_the_accumulators(ctx):  # noqa: F811
    """Steps of K around whole rounds (48 of rank 64, 128 of rank 16), alone and shared by blocks, element by element."""
    from tests.test_gpu_lora import _check
    for r, steps in ((64, (47, 48, 49, 96, 97, 150)), (16, (127, 128, 129, 257))):
        for n in steps:
            _check(ctx, _problem(9500, 64 * n - 8, 72, r, 2, 3, 5, seed=n, none=False))
    _check(ctx, _problem(1100, 64 * 200, 64, 64, 1, 1, seed=1, none=False))
    _check(ctx, _problem(1100, 64 * 500 + 8, 64, 48, 1, 1, seed=1, none=False))
    _check(ctx, _problem(1100, 64, 64 * 400, 64, 1, 1, seed=1, none=False), grad_dtype=torch.bfloat16)


def test_bf16_gradients_of_many_rows(ctx):  # noqa: F811
    """dA of 524288 rows and 4096 features, all terms positive: a block's part of a sum is some 58000 rows, which leave the tensor core after
    8192 at most.  512 instructions lose up to 2^-23 each of a sum that is half the final one on average: 3.1e-5.  What the roundings
    to bf16 (2^-9.2 in square mean) do differently for 65536 results, whose sizes are spread over an octave, averages out to 7e-6."""
    from paper_2409_09099_b200.lora import LoraAdapters, LoraPlan
    rows, I, r = 524288, 4096, 16
    gen = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda *shape: torch.empty(shape, dtype=torch.bfloat16, device="cuda").uniform_(0.1, 1.1, generator=gen)
    size = torch.exp2(torch.rand(I, device="cuda", generator=gen))
    X = torch.empty((rows, I), dtype=torch.bfloat16, device="cuda")
    for i in range(0, rows, 8192):
        X[i:i + 8192] = (torch.rand((8192, I), device="cuda", generator=gen) + 0.1) * size
    dY, Bw = rnd(rows, 8), rnd(1, 8, r)
    lo = LoraAdapters(ctx, rnd(1, r, I), Bw, torch.ones(1, device="cuda"), rows, grad_dtype=torch.bfloat16)
    lo.V.fill_(1.0)
    _, dA, dB = lo.backward(dY, X, None, LoraPlan([0, rows], [0], rows, 1))
    U = dY.double() @ Bw[0].double()
    want = torch.zeros((r, I), dtype=torch.float64, device="cuda")
    for i in range(0, rows, 8192):
        want += U[i:i + 8192].t() @ X[i:i + 8192].double()
    off = float(((dA[0].double() - want.bfloat16().double()) / want).mean())
    print(f"dA, {rows} rows, bf16: {off:.2e} on average")
    assert abs(off) < 4e-5
    # element by element: half a step, and the bound of the loss
    assert bool(((dA[0].double() - want).abs() <= want * (2.0 ** -8 + 2.0 ** -14)).all())
    sums = dY.double().sum(0)[:, None]
    assert bool(((dB[0].double() - sums).abs() <= sums * (2.0 ** -8 + 2.0 ** -14)).all())


@pytest.mark.parametrize("r", [16, 32, 64])
@pytest.mark.parametrize("kept", [None, "int8"])
def test_bf16_gradients_that_are_emptied_on_the_way(ctx, r, kept):  # noqa: F811
    """Adapters of 80000 rows and of a few, so that a block has whole sums, ends of sums and parts of more than 8192 rows in turn: element by element."""
    from tests.test_gpu_lora import _check
    p = _problem(170003, 4104, 200, r, 4, 6, 11, seed=r, none=False)
    p["adapters"] = [0, 1, 0, 2, 3, 1]
    p["bounds"] = [0, 300, 80001, 80100, 160033, 165000, 169992]
    for (b, e), a in zip(zip(p["bounds"], p["bounds"][1:]), p["adapters"]):
        p["ids"][b:e] = a
    _check(ctx, p, kept, torch.bfloat16)


@pytest.mark.parametrize("r", [16, 32, 64])
def test_bf16_gradients_of_many_rows_on_small_tiles(ctx, r):  # noqa: F811
    """The same on tiles of 32 rows, and so many adapters (one of them in use) that a block has a whole sum: each warp's share is 131072 rows and more.
    Both bf16 numbers of U go to one accumulator here: 1024 instructions for 8192 rows, 6.1e-5."""
    from paper_2409_09099_b200.lora import LoraAdapters, LoraPlan
    rows, I, n = 524288, 4096, 64
    gen = torch.Generator(device="cuda").manual_seed(r)
    rnd = lambda *shape: torch.empty(shape, dtype=torch.bfloat16, device="cuda").uniform_(0.1, 1.1, generator=gen)
    size = torch.exp2(torch.rand(I, device="cuda", generator=gen))
    X = torch.empty((rows, I), dtype=torch.bfloat16, device="cuda")
    for i in range(0, rows, 8192):
        X[i:i + 8192] = (torch.rand((8192, I), device="cuda", generator=gen) + 0.1) * size
    dY, Bw = rnd(rows, 8), rnd(n, 8, r)
    lo = LoraAdapters(ctx, rnd(n, r, I), Bw, torch.ones(n, device="cuda"), rows, grad_dtype=torch.bfloat16)
    lo.V.fill_(1.0)
    _, dA, _ = lo.backward(dY, X, None, LoraPlan([0, rows], [5], rows, n, tile_rows=32))
    U = dY.double() @ Bw[5].double()
    want = torch.zeros((r, I), dtype=torch.float64, device="cuda")
    for i in range(0, rows, 8192):
        want += U[i:i + 8192].t() @ X[i:i + 8192].double()
    off = float(((dA[5].double() - want.bfloat16().double()) / want).mean())
    print(f"dA, {rows} rows, bf16, tiles of 32, rank {r}: {off:.2e} on average")
    assert abs(off) < 7e-5
    assert bool(((dA[5].double() - want).abs() <= want * (2.0 ** -8 + 2.0 ** -14)).all())
    assert not bool(dA[:5].any()) and not bool(dA[6:].any())
