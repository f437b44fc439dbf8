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
