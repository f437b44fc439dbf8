"""The stated error of kept values, for every bf16 number as a block's maximum and beside one, the smallest included."""
import pytest
import torch

from tests.gpu_util import DEV
from tests.test_gpu_ckpt import ctx  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_stated_error(ctx, fmt):  # noqa: F811
    """INT8: 1/127 of the block's maximum, at the least exponent 2^-125 (half of 2^-124).  E4M3: 2^-4 of the element or 2^-17 of the maximum; at the
    least exponent the steps of tiny elements are bf16's own, 2^-133."""
    from paper_2409_09099_b200.checkpoint import ActivationCheckpoint
    limit = (1.875 if fmt == "e4m3" else 1.96875) * 2.0 ** 127
    p = torch.arange(0x7f80, device=DEV, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)          # zero and all finite magnitudes
    gen = torch.Generator(device=DEV).manual_seed(1)
    for down in (0, 1, 7, 14, 30):                              # neighbours of the maximum's size, and ever smaller ones
        x = (p.float()[:, None] * torch.rand((len(p), 32), device=DEV, generator=gen) * 2.0 ** -down).bfloat16()
        x = torch.where(torch.rand(x.shape, device=DEV, generator=gen) < 0.5, x, -x)
        x[:, 11] = p
        k = ActivationCheckpoint(ctx, x.shape, fmt)
        k.store(x)
        off, x = (k.load().double() - x.double().clamp(-limit, limit)).abs(), x.double().abs()
        high = x.amax(1, keepdim=True).expand_as(x)
        room = torch.maximum(high / 127, torch.full_like(x, 2.0 ** -125)) if fmt == "int8" else torch.maximum(x * 2.0 ** -4, high * 2.0 ** -17)
        assert bool((off <= room).all()), (down, x[off > room][:4], high[off > room][:4])
