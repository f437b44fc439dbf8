"""Numbers that a plan is made of: whole ones within 32 bits, or an error; none is cut to something else."""
import numpy as np
import pytest
import torch

from paper_2409_09099_b200 import binding as B, build


@pytest.fixture(scope="module", autouse=True)
def built():
    build.build()


def test_rows_per_tile_past_32_bits():
    for tile_rows in (2 ** 32 + 16, 2 ** 40, -2 ** 32 + 16):
        with pytest.raises(ValueError):
            B.lora_plan_build([0, 5], [0], 5, 1, tile_rows)


def test_numbers_that_are_not_whole():
    from paper_2409_09099_b200.lora import LoraPlan
    for offsets, adapters in (([0, 3.7], [0]), ([0, 3], [0.5]), ([0.25, 3], [0]), ([0, "3"], [0]), (torch.tensor([0, 3.5]), [0])):
        with pytest.raises(ValueError):
            LoraPlan(offsets, adapters, 5, 1, device="cpu")


def test_bounds_one_too_many_or_few():
    for offsets in ([0], [0, 2], [0, 2, 4, 5]):
        with pytest.raises(ValueError):
            B.lora_plan_build(offsets, [0, 1], 5, 2)


def test_numbers_of_any_integer_type():
    from paper_2409_09099_b200.lora import LoraPlan
    want = LoraPlan([0, 3, 5], [1, 0], 5, 2, device="cpu").table
    for offsets, adapters in ((np.array([0, 3, 5]), np.array([1, 0], dtype=np.int16)), (torch.tensor([0, 3, 5]), torch.tensor([1, 0])),
                              ((0, np.int32(3), 5), (True, False)),
                              (np.array([0.0, 3.0, 5.0]), [1, 0])):
        assert torch.equal(LoraPlan(offsets, adapters, 5, 2, device="cpu").table, want)
