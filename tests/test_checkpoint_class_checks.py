"""Where ActivationCheckpoint puts what it keeps, on the host: allocations are recorded, nothing is launched."""
import types

import pytest
import torch

from paper_2409_09099_b200 import build


@pytest.mark.parametrize("device", [None, "cuda", "cuda:1", torch.device("cuda"), torch.device("cuda", 1)])
def test_everything_is_on_the_contexts_device(monkeypatch, device):
    """Also where the device is given without an index and another one is current."""
    build.build()
    from paper_2409_09099_b200 import checkpoint
    asked = []
    monkeypatch.setattr(checkpoint.torch, "empty", lambda shape, dtype, device: asked.append(torch.device(device)))
    k = checkpoint.ActivationCheckpoint(types.SimpleNamespace(device=1), (4, 64), "int8", act="silu_gate", device=device)
    k._buffer("y")
    assert k.device == torch.device("cuda", 1) and asked == [torch.device("cuda", 1)] * 5


@pytest.mark.parametrize("device", ["cuda:0", "cpu"])
def test_another_device_is_refused(device):
    build.build()
    from paper_2409_09099_b200 import checkpoint
    with pytest.raises(ValueError):
        checkpoint.ActivationCheckpoint(types.SimpleNamespace(device=1), (4, 64), "int8", device=device)
