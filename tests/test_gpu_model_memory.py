"""What the decoder's options cost in device memory between forward and backward, from the second step on (all buffers are there by then)."""
import gc

import pytest
import torch

pytestmark = pytest.mark.gpu

SIZES = dict(n_layer=6, d=256, n_head=4, d_ff=1024, seq=256, batch=8, vocab=640)


@pytest.fixture(scope="module")
def ctx():
    from paper_2409_09099_b200 import binding as B
    c = B.Context(0)
    yield c
    c.close()


def _waiting(ctx, **kw):
    """(device memory between forward and backward of the third step over what there was before the model, peak of that step, the model)"""
    from paper_2409_09099_b200.model import SsteGpt2, synthetic_batch
    gc.collect()
    before = torch.cuda.memory_allocated()
    m = SsteGpt2(ctx, **SIZES, **kw)
    batch = synthetic_batch(m, 4)
    for _ in range(2):
        m.train_step(*batch)
    torch.cuda.reset_peak_memory_stats()
    for s in m.linears:
        s.refresh()
    m.opt.zero_grad(set_to_none=True)
    loss = m.loss(*batch)
    between = torch.cuda.memory_allocated() - before
    loss.backward()
    return between, torch.cuda.max_memory_allocated() - before, m


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_kept_activations_save_what_they_say(ctx, fmt):
    _waiting(ctx)                                                # (torch's libraries get their workspaces)
    plain, plain_peak, m = _waiting(ctx)
    T = m.batch * m.seq
    # in bf16: the inputs of qkv, fc1 and fc2, and the GELUs' (its output is fc2's input).  That of the attention's output projection waits in
    # both, for torch's attention, whose output it is.
    bf16 = 2 * T * (2 * SIZES["d"] + 2 * SIZES["d_ff"]) * SIZES["n_layer"]
    del m
    kept, kept_peak, m = _waiting(ctx, checkpoint=fmt)
    codes = sum(k.nbytes for k in {id(s.kept): s.kept for s in m.linears}.values())
    rooms = sum(t.nbytes for t in m._rooms.values())
    assert codes == sum(T * i * 33 // 32 for i in (256, 256, 256, 1024)) * SIZES["n_layer"]
    # one bf16 tensor of each kind for the whole model: GELU output, restored inputs of the two widths
    assert rooms == 2 * T * (2 * SIZES["d_ff"] + SIZES["d"])
    print(f"{fmt}: {plain / 2 ** 20:.1f} MB waiting, peak {plain_peak / 2 ** 20:.1f}; kept {kept / 2 ** 20:.1f}, peak {kept_peak / 2 ** 20:.1f}")
    # (the allocator rounds each tensor up to 512 bytes)
    assert kept <= plain - bf16 + codes + rooms + 512 * 40 * SIZES["n_layer"]
    assert kept_peak < plain_peak
