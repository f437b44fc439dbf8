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


def test_the_linears_adapters_share_one_scratch(ctx):
    """Not a scratch for each linear: one, grown to the largest need, beside smaller ones that it has outgrown."""
    from paper_2409_09099_b200.model import SsteGpt2, synthetic_batch
    m = SsteGpt2(ctx, **SIZES, adapter_rank=16)
    batch = synthetic_batch(m, 4)
    for _ in range(2):
        m.train_step(*batch)
    need = max(ctx.lib.sste_lora_scratch_bytes(s.lora.at, m.plan.at) for s in m.linears)
    scratches = {t.data_ptr(): t.nbytes for s in m.linears for t in s.lora._scratch.values()}
    assert need <= max(scratches.values()) <= 3 * need // 2
    # each is 1.5 times the one before it, or more: together they are less than three times the largest
    assert sum(scratches.values()) <= 3 * max(scratches.values())


@pytest.mark.parametrize("tile_rows", [16, 128])
def test_a_shared_scratch_changes_no_result(ctx, tile_rows):
    from paper_2409_09099_b200.lora import LoraAdapters, LoraPlan, LoraScratch
    from tests.test_gpu_lora import _problem
    shared, objects, want = LoraScratch(), [], []
    for seed, (I, O, r) in enumerate([(256, 512, 16), (1032, 136, 40), (64, 2048, 64)]):
        p = _problem(1100, I, O, r, 3, 5, 20, seed=seed, none=False)
        own = LoraAdapters(ctx, p["A"], p["B"], p["scale"], 1100)
        objects.append((p, LoraAdapters(ctx, p["A"], p["B"], p["scale"], 1100, scratch=shared), LoraPlan(p["bounds"], p["adapters"], 1100, 3, tile_rows=tile_rows)))
        y = own.forward(p["X"], p["Y"], objects[-1][2], out=torch.zeros_like(p["Y"]))
        want.append([t.clone() for t in (y, *own.backward(p["dY"], p["X"], p["dX"], objects[-1][2], out=torch.zeros_like(p["dX"])))])
    for _ in range(2):
        for order in ((0, 1, 2), (2, 0, 1)):
            ys = {i: lo.forward(p["X"], p["Y"], plan, out=torch.zeros_like(p["Y"])) for i, (p, lo, plan) in ((i, objects[i]) for i in order)}
            for i in order:
                p, lo, plan = objects[i]
                got = (ys[i], *lo.backward(p["dY"], p["X"], p["dX"], plan, out=torch.zeros_like(p["dX"])))
                assert all(torch.equal(a, b) for a, b in zip(got, want[i]))
