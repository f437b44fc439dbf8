"""What the calls on kept activations and low-rank adapters refuse, and the plan of a batch's requests (no GPU needed).

The context and the buffers are addresses that nothing looks at: a call that gets as far as the device returns ERR_CUDA here.
"""
import ctypes
import random

import pytest

from paper_2409_09099_b200 import binding as B, build

CTX = ctypes.create_string_buffer(4096)
P = 0x100000


@pytest.fixture(scope="module")
def lib():
    build.build()
    return B.load()


@pytest.fixture(scope="module")
def no_gpu():
    import torch
    if torch.cuda.is_available():
        pytest.skip("addresses without memory behind them: not where a device could be asked")


def _ckpt(lib, call, **kw):
    d = dict(x=P, up=None, dy=P, n=100, dt=B.BF16, fmt=B.CKPT_INT8, act=B.ACT_GELU, codes=P, scales=P, up_codes=None, up_scales=None, y=P,
             dx=P, dup=None, ctx=CTX)
    if kw.get("act") == B.ACT_SILU_GATE:
        d.update(up=P, up_codes=P, up_scales=P, dup=P)
    d.update(kw)
    k = [d[n] for n in ("codes", "scales", "up_codes", "up_scales")]
    if call == "store":
        return lib.sste_ckpt_store(d["ctx"], d["x"], d["up"], d["n"], d["dt"], d["fmt"], d["act"], *k, d["y"], None)
    if call == "load":
        return lib.sste_ckpt_load(d["ctx"], *k, d["n"], d["fmt"], d["act"], d["y"], d["dt"], None)
    return lib.sste_ckpt_act_bwd(d["ctx"], d["dy"], *k, d["n"], d["dt"], d["fmt"], d["act"], d["dx"], d["dup"], d["y"], None)


@pytest.mark.parametrize("call", ["store", "load", "bwd"])
def test_kept_activations(lib, no_gpu, call):
    for act in (B.ACT_GELU, B.ACT_SILU_GATE):
        assert _ckpt(lib, call, act=act) == B.ERR_CUDA                          # nothing wrong: as far as the device
        assert _ckpt(lib, call, act=act, n=0, codes=None, x=None) == B.OK
        for name in ("codes", "scales") + (("up_codes", "up_scales") if act == B.ACT_SILU_GATE else ()):
            assert _ckpt(lib, call, act=act, **{name: None}) == B.ERR_INVALID_ARG, name
        for name in ("codes",) + (("up_codes",) if act == B.ACT_SILU_GATE else ()):
            assert _ckpt(lib, call, act=act, **{name: P + 8}) == B.ERR_ALIGN, name
        assert _ckpt(lib, call, act=act, fmt=2) == B.ERR_INVALID_ARG
        assert _ckpt(lib, call, act=act, ctx=None) == B.ERR_INVALID_ARG
        for dt in (B.F32, B.E4M3, B.E5M2):
            assert _ckpt(lib, call, act=act, dt=dt) == B.ERR_DTYPE
        needed = {"store": ("x", "y"), "load": ("y",), "bwd": ("dy", "dx")}[call]
        if act == B.ACT_SILU_GATE:
            needed += {"store": ("up",), "load": (), "bwd": ("dup",)}[call]
        for name in needed:
            assert _ckpt(lib, call, act=act, **{name: None}) == B.ERR_INVALID_ARG, name
            assert _ckpt(lib, call, act=act, **{name: P + 16}) == B.ERR_ALIGN, name
    assert _ckpt(lib, call, act=3) == B.ERR_INVALID_ARG
    assert _ckpt(lib, call, up_codes=P, up_scales=P) == B.ERR_INVALID_ARG      # GELU has one input
    none = dict(act=B.ACT_NONE, y=P if call == "load" else None)
    assert _ckpt(lib, call, **none) == (B.ERR_INVALID_ARG if call == "bwd" else B.ERR_CUDA)
    if call == "store":
        assert _ckpt(lib, call, act=B.ACT_NONE, y=P) == B.ERR_INVALID_ARG      # nothing to compute
        assert _ckpt(lib, call, up=P) == B.ERR_INVALID_ARG
    if call == "bwd":
        assert _ckpt(lib, call, y=None) == B.ERR_CUDA                          # the output again is optional
        assert _ckpt(lib, call, dup=P) == B.ERR_INVALID_ARG


def test_sizes_of_kept_activations(lib):
    for n in (0, 1, 31, 32, 33, 2 ** 33 + 1):
        assert lib.sste_ckpt_scale_bytes(n) == (n + 31) // 32 and lib.sste_ckpt_code_bytes(n) == (n + 31) // 32 * 32


def _lora(**kw):
    d = dict(n_adapters=3, rank=16, I=128, O=64, A=P, B=P, scale=P)
    d.update(kw)
    return B.LoraStruct(*[d[k] for k in ("n_adapters", "rank", "I", "O", "A", "B", "scale")])


def _plan(**kw):
    d = dict(T=40, n_adapters=3, tile_rows=16, n_tiles=4, table=P)
    d.update(kw)
    return B.LoraPlanStruct(*[d[k] for k in ("T", "n_adapters", "tile_rows", "n_tiles", "table")])


def _call(lib, call, lora=None, plan=None, **kw):
    d = dict(X=P, ldx=128, Y=2 * P, ldy=64, Y_in=2 * P, dX_in=3 * P, dX=3 * P, lddx=128, V=P, dA=P, dB=P, gdt=B.F32, codes=None, scales=None, fmt=B.CKPT_INT8,
             ctx=CTX, scratch=P, bytes=1 << 40)
    d.update(kw)
    l, p = ctypes.byref(lora or _lora()), ctypes.byref(plan or _plan())
    if call == "fwd":
        return lib.sste_lora_fwd(d["ctx"], l, p, d["X"], d["ldx"], d["Y_in"], d["Y"], d["ldy"], d["V"], d["scratch"], d["bytes"], None)
    return lib.sste_lora_bwd(d["ctx"], l, p, d["X"], d["ldx"], d["codes"], d["scales"], d["fmt"], d["Y"], d["ldy"], d["V"], d["dX_in"], d["dX"],
                             d["lddx"], d["dA"], d["dB"], d["gdt"], d["scratch"], d["bytes"], None)


@pytest.mark.parametrize("call", ["fwd", "bwd"])
def test_adapters(lib, no_gpu, call):
    assert _call(lib, call) == B.ERR_CUDA                                       # nothing wrong: as far as the device
    for bad in (0, 4, 12, 72, 128, -8):
        assert _call(lib, call, _lora(rank=bad)) == B.ERR_SHAPE
    for name in ("I", "O"):
        for bad in (0, 4, 12, -8, (1 << 24) + 8):
            assert _call(lib, call, _lora(**{name: bad})) == B.ERR_SHAPE
    for name in ("A", "B", "scale"):
        assert _call(lib, call, _lora(**{name: None})) == B.ERR_INVALID_ARG
        assert _call(lib, call, _lora(**{name: P + 2})) == B.ERR_ALIGN
    assert _call(lib, call, _lora(n_adapters=0), _plan(n_adapters=0)) == B.ERR_INVALID_ARG
    for bad in (dict(n_adapters=2), dict(T=-1), dict(tile_rows=0), dict(tile_rows=48), dict(n_tiles=-1), dict(n_tiles=1 << 24), dict(table=None)):
        assert _call(lib, call, None, _plan(**bad)) == B.ERR_INVALID_ARG
    assert _call(lib, call, None, _plan(table=P + 4)) == B.ERR_ALIGN
    assert _call(lib, call, ctx=None) == B.ERR_INVALID_ARG
    for name, least in (("ldx", 128), ("ldy", 64)) + ((("lddx", 128),) if call == "bwd" else ()):
        for bad in (least - 8, least + 4, 0, -least):
            assert _call(lib, call, **{name: bad}) == B.ERR_SHAPE, (name, bad)
        assert _call(lib, call, **{name: least + 8}) == B.ERR_CUDA
    need = lib.sste_lora_scratch_bytes(ctypes.byref(_lora()), ctypes.byref(_plan()))
    assert need > 0 and _call(lib, call, bytes=need) == B.ERR_CUDA
    assert _call(lib, call, bytes=need - 1) == B.ERR_WORKSPACE and _call(lib, call, scratch=None) == B.ERR_WORKSPACE
    assert _call(lib, call, scratch=P + 128) == B.ERR_ALIGN
    nothing = dict(X=None, Y=None, scratch=None, **(dict(dA=None, dB=None) if call == "bwd" else {}))
    assert _call(lib, call, None, _plan(T=0, n_tiles=0), **nothing) == B.OK


def test_operands_of_adapters(lib, no_gpu):
    for call, names in (("fwd", ("X", "Y")), ("bwd", ("X", "Y", "V", "dA", "dB", "dX"))):
        for name in names:
            assert _call(lib, call, **{name: None}) == B.ERR_INVALID_ARG, (call, name)
    for call, names in (("fwd", ("X", "Y", "Y_in", "V")), ("bwd", ("X", "Y", "V", "dX_in", "dX"))):
        for name in names:
            assert _call(lib, call, **{name: P + 8}) == B.ERR_ALIGN, (call, name)
    assert _call(lib, "fwd", Y_in=None, V=None) == B.ERR_CUDA                   # zeros, and nothing kept
    assert _call(lib, "bwd", dX_in=None) == B.ERR_CUDA
    assert _call(lib, "bwd", dX_in=None, dX=None, lddx=0) == B.ERR_CUDA         # gradients of the weights alone
    assert _call(lib, "bwd", dA=None, dB=None, X=None, V=None, ldx=0) == B.ERR_CUDA        # the input's alone
    assert _call(lib, "bwd", dA=None, dB=None, dX_in=None, dX=None) == B.ERR_INVALID_ARG
    for gdt in (B.E4M3, B.E5M2, 7):
        assert _call(lib, "bwd", gdt=gdt) == B.ERR_DTYPE
    kept = dict(X=None, codes=P, scales=P)
    assert _call(lib, "bwd", **kept) == B.ERR_CUDA
    assert _call(lib, "bwd", **{**kept, "fmt": 5}) == B.ERR_INVALID_ARG
    assert _call(lib, "bwd", **{**kept, "scales": None}) == B.ERR_INVALID_ARG
    assert _call(lib, "bwd", **{**kept, "X": P}) == B.ERR_INVALID_ARG
    assert _call(lib, "bwd", **{**kept, "codes": P + 8}) == B.ERR_ALIGN
    assert _call(lib, "bwd", dA=P + 8) == B.ERR_ALIGN and _call(lib, "bwd", dB=P + 8, gdt=B.BF16) == B.ERR_ALIGN
    assert _call(lib, "fwd", Y=P) == B.ERR_INVALID_ARG                          # a block may still read X when another has written its rows of Y
    assert _call(lib, "bwd", dX=P) == B.ERR_INVALID_ARG and _call(lib, "bwd", dX=2 * P) == B.ERR_INVALID_ARG
    assert lib.sste_lora_scratch_bytes(None, ctypes.byref(_plan())) == 0
    assert lib.sste_lora_scratch_bytes(ctypes.byref(_lora(rank=65)), ctypes.byref(_plan())) == 0


def _rows_of(plan, table):
    """(rows covered with their adapter, the tiles of each adapter) of a plan."""
    first = table[:plan.n_adapters + 1].tolist()
    at = (plan.n_adapters + 1 + 3) // 4 * 4
    tiles = table[at:at + 4 * plan.n_tiles].view(-1, 4).tolist()
    return first, tiles


@pytest.mark.parametrize("tile_rows", [0, 16, 32, 64, 128])
def test_plan_covers_each_row_once(lib, tile_rows):
    rng = random.Random(tile_rows)
    for trial in range(60):
        n, S = rng.choice([1, 2, 5, 40]), rng.choice([0, 1, 2, 7, 50])
        T = rng.choice([0, 1, 15, 16, 17, 300, 5000])
        bounds = sorted(rng.randint(0, T) for _ in range(S + 1))
        adapters = [rng.randrange(-1, n) for _ in range(S)]
        plan, table = B.lora_plan_build(bounds, adapters, T, n, tile_rows, 0)
        assert plan.tile_rows in (16, 32, 64, 128) and (tile_rows == 0 or plan.tile_rows == tile_rows)
        first, tiles = _rows_of(plan, table)
        seen = {}
        for row, rows, a, zero in tiles:
            assert 1 <= rows <= plan.tile_rows and zero == 0
            for t in range(row, row + rows):
                assert t not in seen
                seen[t] = a
        assert seen == {t: a for (b, e), a in zip(zip(bounds, bounds[1:]), adapters) for t in range(b, e)}
        for a in range(n):
            mine = tiles[first[a]:first[a + 1]]
            assert all(t[2] == a for t in mine) and sorted(mine) == mine
        assert first[0] == 0 and all(t[2] == -1 for t in tiles[first[n]:])
        # room for more
        more, table2 = B.lora_plan_build(bounds, adapters, T, n, plan.tile_rows, plan.n_tiles + 3)
        assert more.n_tiles == plan.n_tiles + 3 and _rows_of(more, table2)[1][-3:] == [[0, 0, -1, 0]] * 3
        assert _rows_of(more, table2)[1][:-3] == tiles


def test_plan_joins_neighbouring_requests(lib):
    plan, table = B.lora_plan_build([0, 3, 3, 10, 12], [1, 1, 1, 0], 12, 2, 16, 0)
    assert _rows_of(plan, table) == ([0, 1, 2], [[10, 2, 0, 0], [0, 10, 1, 0]])


def test_numbers_past_32_bits(lib):
    for offsets, adapters, T in (([0, 2 ** 32 + 5], [0], 8), ([0, 8], [2 ** 32], 8), ([0, 8], [0], 2 ** 32 + 8)):
        with pytest.raises(ValueError):
            B.lora_plan_build(offsets, adapters, T, 1)


def test_plan_refusals(lib):
    for bounds, adapters, T, n in (([0, 5], [2], 5, 2), ([0, 5], [-2], 5, 2), ([0, 6], [0], 5, 2), ([-1, 5], [0], 5, 2),
                                   ([3, 2], [0], 5, 2), ([0, 5], [0], 5, 0), ([0, 5], [0], 5, 65536)):
        with pytest.raises(B.SsteError) as e:
            B.lora_plan_build(bounds, adapters, T, n)
        assert e.value.code == B.ERR_INVALID_ARG, (bounds, adapters, T, n)
    for tile_rows in (1, 8, 48, 256, -16):
        with pytest.raises(B.SsteError):
            B.lora_plan_build([0, 5], [0], 5, 1, tile_rows)
    arr, plan = (ctypes.c_int * 64)(), B.LoraPlanStruct()
    args = ((ctypes.c_int * 2)(0, 300), (ctypes.c_int * 1)(0), 1, 300, 1, 16, 0, arr)
    assert lib.sste_lora_plan_build(*args, 64, ctypes.byref(plan)) == B.ERR_WORKSPACE      # 19 tiles need 80 numbers
    assert lib.sste_lora_plan_build(*args[:7], None, 1000, ctypes.byref(plan)) == B.ERR_INVALID_ARG
    assert lib.sste_lora_plan_build(*args, 64, None) == B.ERR_INVALID_ARG
    assert lib.sste_lora_plan_build(None, *args[1:], 64, ctypes.byref(plan)) == B.ERR_INVALID_ARG
    assert lib.sste_lora_plan_ints(300, 1, 1, 0) >= 80 and lib.sste_lora_plan_ints(-1, 1, 1, 0) == 0
