"""Cases of the operators that stand beside the S-STE linear: activations kept in 8 bits, and low-rank adapters.

  op = "keep"   the input of a linear is kept in 8 bits after the forward and restored for the weight gradient
  op = "act"    an activation (GELU, or the SiLU gate of two inputs) whose inputs are kept in 8 bits: its forward, then its backward from
                what was kept, which also gives the activation's output again (the next linear's input)
  op = "adapt"  low-rank adapters of the requests of a batch, added to the output of the shared linear
  op = "tune"   the gradients of such adapters and their part of the input gradient; the linear's input is bf16, or kept in 8 bits

T = rows (tokens), F = width of an activation, I, O = in and out features, r = rank, n = adapters, S = requests: consecutive rows that
share an adapter; `tail` rows follow the last request (a padded batch) and are left as they were.  S = T is one token for each request.

Kept values: blocks of 32 consecutive elements share a power of two 2^e, e the least (at least -124) with max|x| <= 448 * 2^e (E4M3) or
127 * 2^e (INT8) over the block's finite elements; an element is x * 2^-e rounded to nearest, ties to even.  Elements that are not finite
are restored as NaN; magnitudes above 1.875 * 2^127 (E4M3) or 1.96875 * 2^127 (INT8) count as that.
"""
from __future__ import annotations

import math
import random

import torch
import torch.nn.functional as F

own = False

MAX_T, MAX_F = 16384, 11008            # longest batch and widest layer of the shipped configurations


def _keep(T, width, fmt):
    return dict(op="keep", T=T, F=width, fmt=fmt)


def _act(act, T, width, fmt):
    return dict(op="act", act=act, T=T, F=width, fmt=fmt)


def _adapt(T, I, O, r, n=1, S=1, tail=0, train=False):
    return dict(op="adapt", T=T, I=I, O=O, r=r, n=n, S=S, tail=tail, train=train)


def _tune(T, I, O, r, n=1, S=1, tail=0, kept="", grads="bf16"):
    return dict(op="tune", T=T, I=I, O=O, r=r, n=n, S=S, tail=tail, kept=kept, grads=grads)


def listed():
    return [
        # the smallest layer of the repository's configurations: launches and host work are what it costs
        dict(name="keep_layer_256", **_keep(512, 256, "int8")),
        # input of the attention linears of a GPT-2-large block, 16 x 1024 tokens
        dict(name="keep_large", **_keep(16384, 1280, "e4m3")),
        # GELU of the GPT-2-large MLP
        dict(name="gelu_large", **_act("gelu", 16384, 5120, "int8")),
        # SiLU gate of the 7B-shaped FFN: the largest activation
        dict(name="gate_ffn", **_act("silu_gate", 16384, 11008, "e4m3")),
        # a batch of 1000 tokens, odd width: the last block is cut, rows start anywhere
        dict(name="gate_ragged", **_act("silu_gate", 1000, 1001, "int8")),
        # serving, one token of one request, through the attention output of a GPT-2-small block
        dict(name="adapt_token", **_adapt(1, 768, 768, 8)),
        # serving, 64 requests of one token each with adapters of their own, 7B-shaped up projection
        dict(name="adapt_decode", **_adapt(64, 4096, 11008, 16, n=64, S=64)),
        # serving, prompts of odd lengths, some without an adapter, padding rows behind; GPT-2-large qkv
        dict(name="adapt_prompts", **_adapt(4099, 1280, 3840, 32, n=8, S=13, tail=61)),
        # fine-tuning one adapter on the GPT-2-small qkv linear, 8 x 1024 tokens: forward, then backward
        dict(name="adapt_train", **_adapt(8192, 768, 2304, 16, train=True)),
        dict(name="tune_train", **_tune(8192, 768, 2304, 16)),
        # eight adapters at once on batches of odd lengths, inputs kept in 8 bits, fp32 gradients; GPT-2-large fc1
        dict(name="tune_ragged_kept", **_tune(4099, 1280, 5120, 24, n=8, S=11, tail=35, kept="int8", grads="fp32")),
        # one adapter of rank 64 on the 7B-shaped up projection: the most work
        dict(name="tune_ffn", **_tune(16384, 4096, 11008, 64, kept="e4m3")),
    ]


def draw(rng):
    def size(lo, hi):
        return int(round(lo * (hi / lo) ** rng.random()))

    def features():
        return max(64, size(64, MAX_F) // 8 * 8)

    caps = {op: max(work(c)["bytes"] for c in listed() if c["op"] == op) for op in ("keep", "act", "adapt", "tune")}
    while True:
        op = rng.choice(["keep", "act", "act", "adapt", "adapt", "tune", "tune"])
        fmt = rng.choice(["int8", "e4m3"])
        if op == "keep":
            case = _keep(size(16, MAX_T), size(64, MAX_F), fmt)
        elif op == "act":
            case = _act(rng.choice(["gelu", "silu_gate"]), size(16, MAX_T), size(64, MAX_F), fmt)
        else:
            r = 8 * rng.choice([1, 2, 2, 3, 4, 4, 5, 6, 7, 8])
            n = rng.choice([1, size(1, 64)])
            n = min(n, 1024 // r)
            if op == "adapt" and rng.random() < 0.4:      # one token for each request
                T = size(1, 256)
                case = _adapt(T, features(), features(), r, n=n, S=T)
            else:
                T = size(16, MAX_T)
                tail = rng.choice([0, rng.randrange(0, T // 4 + 1)])
                S = rng.choice([n, 2 * n + 1])
                if op == "adapt":
                    case = _adapt(T, features(), features(), r, n=n, S=S, tail=tail, train=rng.random() < 0.5)
                else:
                    case = _tune(T, features(), features(), r, n=n, S=S, tail=tail, kept=rng.choice(["", "", "int8", "e4m3"]),
                                 grads=rng.choice(["bf16", "fp32"]))
        if work(case)["bytes"] <= caps[op] and not any(all(c[k] == v for k, v in case.items() if k in c) for c in listed()
                                                       if c["op"] == op):
            return case


def _requests(case, seed):
    """Bounds of the requests (S + 1 of them) and the adapter of each, -1 for none."""
    rng = random.Random(seed * 7919 + 13)
    S, rows = case["S"], case["T"] - case["tail"]
    if S == case["T"]:
        bounds = list(range(S + 1))
    else:
        bounds = [0] + sorted(rng.randint(0, rows) for _ in range(S - 1)) + [rows]
    adapters = [rng.randrange(case["n"]) if case["n"] > 1 else 0 for _ in range(S)]
    if S > case["n"]:                                    # requests of the shared model itself
        adapters = [-1 if s % 5 == 4 else a for s, a in enumerate(adapters)]
    return bounds, adapters


def _codes(x, fmt):
    """The kept form of x (see the top): codes as bytes, one for each element of the blocks, and e + 127 of each block."""
    limit, top, full, mantissa = (1.875, 8, 448.0, 1.75) if fmt == "e4m3" else (1.96875, 6, 127.0, 127.0 / 64.0)
    x = F.pad(x.reshape(-1).float(), (0, -x.numel() % 32)).view(-1, 32)
    fine = torch.isfinite(x)
    x = x.clamp(-limit * 2.0 ** 127, limit * 2.0 ** 127)
    high = torch.where(fine, x.abs(), torch.zeros_like(x)).amax(1, keepdim=True)
    m, ex = torch.frexp(high)
    e = ex.int() - 1 - top + (2 * m > mantissa).int()
    e = torch.where(high > 0, e, torch.full_like(e, -124)).clamp(min=-124)
    v = x * ((127 - e) << 23).view(torch.float32)
    if fmt == "e4m3":
        codes = v.to(torch.float8_e4m3fn).view(torch.uint8)
        codes = torch.where(fine, codes, torch.full_like(codes, 0x7f))
    else:
        codes = torch.where(fine, v.round(), torch.full_like(v, -128.0)).to(torch.int8).view(torch.uint8)
    return codes.view(-1), (e + 127).to(torch.uint8).view(-1)


def _restored(codes, scales, shape, fmt):
    q = codes.view(-1, 32)
    if fmt == "e4m3":
        v = q.view(torch.float8_e4m3fn).float()
    else:
        v = q.view(torch.int8).float()
        v = torch.where(v == -128.0, torch.full_like(v, math.nan), v)
    s = (scales.int().clamp(min=1) << 23).view(torch.float32)
    return (v * s[:, None]).view(-1)[:math.prod(shape)].view(shape)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def gaussian(shape, sigma):
        return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(0.0, sigma, generator=gen)

    def activation(rows, width):
        # a few wide columns, as activations of trained transformers have them
        x = gaussian((rows, width), 1.0)
        x[:, (seed * 5 + 3) % width::97] *= 16.0
        return x

    T, s = case["T"], dict(case=case)
    if case["op"] == "keep":
        s["x"] = activation(T, case["F"])
        if own:
            from paper_2409_09099_b200 import binding as B
            from paper_2409_09099_b200.checkpoint import ActivationCheckpoint
            s["kept"] = ActivationCheckpoint(_context(B), s["x"].shape, case["fmt"])
        return s
    if case["op"] == "act":
        s["x"], s["dy"] = activation(T, case["F"]), gaussian((T, case["F"]), 1e-2)
        s["up"] = activation(T, case["F"]) if case["act"] == "silu_gate" else None
        if own:
            from paper_2409_09099_b200 import binding as B
            from paper_2409_09099_b200.checkpoint import ActivationCheckpoint
            s["kept"] = ActivationCheckpoint(_context(B), s["x"].shape, case["fmt"], act=case["act"])
        return s
    I, O, r, n = case["I"], case["O"], case["r"], case["n"]
    bounds, adapters = _requests(case, seed)
    ids = [-2] * T                                       # the adapter of each row: -1 none, -2 behind the last request
    for (b, e), a in zip(zip(bounds, bounds[1:]), adapters):
        ids[b:e] = [a] * (e - b)
    s["ids"] = torch.tensor(ids, device="cuda")
    s["A"], s["B"] = gaussian((n, r, I), I ** -0.5), gaussian((n, O, r), 0.05)
    s["scale"] = torch.linspace(2.0, 0.5, n, device="cuda")
    s["X"] = activation(T, I)
    if case["op"] == "adapt":
        s["Y"], s["out"] = gaussian((T, O), 0.5), torch.zeros((T, O), dtype=torch.bfloat16, device="cuda")
    else:
        s["dY"], s["dX"] = gaussian((T, O), 1e-2), gaussian((T, I), 1e-2)
        s["out"] = torch.zeros((T, I), dtype=torch.bfloat16, device="cuda")
        # what the forward left: s X A^T of each row, and the input, perhaps in 8 bits
        s["V"] = torch.zeros((T, r), device="cuda")
        for a in sorted(set(adapters) - {-1}):
            rows = s["ids"] == a
            s["V"][rows] = s["X"][rows].float() @ s["A"][a].float().t() * s["scale"][a]
        if case["kept"]:
            s["codes"], s["scales"] = _codes(s.pop("X"), case["kept"])
    if own:
        from paper_2409_09099_b200 import binding as B
        from paper_2409_09099_b200.checkpoint import ActivationCheckpoint
        from paper_2409_09099_b200.lora import LoraAdapters, LoraPlan
        ctx = _context(B)
        s["plan"] = LoraPlan(bounds, adapters, T, n, device=0)
        s["lora"] = LoraAdapters(ctx, s["A"], s["B"], s["scale"], T,
                                 grad_dtype=torch.float32 if case.get("grads") == "fp32" else torch.bfloat16)
        if case["op"] == "tune":
            s["lora"].V.copy_(s["V"])
            s["input"] = s.get("X")
            if case["kept"]:
                s["input"] = ActivationCheckpoint.of(ctx, s["codes"], s["scales"], (T, I), case["kept"])
        elif case["train"]:
            s["lora"].V.zero_()
    return s


_ctx = None


def _context(B):
    """One context, kept for the life of the program."""
    global _ctx
    if _ctx is None:
        _ctx = B.Context(0)
    return _ctx


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    case = s["case"]
    if case["op"] == "keep":
        s["kept"].store(s["x"])
        return {"x": s["kept"].load()}
    if case["op"] == "act":
        y = s["kept"].store(s["x"], s["up"])
        if s["up"] is None:
            dx, again = s["kept"].backward(s["dy"], again=True)
            return {"y": y, "dx": dx, "again": again}
        dx, dup, again = s["kept"].backward(s["dy"], again=True)
        return {"y": y, "dx": dx, "dup": dup, "again": again}
    if case["op"] == "adapt":
        y = s["lora"].forward(s["X"], s["Y"], s["plan"], out=s["out"], train=case["train"])
        return {"y": y, "V": s["lora"].V} if case["train"] else {"y": y}
    dx, da, db = s["lora"].backward(s["dY"], s["input"], s["dX"], s["plan"], out=s["out"])
    return {"dx": dx, "dA": da, "dB": db}


def _run_plain(s):
    case = s["case"]
    if case["op"] == "keep":
        return {"x": _restored(*_codes(s["x"], case["fmt"]), s["x"].shape, case["fmt"]).bfloat16()}
    if case["op"] == "act":
        return _plain_act(s, case)
    ids, n, r, T = s["ids"], case["n"], case["r"], case["T"]
    mine = ids[:, None] == torch.arange(n, device=ids.device)             # [T, n]
    Aall = s["A"].float().reshape(n * r, -1)
    Ball = s["B"].float().permute(1, 0, 2).reshape(-1, n * r)             # [O, n r]
    zero = torch.zeros((), device=ids.device)

    def chosen(v):                                                        # of the products with all adapters, the row's own
        return torch.where(mine[:, :, None], v.view(T, n, r) * s["scale"][:, None], zero).reshape(T, n * r)

    inside = (ids > -2)[:, None]
    if case["op"] == "adapt":
        v = chosen(s["X"].float() @ Aall.t())
        y = (s["Y"].float() + v @ Ball.t()).bfloat16()
        y = torch.where(inside, y, s["out"])
        return {"y": y, "V": v.view(T, n, r).sum(1)} if case["train"] else {"y": y}
    x = _restored(s["codes"], s["scales"], (T, case["I"]), case["kept"]) if case["kept"] else s["X"].float()
    g = s["dY"].float()
    u = chosen(g @ Ball)
    dx = torch.where(inside, (s["dX"].float() + u @ Aall).bfloat16(), s["out"])
    v = torch.where(mine[:, :, None], s["V"][:, None], zero).reshape(T, n * r)
    dA = (u.t() @ x).view(n, r, -1)
    dB = (g.t() @ v).view(-1, n, r).permute(1, 0, 2).contiguous()
    dt = torch.float32 if case["grads"] == "fp32" else torch.bfloat16
    return {"dx": dx, "dA": dA.to(dt), "dB": dB.to(dt)}


def _plain_act(s, case):
    dy, x = s["dy"].float(), s["x"].float()
    xk = _restored(*_codes(s["x"], case["fmt"]), x.shape, case["fmt"])
    if case["act"] == "gelu":
        def cdf(h):
            return 0.5 * (1 + torch.tanh(math.sqrt(2 / math.pi) * (h + 0.044715 * h * h * h)))

        y, p = x * cdf(x), cdf(xk)
        slope = p + xk * 2 * p * (1 - p) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * xk * xk)
        return {"y": y.bfloat16(), "dx": (dy * slope).bfloat16(), "again": (xk * p).bfloat16()}
    up = s["up"].float()
    uk = _restored(*_codes(s["up"], case["fmt"]), x.shape, case["fmt"])
    p = 1 / (1 + torch.exp(-xk))
    y = x / (1 + torch.exp(-x)) * up
    return {"y": y.bfloat16(), "dx": (dy * uk * p * (1 + xk * (1 - p))).bfloat16(), "dup": (dy * xk * p).bfloat16(),
            "again": (xk * p * uk).bfloat16()}


def work(case):
    T = case["T"]
    kept = 1 + 1 / 32
    if case["op"] == "keep":                             # in, kept, read again, out
        return {"bytes": T * case["F"] * (2 + 2 * kept + 2), "flops": 4 * T * case["F"]}
    if case["op"] == "act":
        n, inputs = T * case["F"], 2 if case["act"] == "silu_gate" else 1
        # forward: inputs in, output and the kept inputs out; backward: gradient and the kept inputs in, gradients and output out
        return {"bytes": n * (2 * inputs + 2 + kept * inputs + 2 + kept * inputs + 2 * inputs + 2), "flops": 30 * n}
    I, O, r, rows = case["I"], case["O"], case["r"], T - case["tail"]
    weights = 2 * min(case["n"], case["S"]) * r * (I + O)
    if case["op"] == "adapt":
        return {"bytes": rows * (2 * I + 4 * O + (4 * r if case["train"] else 0)) + weights, "flops": 2 * rows * r * (I + O)}
    grads = case["n"] * r * (I + O) * (4 if case["grads"] == "fp32" else 2)
    x = kept if case["kept"] else 2
    return {"bytes": rows * (2 * O + x * I + 4 * I + 4 * r) + weights + grads, "flops": 4 * rows * r * (I + O)}


def exact(case, seed):
    """From the definitions in 64 bits, an adapter at a time."""
    s = prepare(case, seed)

    def kept(x):
        """x as its kept form stands for it: the least exponent by search over the powers of two, then round to the format's grid."""
        e4m3 = (case.get("fmt") or case.get("kept")) == "e4m3"
        flat = F.pad(x.double().reshape(-1), (0, -x.numel() % 32)).view(-1, 32)
        high = flat.abs().amax(1, keepdim=True)
        e = torch.ceil(torch.log2(torch.clamp(high, min=1e-300) / (448.0 if e4m3 else 127.0)))
        e = torch.where(high > (448.0 if e4m3 else 127.0) * torch.exp2(e), e + 1, e)         # (the logarithm may be a hair off)
        e = torch.where(high <= (448.0 if e4m3 else 127.0) * torch.exp2(e - 1), e - 1, e)
        e = torch.clamp(e, min=-124.0)
        v = flat / torch.exp2(e)
        grid = torch.exp2(torch.floor(torch.log2(torch.clamp(v.abs(), min=2.0 ** -6))) - 3) if e4m3 else torch.ones_like(v)
        return (torch.round(v / grid) * grid * torch.exp2(e)).view(-1)[:x.numel()].view(x.shape)

    if case["op"] == "keep":
        return {"x": kept(s["x"])}
    if case["op"] == "act":
        x, dy, xk = s["x"].double(), s["dy"].double(), kept(s["x"])
        if case["act"] == "gelu":
            c = math.sqrt(2 / math.pi)

            def parts(h):
                t = torch.tanh(c * (h + 0.044715 * h ** 3))
                return 0.5 * h * (1 + t), 0.5 * (1 + t) + 0.5 * h * (1 - t * t) * c * (1 + 3 * 0.044715 * h ** 2)

            again, slope = parts(xk)
            return {"y": parts(x)[0], "dx": dy * slope, "again": again}
        uk = kept(s["up"])
        sig = torch.sigmoid(xk)
        return {"y": x * torch.sigmoid(x) * s["up"].double(), "dx": dy * uk * (sig + xk * sig * (1 - sig)), "dup": dy * xk * sig,
                "again": xk * sig * uk}
    T, I, O, r, n = (case[k] for k in ("T", "I", "O", "r", "n"))
    out = s["out"].double()
    rows_of = [torch.nonzero(s["ids"] == a).view(-1) for a in range(n)]
    none = torch.nonzero(s["ids"] == -1).view(-1)
    if case["op"] == "adapt":
        V = torch.zeros((T, r), dtype=torch.float64, device="cuda")
        out[none] = s["Y"][none].double()
        for a, rows in enumerate(rows_of):
            V[rows] = s["scale"][a].double() * (s["X"][rows].double() @ s["A"][a].double().t())
            out[rows] = s["Y"][rows].double() + V[rows] @ s["B"][a].double().t()
        return {"y": out, "V": V} if case["train"] else {"y": out}
    if case["kept"]:
        X = _restored(s["codes"], s["scales"], (T, I), case["kept"])
    else:
        X = s["X"]
    dA = torch.zeros((n, r, I), dtype=torch.float64, device="cuda")
    dB = torch.zeros((n, O, r), dtype=torch.float64, device="cuda")
    out[none] = s["dX"][none].double()
    for a, rows in enumerate(rows_of):
        g = s["dY"][rows].double()
        U = s["scale"][a].double() * (g @ s["B"][a].double())
        out[rows] = s["dX"][rows].double() + U @ s["A"][a].double()
        dA[a] = U.t() @ X[rows].double()
        dB[a] = g.t() @ s["V"][rows].double()
    return {"dx": out, "dA": dA, "dB": dB}
