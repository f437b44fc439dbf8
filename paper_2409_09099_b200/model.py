"""A GPT-2-124M-shaped decoder whose linear layers all run through libsste (a harness, not part of the hot path).

12 blocks of d = 768, 12 heads, FFN 3072, sequence 1024, vocabulary 50257.  The 48 linears (per block: qkv
[2304, 768], attention output [768, 768], fc1 [3072, 768], fc2 [768, 3072]) are S-STE linears: every training
step prunes the dense weight (Eq. 4, beta frozen after the first step, Sec. 4.2), runs forward and backward
with the sparse weight (Sec. 5.1) and hands grad_W to the optimiser unchanged (straight-through estimator,
Eq. 3).  Embeddings, layer norms, attention, GELU, the tied output projection, the loss and AdamW are stock
torch operations: they only produce the activations and gradients the S-STE linears consume.

Used by the config-4 test and by ``bench.py --config 4``; `on_call` lets a test inspect every libsste call.
"""
from __future__ import annotations

import torch
import torch.nn.functional as F

from . import binding as B
from .checkpoint import ActivationCheckpoint
from .layer import SsteLinear
from .lora import LoraAdapters, LoraPlan, LoraScratch


class _SsteFn(torch.autograd.Function):
    """Y = X S(W)^T through libsste; the gradient with respect to the fp32 master weight is grad_W (Eq. 3)."""

    @staticmethod
    def forward(ctx, x, w_master, owner):
        ctx.owner = owner
        lin = owner.lin
        owner.t0 = owner.model._tick()
        y = lin.forward(x)
        owner.model._tock(owner.t0)
        owner.x = x
        return y.detach()          # a fresh tensor object over the layer's output buffer

    @staticmethod
    def backward(ctx, dy):
        owner = ctx.owner
        lin, model = owner.lin, owner.model
        dy = dy.contiguous()
        t0 = model._tick()
        dx, dw = lin.backward(dy, step=model.step_index)
        model._tock(t0)
        if model.on_call is not None:
            model.on_call(owner.index, model.step_index, lin, owner.x, dy)
        return dx, dw.float(), None


class _SsteLeanFn(torch.autograd.Function):
    """_SsteFn with the input kept in 8 bits for the backward pass, a low-rank adapter beside the linear, or both."""

    @staticmethod
    def forward(ctx, x, w_master, a_master, b_master, owner):
        ctx.owner = owner
        lin, model = owner.lin, owner.model
        t0 = model._tick()
        y = lin.forward(x)
        if owner.kept is not None:
            lin.X = None                       # kept in 8 bits instead (the GELU in front may have kept its own input for it)
            if owner.kept.act is None:
                owner.kept.store(x)
        if owner.lora is not None:
            owner.lora.forward(x, y, model.plan)
        model._tock(t0)
        owner.x = x if owner.kept is None else None
        return y.detach()

    @staticmethod
    def backward(ctx, dy):
        owner = ctx.owner
        lin, model, kept = owner.lin, owner.model, owner.kept
        dy = dy.contiguous()
        t0 = model._tick()
        x = owner.x
        if kept is not None:
            x = lin.X = kept.load(out=model.room(x_of=lin))
        dx, dw = lin.backward(dy, step=model.step_index)
        da = db = None
        if owner.lora is not None:
            # (the checkpoint of a linear's own input is read as it is)
            _, da, db = owner.lora.backward(dy, kept if kept is not None and kept.act is None else x, dx, model.plan)
        model._tock(t0)
        if model.on_call is not None:
            model.on_call(owner.index, model.step_index, lin, x, dy)
        if kept is not None:
            lin.X = None
        return dx, dw.float(), da, db, None


class _GeluFn(torch.autograd.Function):
    """GELU (tanh form) that keeps its input in 8 bits: for its own gradient, and for its output as the next linear's input."""

    @staticmethod
    def forward(ctx, h, kept, model):
        ctx.kept, ctx.model = kept, model
        t0 = model._tick()
        y = kept.store(h, out=model.room(kept))
        model._tock(t0)
        return y.detach()

    @staticmethod
    def backward(ctx, dy):
        t0 = ctx.model._tick()
        # (where the outputs went: by now those have been read, and the layer in front takes the gradient before another GELU's comes)
        dx = ctx.kept.backward(dy.contiguous(), dx=ctx.model.room(ctx.kept))
        ctx.model._tock(t0)
        return dx, None, None


class SparseLinear:
    """fp32 master weight + bias (torch parameters) in front of one SsteLinear working on a bf16 copy."""

    def __init__(self, model, index, O, I, T, std, gen):
        dev = model.device
        self.model, self.index = model, index
        self.w = torch.nn.Parameter(torch.randn((O, I), device=dev, generator=gen) * std)
        self.b = torch.nn.Parameter(torch.zeros(O, device=dev))
        self.w16 = torch.empty((O, I), dtype=torch.bfloat16, device=dev)
        self.lin = SsteLinear(model.ctx, self.w16, T, tensor_id=index, seed=model.seed)
        self.beta_launches = 0
        self.x = None
        # the input in 8 bits: a checkpoint of its own, or (set by the model) that of the GELU in front
        self.kept = ActivationCheckpoint(model.ctx, (T, I), model.checkpoint) if model.checkpoint else None
        self.lora = None
        if model.adapter_rank:
            r = model.adapter_rank
            self.a = torch.nn.Parameter(torch.randn((1, r, I), device=dev, generator=gen) * I ** -0.5)
            self.bt = torch.nn.Parameter(torch.zeros((1, O, r), device=dev))
            self.lora = LoraAdapters(model.ctx, self.a.detach().bfloat16(), self.bt.detach().bfloat16(), torch.full((1,), 2.0, device=dev), T,
                                     scratch=model.lora_scratch)

    def refresh(self):
        """Start of a training step: the dense weight as bf16, beta in the first step only, then the projection."""
        self.w16.copy_(self.w.detach())
        t0 = self.model._tick()
        if not self.lin.beta_ready:
            self.lin.init_beta()
            self.beta_launches += 1
        self.lin.prune()
        self.model._tock(t0)
        if self.lora is not None:
            self.lora.A.copy_(self.a.detach())
            self.lora.B.copy_(self.bt.detach())

    def __call__(self, x):
        if self.kept is not None or self.lora is not None:
            a, bt = (self.a, self.bt) if self.lora is not None else (None, None)
            return _SsteLeanFn.apply(x, self.w, a, bt, self) + self.b.to(torch.bfloat16)
        return _SsteFn.apply(x, self.w, self) + self.b.to(torch.bfloat16)


class SsteGpt2:
    """``checkpoint`` ("int8" or "e4m3"): the linears' inputs and the GELUs' wait for the backward pass in 8 bits (checkpoint.py); per block
    that is 8.25 bits for each element of the inputs of qkv, attention output, fc1 and GELU, and nothing for fc2's; restored inputs, GELU outputs
    and their gradients share one tensor of each kind.  (torch's attention keeps its output in bf16 for itself.)  ``adapter_rank``: a
    low-rank adapter of this rank beside every linear, trained with it (lora.py).  Neither changes the default path."""

    def __init__(self, ctx: B.Context, n_layer=12, d=768, n_head=12, d_ff=3072, seq=1024, batch=8, vocab=50257,
                 seed=4, lr=3e-4, checkpoint: str | None = None, adapter_rank: int = 0):
        self.ctx, self.device, self.seed = ctx, f"cuda:{ctx.device}", seed
        self.n_layer, self.d, self.n_head, self.seq, self.batch, self.vocab = n_layer, d, n_head, seq, batch, vocab
        self.checkpoint, self.adapter_rank = checkpoint, adapter_rank
        T = batch * seq
        self.plan = LoraPlan([0, T], [0], T, 1, device=ctx.device) if adapter_rank else None
        self.lora_scratch = LoraScratch()        # (all linears' calls are in one stream's order)
        self.gelus, self._rooms = [], {}
        gen = torch.Generator(device=self.device).manual_seed(seed)
        self.wte = torch.nn.Parameter(torch.randn((vocab, d), device=self.device, generator=gen) * 0.02)
        self.wpe = torch.nn.Parameter(torch.randn((seq, d), device=self.device, generator=gen) * 0.02)
        self.linears, self.norms = [], []
        for l in range(n_layer):
            for O, I in ((3 * d, d), (d, d), (d_ff, d), (d, d_ff)):
                self.linears.append(SparseLinear(self, len(self.linears), O, I, T, 0.02, gen))
            if checkpoint:
                self.gelus.append(ActivationCheckpoint(ctx, (T, d_ff), checkpoint, act="gelu"))
                self.linears[-1].kept = self.gelus[-1]
            self.norms.append([torch.nn.Parameter(torch.ones(d, device=self.device)),
                               torch.nn.Parameter(torch.zeros(d, device=self.device)),
                               torch.nn.Parameter(torch.ones(d, device=self.device)),
                               torch.nn.Parameter(torch.zeros(d, device=self.device))])
        self.ln_f = [torch.nn.Parameter(torch.ones(d, device=self.device)),
                     torch.nn.Parameter(torch.zeros(d, device=self.device))]
        params = [self.wte, self.wpe] + [p for s in self.linears for p in (s.w, s.b) + ((s.a, s.bt) if s.lora else ())] + \
                 [p for n in self.norms for p in n] + self.ln_f
        self.opt = torch.optim.AdamW(params, lr=lr, weight_decay=0.0)
        self.step_index = 0
        self.on_call = None
        self._timing = None        # list of (start, end) CUDA events of the libsste calls of one step

    def room(self, kept=None, x_of=None):
        """A bf16 tensor that lives until the next one of its kind is wanted: a GELU's output or its input's gradient, or a linear's restored input."""
        key, shape = ("x", (x_of.T, x_of.I)) if kept is None else ("y", tuple(kept.shape))
        t = self._rooms.get((key, shape))
        if t is None:
            t = self._rooms[key, shape] = torch.empty(shape, dtype=torch.bfloat16, device=self.device)
        return t

    # ---- time spent inside libsste (CUDA events around its calls, when enabled)
    def _tick(self):
        if self._timing is None:
            return None
        e = torch.cuda.Event(enable_timing=True)
        e.record()
        return e

    def _tock(self, e0):
        if e0 is not None:
            e1 = torch.cuda.Event(enable_timing=True)
            e1.record()
            self._timing.append((e0, e1))

    def flops_per_step(self):
        """dense-equivalent flops of the S-STE linears: 6 T I O each (forward, grad_W, grad_X)."""
        return sum(6.0 * self.batch * self.seq * s.lin.O * s.lin.I for s in self.linears)

    def loss(self, tokens, targets):
        Bsz, S, d, H = self.batch, self.seq, self.d, self.n_head
        x = (self.wte[tokens] + self.wpe[None, :S]).to(torch.bfloat16).view(Bsz * S, d)
        for l in range(self.n_layer):
            qkv_l, proj_l, fc1_l, fc2_l = self.linears[4 * l: 4 * l + 4]
            g1, b1, g2, b2 = self.norms[l]
            h = F.layer_norm(x.float(), (d,), g1, b1).to(torch.bfloat16)
            q, k, v = qkv_l(h).view(Bsz, S, 3, H, d // H).permute(2, 0, 3, 1, 4)
            a = F.scaled_dot_product_attention(q, k, v, is_causal=True)
            a = a.transpose(1, 2).reshape(Bsz * S, d).contiguous()
            x = x + proj_l(a)
            h = F.layer_norm(x.float(), (d,), g2, b2).to(torch.bfloat16)
            if self.checkpoint:
                x = x + fc2_l(_GeluFn.apply(fc1_l(h), self.gelus[l], self))
            else:
                x = x + fc2_l(F.gelu(fc1_l(h), approximate="tanh").contiguous())
        h = F.layer_norm(x.float(), (d,), *self.ln_f).to(torch.bfloat16)
        logits = h @ self.wte.to(torch.bfloat16).t()            # tied output projection, dense
        return F.cross_entropy(logits.float(), targets.view(-1))

    def train_step(self, tokens, targets, time_libsste=False):
        """Prune every linear, forward, backward, optimiser step.  Returns (loss, seconds in libsste or None)."""
        self._timing = [] if time_libsste else None
        for s in self.linears:
            s.refresh()
        self.opt.zero_grad(set_to_none=True)
        loss = self.loss(tokens, targets)
        loss.backward()
        self.opt.step()
        inside = None
        if time_libsste:
            torch.cuda.synchronize()
            inside = sum(a.elapsed_time(b) for a, b in self._timing) * 1e-3
            self._timing = None
        self.step_index += 1
        return loss.detach(), inside


def synthetic_batch(model: SsteGpt2, seed: int):
    """Uniform token ids in [0, vocab) and next-token targets (a fixed synthetic batch)."""
    gen = torch.Generator(device=model.device).manual_seed(seed)
    ids = torch.randint(0, model.vocab, (model.batch, model.seq + 1), device=model.device, generator=gen)
    return ids[:, :-1].contiguous(), ids[:, 1:].contiguous()

