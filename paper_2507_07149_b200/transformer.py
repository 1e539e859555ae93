"""The operators of a transformer's training step as differentiable functions and layers, and a small trainer.

``attention``, ``residual_norm``, ``embedding``, ``rotary_norm`` and ``clip_grad_norm_`` run the CUDA kernels behind the C ABI; they can
be differentiated once.  ``Muon`` steps by orthogonalised updates.  Attention keeps q, k, v, its output and one float per row for the
backward pass, the join keeps its two activations, rotary norms keep q and k as they were, the embedding its tokens; what they keep goes through autograd's saved-tensor hooks, so inside ``saved_activation_compression`` it is held in compressed
form like every other activation.  Attention's row statistics belong to the scores they were taken from: at 8 bits per value they are kept as they
are, below that (or with a store, which may drop a tensor) the backward pass takes them, and the output, anew from the
restored q, k and v, at the price of a second forward pass of attention and without keeping the output.
Nothing here waits for the device; ``check_device`` (and ``check_status`` of the compression) tell whether an attention kernel
gave up.

    python -m paper_2507_07149_b200.transformer --steps 20            # trains a small classifier on synthetic sequences
    python -m paper_2507_07149_b200.transformer --steps 20 --plain    # the same without compressed activations
    python -m paper_2507_07149_b200.transformer --language            # a small language model: token embedding, rotary norms, Muon
"""
from __future__ import annotations

import argparse
import math

import torch
from torch.autograd.function import once_differentiable

from . import attention as _attention
from . import attention_grad, check_device, clip_grad_norm
from . import embedding as _embedding
from . import embedding_grad, gap_free, orthogonalize
from . import residual_norm as _residual_norm
from . import residual_norm_grad
from . import rotary_norm as _rotary_norm
from . import rotary_norm_grad
from .autograd import active_compression


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, key_lengths, causal, scale):
        out, lse = _attention(q, k, v, causal=causal, scale=scale, key_lengths=key_lengths)
        # Probabilities exp(S' - lse) of restored scores S' with the lse of the exact ones do not sum to one.  Relative error of
        # the gradient of q (256 tokens, heads of 64, q and k of standard deviation 1 / 2 / 3), lse kept against taken anew:
        # 8 bits 0.019 0.062 0.14 / 0.018 0.037 0.078, 4 bits 0.34 2.7 120 / 0.31 0.57 0.91, 2 bits 14 3e8 3e20 / 2.5 1.8 1.6.
        compression = active_compression()
        if compression is not None and compression.coarse:
            ctx.save_for_backward(key_lengths, q, k, v)
            lse = None
        else:
            ctx.save_for_backward(key_lengths, q, k, v, out)
        ctx.lse, ctx.how = lse, (causal, scale)
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_out):
        key_lengths, q, k, v, *out = ctx.saved_tensors
        how = dict(causal=ctx.how[0], scale=ctx.how[1], key_lengths=key_lengths)
        out, lse = (out[0], ctx.lse) if out else _attention(q, k, v, **how)
        return *attention_grad(q, k, v, out, lse, grad_out, **how), None, None, None


def attention(q, k, v, *, causal: bool = False, scale: float | None = None, key_lengths=None):
    """Differentiable ``daf.attention``: q [B, Sq, H, D], k and v [B, Sk, Hkv, D]; returns the output alone."""
    return _Attention.apply(q, k, v, key_lengths, causal, scale)


class _ResidualNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, y, weight, bias, gate, post_weight, post_bias, how):
        ctx.set_materialize_grads(False)
        z, h = _residual_norm(x, y, weight, bias, gate=gate, post_weight=post_weight, post_bias=post_bias, **how)
        ctx.save_for_backward(z, y, weight, bias, gate, post_weight, post_bias)
        ctx.how = how
        return z, h

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_z, grad_h):
        z, y, weight, bias, gate, post_weight, post_bias = ctx.saved_tensors
        if grad_h is None:                                          # h was not used
            grad_h = torch.zeros_like(z)
        g = residual_norm_grad(z, y, weight, bias, None if grad_z is None else grad_z.contiguous(), grad_h.contiguous(), gate=gate,
                               post_weight=post_weight, post_bias=post_bias, **ctx.how)
        return g["x"], g["y"], g["weight"], g["bias"], g["gate"], g["post_weight"], g["post_bias"], None


def residual_norm(x, y, weight, bias=None, *, gate=None, post_weight=None, post_bias=None, residual_scale: float = 1.0,
                  kind: str = "layer", eps: float = 1e-6):
    """Differentiable ``daf.residual_norm``: (z, h) of the join z = x + residual_scale * gate * post_norm(y), h = norm(z).  x and y
    may differ in type (a block under autocast): both are then taken in the wider one."""
    if x.dtype != y.dtype:
        wide = torch.promote_types(x.dtype, y.dtype)
        x, y = x.to(wide), y.to(wide)
    return _ResidualNorm.apply(x.contiguous(), y.contiguous(), weight, bias, gate, post_weight, post_bias,
                               dict(residual_scale=residual_scale, kind=kind, eps=eps))


class _Embedding(torch.autograd.Function):
    @staticmethod
    def forward(ctx, tokens, weight, scale, padding, dtype):
        if padding is not None and not 0 <= padding < weight.shape[0]:
            raise ValueError("embedding: padding is a token, or None")
        ctx.save_for_backward(tokens)
        ctx.how = (weight.shape[0], scale, padding, weight.dtype)
        return _embedding(tokens, weight, scale=scale, dtype=dtype)

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_out):
        vocabulary, scale, padding, dtype = ctx.how
        return None, embedding_grad(*ctx.saved_tensors, grad_out, vocabulary, scale=scale, padding=padding, dtype=dtype), None, None, None


def embedding(tokens, weight, *, scale: float = 1.0, padding: int | None = None, dtype=None):
    """Differentiable ``daf.embedding``: scale * weight[tokens].  The row of the padding token takes no gradient."""
    return _Embedding.apply(tokens, weight, scale, padding, dtype)


class _RotaryNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, q_weight, k_weight, positions, how):
        ctx.set_materialize_grads(False)
        at = positions if isinstance(positions, torch.Tensor) else None
        ctx.save_for_backward(q, k, q_weight, k_weight, at)
        ctx.how = how if at is not None else dict(how, positions=positions)
        out = _rotary_norm(q, k, q_weight, k_weight, **dict(how, positions=positions))
        return out if k is not None else out[0]

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_q, grad_k=None):
        q, k, q_weight, k_weight, at = ctx.saved_tensors
        how = ctx.how if at is None else dict(ctx.how, positions=at)
        if grad_q is None:                                          # not used
            grad_q = torch.zeros_like(q)
        if grad_k is None and k is not None:
            grad_k = torch.zeros_like(k)
        return *rotary_norm_grad(q, k, q_weight, k_weight, grad_q, grad_k, **how), None, None


def rotary_norm(q, k, q_weight=None, k_weight=None, *, positions=None, rotary_dim: int | None = None, base: float = 10000.0,
                style: str = "halves", eps: float = 1e-6, frequencies=None):
    """Differentiable ``daf.rotary_norm``: (q, k) with every head's row divided by its root mean square, times its weight, and turned
    by position; q alone where k is None."""
    return _RotaryNorm.apply(q, k, q_weight, k_weight, positions, dict(rotary_dim=rotary_dim, base=base, style=style, eps=eps, frequencies=frequencies))


def clip_grad_norm_(parameters, max_norm: float, *, eps: float = 1e-6):
    """Clips the gradients of ``parameters`` in place by their global 2-norm, two launches for all of them; returns the norm
    as a scalar tensor on the device.  Gradients with gaps in their memory are replaced by copies without first."""
    grads, parameters = [], list(parameters)
    for p in parameters:
        if p.grad is not None:
            if not (p.grad.is_contiguous() or gap_free(p.grad)):
                p.grad = p.grad.contiguous()
            grads.append(p.grad)
    if parameters and not grads:
        return torch.zeros((), dtype=torch.float32, device=parameters[0].device)
    return clip_grad_norm(grads, max_norm, eps=eps)


class ResidualNorm(torch.nn.Module):
    """The join between two blocks as a layer: forward(x, y) returns (z, h).  gate_init: a gate for each channel, starting
    there (None: no gate); post: a norm on the block's output, too."""

    def __init__(self, width: int, *, kind: str = "layer", bias: bool = True, gate_init: float | None = None, post: bool = False,
                 residual_scale: float = 1.0, eps: float = 1e-6, dtype=None, device=None):
        super().__init__()
        made = dict(dtype=dtype, device=device)
        self.kind, self.residual_scale, self.eps = kind, float(residual_scale), float(eps)
        par = torch.nn.Parameter
        self.weight = par(torch.ones(width, **made))
        self.bias = par(torch.zeros(width, **made)) if bias else None
        self.gate = par(torch.full((width,), float(gate_init), **made)) if gate_init is not None else None
        self.post_weight = par(torch.ones(width, **made)) if post else None
        self.post_bias = par(torch.zeros(width, **made)) if post and bias else None

    def forward(self, x, y):
        return residual_norm(x, y, self.weight, self.bias, gate=self.gate, post_weight=self.post_weight, post_bias=self.post_bias,
                             residual_scale=self.residual_scale, kind=self.kind, eps=self.eps)


class Embedding(torch.nn.Module):
    """A table of token vectors: forward(tokens) returns scale * weight[tokens], in ``out_dtype`` where that is given."""

    def __init__(self, vocabulary: int, width: int, *, scale: float = 1.0, padding: int | None = None, out_dtype=None, dtype=None, device=None):
        super().__init__()
        self.scale, self.padding, self.out_dtype = float(scale), padding, out_dtype
        self.weight = torch.nn.Parameter(torch.randn(vocabulary, width, dtype=dtype, device=device) / float(scale))

    def forward(self, tokens):
        return embedding(tokens, self.weight, scale=self.scale, padding=self.padding, dtype=self.out_dtype)


class Block(torch.nn.Module):
    """A transformer block between two joins: forward((x, h)) takes the residual stream and its norm and returns both.  rotary:
    queries and keys go through ``rotary_norm`` (with weights of their own) before attention."""

    def __init__(self, width: int, heads: int, hidden: int, *, kv_heads: int | None = None, causal: bool = False, rotary: bool = False,
                 base: float = 10000.0, **join):
        super().__init__()
        self.base = float(base)
        self.q_norm = torch.nn.Parameter(torch.ones(width // heads)) if rotary else None
        self.k_norm = torch.nn.Parameter(torch.ones(width // heads)) if rotary else None
        self.heads, self.kv_heads, self.dim, self.causal = heads, kv_heads or heads, width // heads, causal
        self.qkv = torch.nn.Linear(width, (heads + 2 * self.kv_heads) * self.dim)
        self.out = torch.nn.Linear(heads * self.dim, width)
        self.up, self.down = torch.nn.Linear(width, hidden), torch.nn.Linear(hidden, width)
        self.join1, self.join2 = ResidualNorm(width, **join), ResidualNorm(width, **join)

    def forward(self, x, h, key_lengths=None, positions=None):
        b, s, _ = x.shape
        qkv = self.qkv(h).view(b, s, self.heads + 2 * self.kv_heads, self.dim)
        q, k, v = qkv.split((self.heads, self.kv_heads, self.kv_heads), 2)       # slices of one projection, read in place
        if self.q_norm is not None:
            q, k = rotary_norm(q, k, self.q_norm, self.k_norm, positions=positions, base=self.base)
        a = attention(q, k, v, causal=self.causal, key_lengths=key_lengths)
        x, h = self.join1(x, self.out(a.reshape(b, s, -1)))
        return self.join2(x, self.down(torch.nn.functional.gelu(self.up(h))))


class Classifier(torch.nn.Module):
    """Sequences of feature vectors in, class scores out: projection, blocks, mean over the tokens (the first
    key_lengths of each sequence), head."""

    def __init__(self, features: int, classes: int, tokens: int, width: int = 256, heads: int = 4, blocks: int = 4, hidden: int = 1024, **block):
        super().__init__()
        self.embed = torch.nn.Linear(features, width)
        self.place = torch.nn.Parameter(0.02 * torch.randn(1, tokens, width))
        self.first = torch.nn.LayerNorm(width)
        self.blocks = torch.nn.ModuleList(Block(width, heads, hidden, **block) for _ in range(blocks))
        self.head = torch.nn.Linear(width, classes)

    def forward(self, inputs, key_lengths=None):
        x = self.embed(inputs) + self.place.to(inputs.dtype)
        h = self.first(x)
        for block in self.blocks:
            x, h = block(x, h, key_lengths)
        if key_lengths is None:
            return self.head(h.mean(1))
        n = key_lengths.clamp(0, h.shape[1])[:, None]                # the padding takes no part
        here = torch.arange(h.shape[1], device=h.device) < n
        return self.head(h.where(here[..., None], 0).sum(1) / n.clamp(min=1).to(h.dtype))


class LanguageModel(torch.nn.Module):
    """Tokens in, scores of the next token out: embedding, causal blocks with rotary norms, head."""

    def __init__(self, vocabulary: int, width: int = 256, heads: int = 4, blocks: int = 4, hidden: int = 1024, *, padding: int | None = None, **block):
        super().__init__()
        self.embed = Embedding(vocabulary, width, padding=padding)
        self.first = torch.nn.LayerNorm(width)
        self.blocks = torch.nn.ModuleList(Block(width, heads, hidden, causal=True, rotary=True, **block) for _ in range(blocks))
        self.head = torch.nn.Linear(width, vocabulary, bias=False)

    def forward(self, tokens, key_lengths=None, positions=None):
        x = self.embed(tokens)
        h = self.first(x)
        for block in self.blocks:
            x, h = block(x, h, key_lengths, positions)
        return self.head(h)


class Muon(torch.optim.Optimizer):
    """Momentum whose steps are orthogonalised (``daf.orthogonalize``), for the matrices between a model's input and output:
    buffer = momentum * buffer + gradient, update = gradient + momentum * buffer (nesterov) or buffer, and
    p = (1 - lr * weight_decay) p - lr * sqrt(max(1, rows / columns)) * orthogonalised(update).
    Dimensions behind the first count as columns.  Buffers are float32; the matrices are orthogonalised in ``dtype``, all of a
    group on one device in one call."""

    def __init__(self, params, lr: float = 0.02, *, momentum: float = 0.95, nesterov: bool = True, weight_decay: float = 0.0, steps: int = 5,
                 dtype=torch.bfloat16):
        if lr < 0 or not 0 <= momentum < 1 or weight_decay < 0:
            raise ValueError("Muon: lr and weight_decay are not negative, momentum is in [0, 1)")
        super().__init__(params, dict(lr=lr, momentum=momentum, nesterov=nesterov, weight_decay=weight_decay, steps=steps, dtype=dtype))

    def add_param_group(self, param_group):
        super().add_param_group(param_group)
        if any(p.dim() < 2 for p in self.param_groups[-1]["params"]):
            self.param_groups.pop()
            raise ValueError("Muon: steps matrices; give vectors to another optimizer")

    def load_state_dict(self, state_dict):
        super().load_state_dict(state_dict)                         # takes states in their parameter's type
        saved = [i for g in state_dict["param_groups"] for i in g["params"]]
        for i, p in zip(saved, [p for g in self.param_groups for p in g["params"]]):
            if "momentum" in state_dict["state"].get(i, {}):
                self.state[p]["momentum"] = state_dict["state"][i]["momentum"].to(p.device, torch.float32, copy=True)

    @torch.no_grad()
    def step(self, closure=None):
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        for group in self.param_groups:
            devices = {}
            for p in group["params"]:
                if p.grad is not None and p.numel():
                    devices.setdefault(p.device, []).append(p)
            for params in devices.values():
                self._step(params, group)
        return loss

    def _step(self, params, group):
        grads = [p.grad.float() for p in params]
        for p in params:
            if "momentum" not in self.state[p]:
                self.state[p]["momentum"] = torch.zeros_like(p, dtype=torch.float32, memory_format=torch.contiguous_format)
        buffers = [self.state[p]["momentum"] for p in params]
        torch._foreach_mul_(buffers, group["momentum"])
        torch._foreach_add_(buffers, grads)
        updates = torch._foreach_add(grads, buffers, alpha=group["momentum"]) if group["nesterov"] else buffers
        made = orthogonalize([u.to(group["dtype"]).contiguous() for u in updates], steps=group["steps"])
        if group["weight_decay"]:
            torch._foreach_mul_(params, 1.0 - group["lr"] * group["weight_decay"])
        for p, u in zip(params, made):
            p.add_(u, alpha=-group["lr"] * math.sqrt(max(1.0, p.shape[0] * p.shape[0] / p.numel())))


def train_language(steps: int = 20, *, compressed: bool = True, bit_budget: float = 8.0, batch: int = 16, tokens: int = 256, vocabulary: int = 4096,
                   dtype=torch.bfloat16, max_norm: float = 1.0, seed: int = 0, lr: float = 0.02):
    """Trains the language model on synthetic sequences, each token of which follows from the one before it most of the time;
    a tenth of the batch is padding.  Returns losses and gradient norms."""
    from .autograd import saved_activation_compression
    torch.manual_seed(seed)
    net = LanguageModel(vocabulary, padding=0, gate_init=0.5).to("cuda", dtype)
    matrices = [p for p in net.blocks.parameters() if p.dim() >= 2]
    chosen = {id(p) for p in matrices}
    optimizers = [Muon(matrices, lr), torch.optim.AdamW([p for p in net.parameters() if id(p) not in chosen], lr=lr / 10)]
    ctx = saved_activation_compression(group_size=256, bit_budget=bit_budget, seed=seed) if compressed else None
    losses, gen = [], torch.Generator(device="cuda").manual_seed(seed + 1)
    follows = torch.randperm(vocabulary - 1, generator=gen, device="cuda") + 1
    for step in range(steps):
        text = torch.randint(1, vocabulary, (batch, tokens + 1), generator=gen, device="cuda")
        surprise = torch.rand((batch, tokens), generator=gen, device="cuda") < 0.1
        for i in range(tokens):
            text[:, i + 1] = torch.where(surprise[:, i], text[:, i + 1], follows[text[:, i] - 1])
        lengths = torch.full((batch,), tokens, dtype=torch.int32, device="cuda")
        lengths[: max(1, batch // 5)] = tokens // 2
        here = torch.arange(tokens, device="cuda") < lengths[:, None]
        inputs, targets = text[:, :-1].where(here, 0), text[:, 1:].where(here, -100)

        def loss_of():
            return torch.nn.functional.cross_entropy(net(inputs, lengths).float().flatten(0, 1), targets.flatten())
        if ctx is not None:
            ctx.reseed(seed + step)
            with ctx:
                loss = loss_of()
        else:
            loss = loss_of()
        for o in optimizers:
            o.zero_grad(set_to_none=True)
        loss.backward()
        norm = clip_grad_norm_(net.parameters(), max_norm)
        for o in optimizers:
            o.step()
        losses.append((loss.detach(), norm))
    if ctx is not None:
        ctx.check_status()
    check_device()
    return [(float(a), float(b)) for a, b in losses]


def train(steps: int = 20, *, compressed: bool = True, bit_budget: float = 8.0, batch: int = 64, tokens: int = 197, dtype=torch.bfloat16,
          max_norm: float = 1.0, seed: int = 0, lr: float = 0.01):
    """Trains the classifier on synthetic sequences whose class is a direction in feature space; returns the losses."""
    from .autograd import saved_activation_compression
    torch.manual_seed(seed)
    features, classes = 48, 10
    net = Classifier(features, classes, tokens, gate_init=0.5).to("cuda", dtype)
    directions = torch.randn(classes, features, device="cuda")
    sgd = torch.optim.SGD(net.parameters(), lr=lr, momentum=0.9)
    ctx = saved_activation_compression(group_size=256, bit_budget=bit_budget, seed=seed) if compressed else None
    losses, gen = [], torch.Generator(device="cuda").manual_seed(seed + 1)
    for step in range(steps):
        labels = torch.randint(classes, (batch,), generator=gen, device="cuda")
        noise = torch.randn((batch, tokens, features), generator=gen, device="cuda")
        inputs = (noise + 0.5 * directions[labels][:, None]).to(dtype)
        if ctx is not None:
            ctx.reseed(seed + step)
            with ctx:
                loss = torch.nn.functional.cross_entropy(net(inputs).float(), labels)
        else:
            loss = torch.nn.functional.cross_entropy(net(inputs).float(), labels)
        sgd.zero_grad(set_to_none=True)
        loss.backward()
        norm = clip_grad_norm_(net.parameters(), max_norm)
        sgd.step()
        losses.append((loss.detach(), norm))
    if ctx is not None:
        ctx.check_status()
    check_device()
    return [(float(a), float(b)) for a, b in losses]


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--plain", action="store_true", help="keep activations uncompressed")
    ap.add_argument("--bit-budget", type=float, default=8.0)
    ap.add_argument("--language", action="store_true", help="a language model on tokens instead of the classifier on vectors")
    ap.add_argument("--batch", type=int, help="64 sequences, 16 of the language model's")
    ap.add_argument("--tokens", type=int, help="197 of a sequence, 256 of the language model's")
    a = ap.parse_args()
    sizes = {n: getattr(a, n) for n in ("batch", "tokens") if getattr(a, n) is not None}
    for i, (loss, norm) in enumerate((train_language if a.language else train)(a.steps, compressed=not a.plain, bit_budget=a.bit_budget, **sizes)):
        assert math.isfinite(loss), "the loss is not a number"
        print(f"step {i:3d}  loss {loss:.4f}  gradient norm {norm:.3f}")


if __name__ == "__main__":
    main()
