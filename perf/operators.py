"""Cases of the transformer training operators: attention with a recomputing backward pass, the residual join with
its norms, and clipping by the global gradient norm.

``listed()`` names the cases, ``draw()`` gives more of the same ranges, ``prepare()`` makes a case's inputs on the GPU,
``run()`` does one pass -- in elementary torch operations, or with ``own`` set through the library's kernels --,
``exact()`` gives the same outputs from the definitions in 64 bits and ``work()`` the bytes and operations of a pass.

The operators (the formulas are written out at ``_attention_plain`` and the functions after it):

  attention   q [B, Sq, H, D], k and v [B, Sk, Hkv, D]; query head h reads key head h // (H / Hkv).  Query i sees key j
              if j < length[b] (all keys without lengths) and, when causal, j <= i + Sk - Sq.
  join        z = x + residual_scale * gate * post_norm(y), h = norm(z) over rows of the last dimension.
  clip        one norm over all tensors; every tensor times min(1, max_norm / (norm + 1e-6)).
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "f16": 2, "bf16": 2}


def _attention(name, mode, dtype, batch, queries, keys, heads, kv_heads, dim, causal=False, packed=False, lengths="all"):
    return {"name": name, "op": "attention", "mode": mode, "dtype": dtype, "batch": batch, "queries": queries, "keys": keys,
            "heads": heads, "kv_heads": kv_heads, "dim": dim, "causal": causal, "packed": packed, "lengths": lengths}


def _join(name, mode, dtype, rows, width, kind, params, post, gates, bias):
    return {"name": name, "op": "join", "mode": mode, "dtype": dtype, "rows": rows, "width": width, "kind": kind,
            "params": params, "post": post, "gates": gates, "bias": bias}


def _clip(name, tensors, dtype, layers, width, hidden, max_norm):
    return {"name": name, "op": "clip", "tensors": tensors, "dtype": dtype, "layers": layers, "width": width,
            "hidden": hidden, "max_norm": max_norm}


def listed():
    return [
        # one short sequence of a small model, forward: what a call costs when there is next to nothing to compute
        _attention("attention_small_fwd", "fwd", "bf16", 1, 61, 61, 4, 4, 64, causal=True),
        # the ViT-B/16 batch of the activation workloads (64 images, 197 tokens, 12 heads of 64), q, k and v as the
        # slices of one projection's output: both directions
        _attention("attention_vit_fwd", "fwd", "bf16", 64, 197, 197, 12, 12, 64, packed=True),
        _attention("attention_vit_bwd", "bwd", "bf16", 64, 197, 197, 12, 12, 64, packed=True),
        # a padded batch of sentences: every sequence has its own length (one is empty), an odd head size
        _attention("attention_padded_bwd", "bwd", "f16", 16, 509, 509, 16, 16, 80, lengths="spread"),
        # full precision fine-tuning on images
        _attention("attention_f32_bwd", "bwd", "f32", 8, 197, 197, 12, 12, 64, packed=True),
        # a long causal sequence with four query heads to a key head, the largest attention: both directions
        _attention("attention_long_fwd", "fwd", "bf16", 1, 8192, 8192, 16, 4, 128, causal=True),
        _attention("attention_long_bwd", "bwd", "bf16", 1, 8192, 8192, 16, 4, 128, causal=True),
        # the join of one image in full precision: layer norm, a gate for each channel
        _join("join_image_fwd", "fwd", "f32", 197, 768, "layer", "f32", False, 1, True),
        # the join of the ViT-B/16 batch, activations in 16 bits and parameters in 32: backward
        _join("join_vit_bwd", "bwd", "bf16", 64 * 197, 768, "layer", "f32", False, 1, True),
        # a wide model with norms on both sides of the block and a gate for each of 8 sequences
        _join("join_wide_bwd", "bwd", "bf16", 16384, 4096, "rms", "same", True, 8, False),
        # the gradients of ResNet-18 (62 tensors, the smallest of 64 values) in full precision
        _clip("clip_resnet18", "resnet18", "f32", 0, 0, 0, 1.0),
        # a transformer's gradients in 16 bits: 0.4 G values
        _clip("clip_transformer", "transformer", "bf16", 8, 2048, 8192, 0.5),
    ]


def _log_int(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["attention", "attention", "attention", "join", "join", "clip"])
    if op == "attention":
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        dim = rng.choice([32, 40, 64, 64, 72, 80, 96, 128, 128])
        kv_heads = rng.choice([1, 2, 3, 4, 8, 12])
        group = rng.choice([1, 1, 2, 4]) if kv_heads <= 8 else 1
        batch = _log_int(rng, 1, 64)
        keys = _log_int(rng, 1, 8192)
        queries = keys if rng.random() < 0.7 else _log_int(rng, 1, 8192)
        most = 2 ** 37 if dtype != "f32" else 2 ** 33          # B * H * Sq * Sk * D of the largest case, and of full precision
        while batch * kv_heads * group * queries * keys * dim > most or batch * kv_heads * group * queries * keys > 2 ** 30:
            if batch > 1:
                batch = max(1, batch // 2)
            else:
                queries, keys = max(1, queries * 2 // 3), max(1, keys * 2 // 3)
        return {k: v for k, v in _attention("", rng.choice(["fwd", "bwd"]), dtype, batch, queries, keys, kv_heads * group, kv_heads,
                                            dim, causal=rng.random() < 0.5, packed=group == 1 and queries == keys and rng.random() < 0.5,
                                            lengths="spread" if rng.random() < 0.3 else "all").items() if k != "name"}
    if op == "join":
        width = 8 * _log_int(rng, 8, 1024)
        rows = max(1, min(_log_int(rng, 1, 65536), 16384 * 4096 // width))
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        gates = rng.choice([0, 1, 1, 4])
        rows = max(4, rows // 4 * 4) if gates == 4 else rows
        return {k: v for k, v in _join("", rng.choice(["fwd", "bwd", "bwd"]), dtype, rows, width, rng.choice(["layer", "rms"]),
                                       rng.choice(["f32", "same"]), rng.random() < 0.5, gates, rng.random() < 0.5).items() if k != "name"}
    return {k: v for k, v in _clip("", "transformer", rng.choice(["bf16", "f16", "f32"]), rng.randint(1, 8), 8 * _log_int(rng, 8, 192) + rng.choice([0, 1]),
                                   _log_int(rng, 100, 4096), rng.choice([0.1, 1.0, 1e6])).items() if k != "name"}


# ---------------------------------------------------------------------------------------------------- inputs
def _randn(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * scale).to(dtype)


def _lengths(case):
    """Keys of each sequence: all of them, or spread from none to all over the batch (a batch of one keeps two thirds)."""
    b, s = case["batch"], case["keys"]
    if case["lengths"] == "all":
        return [s] * b
    return [s * i // (b - 1) for i in range(b)] if b > 1 else [max(1, 2 * s // 3)]


def _clip_shapes(case):
    if case["tensors"] == "resnet18":
        def unit(c_in, c_out):
            return [(c_out, c_in, 3, 3), (c_out,), (c_out,), (c_out, c_out, 3, 3), (c_out,), (c_out,)]
        shapes = [(64, 3, 7, 7), (64,), (64,)] + unit(64, 64) * 2
        for c in (128, 256, 512):
            shapes += unit(c // 2, c) + [(c, c // 2, 1, 1), (c,), (c,)] + unit(c, c)
        return shapes + [(1000, 512), (1000,)]
    w, f = case["width"], case["hidden"]
    return [(3 * w, w), (w, w), (w,), (w,), (f, w), (w, f), (f,)] * case["layers"]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    s = dict(case)
    if case["op"] == "attention":
        dt, b, h, kv, d = _TYPES[case["dtype"]], case["batch"], case["heads"], case["kv_heads"], case["dim"]
        if case["packed"]:
            s["q"], s["k"], s["v"] = _randn(g, (b, case["keys"], 3, h, d), dt).unbind(2)
        else:
            s["q"] = _randn(g, (b, case["queries"], h, d), dt)
            s["k"], s["v"] = (_randn(g, (b, case["keys"], kv, d), dt) for _ in range(2))
        lens = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda")
        s["key_lengths"] = lens if case["lengths"] != "all" else None
        if case["mode"] == "bwd":                                  # what the forward pass of the step has left
            s["grad_out"] = _randn(g, (b, case["queries"], h, d), dt)
            out, s["lse"] = _attention_plain(s)
            s["out"] = out.to(dt)
    elif case["op"] == "join":
        dt = _TYPES[case["dtype"]]
        pt = torch.float32 if case["params"] == "f32" else dt
        n, c = case["rows"], case["width"]
        s["x"], s["y"] = _randn(g, (n, c), dt, 2.0), _randn(g, (n, c), dt, 0.7)     # x: the stream, or in "bwd" the stream behind the join
        s["weight"] = (1 + 0.2 * _randn(g, (c,), torch.float32)).to(pt)
        s["bias_"] = _randn(g, (c,), pt, 0.1) if case["bias"] else None
        s["post_weight"] = (0.5 + 0.1 * _randn(g, (c,), torch.float32)).to(pt) if case["post"] else None
        s["post_bias"] = _randn(g, (c,), pt, 0.1) if case["post"] and case["bias"] else None
        s["gate"] = _randn(g, (c,) if case["gates"] == 1 else (case["gates"], c), pt, 0.5) if case["gates"] else None
        s["residual_scale"] = 0.75
        if case["mode"] == "bwd":
            s["grad_z"], s["grad_h"] = _randn(g, (n, c), dt, 0.3), _randn(g, (n, c), dt)
    else:
        dt = _TYPES[case["dtype"]]
        s["grads"] = [_randn(g, shape, dt, 0.01) for shape in _clip_shapes(case)]
        s["out"] = [torch.empty_like(t) for t in s["grads"]]
    return s


# ---------------------------------------------------------------------------------------------------- the plain forms
def _by_kv_head(t, kv):
    """[B, S, H, D] as [B, Hkv, H / Hkv, S, D] in 32 bits."""
    b, n, h, d = t.shape
    return t.float().reshape(b, n, kv, h // kv, d).permute(0, 2, 3, 1, 4)


def _visible(s):
    """[B, 1, 1, Sq, Sk] truth values, or None where every query sees every key."""
    sq, sk = s["q"].shape[1], s["k"].shape[1]
    j = torch.arange(sk, device="cuda")
    see = None
    if s["causal"]:
        see = (j <= torch.arange(sq, device="cuda")[:, None] + (sk - sq))[None, None, None]
    if s["key_lengths"] is not None:
        short = (j < s["key_lengths"][:, None])[:, None, None, None]
        see = short if see is None else see & short
    return see


def _attention_plain(s):
    """out = softmax(q k^T / sqrt(D)) v over the visible keys (zero where there are none), and the logarithm of each
    row's sum of exponentials, [B, H, Sq]."""
    kv = s["k"].shape[2]
    q, k, v = (_by_kv_head(s[n], kv) for n in "qkv")
    see = _visible(s)
    scores = torch.matmul(q, k.transpose(-1, -2)) * (1.0 / math.sqrt(q.shape[-1]))
    if see is not None:
        scores = scores.masked_fill(~see, -math.inf)
    top = scores.amax(-1, keepdim=True).clamp_min(-1e30)
    p = torch.exp(scores - top)
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, v) / torch.where(total > 0, total, 1.0)
    lse = (top + torch.log(total)).squeeze(-1)
    return out.permute(0, 3, 1, 2, 4).reshape(s["q"].shape), lse.reshape(lse.shape[0], -1, lse.shape[-1])


def _attention_grad_plain(s):
    """p = exp(q k^T / sqrt(D) - lse), delta = sum(grad_out * out), ds = p * (grad_out v^T - delta) / sqrt(D):
    dq = ds k, dk = ds^T q, dv = p^T grad_out, the last two summed over the query heads of a key head."""
    kv = s["k"].shape[2]
    q, k, v, o, g = (_by_kv_head(s[n], kv) for n in ("q", "k", "v", "out", "grad_out"))
    see = _visible(s)
    scale = 1.0 / math.sqrt(q.shape[-1])
    p = torch.exp(torch.matmul(q, k.transpose(-1, -2)) * scale - s["lse"].view(*q.shape[:-1], 1))
    if see is not None:
        p = torch.where(see, p, 0.0)
    ds = p * (torch.matmul(g, v.transpose(-1, -2)) - (g * o).sum(-1, keepdim=True)) * scale
    dq = torch.matmul(ds, k).permute(0, 3, 1, 2, 4).reshape(s["q"].shape)
    dk = torch.matmul(ds.transpose(-1, -2), q).sum(2).permute(0, 2, 1, 3)
    dv = torch.matmul(p.transpose(-1, -2), g).sum(2).permute(0, 2, 1, 3)
    return dq, dk, dv


def _normed(t, kind, eps=1e-6):
    """(t - mean) * r and r, with r = 1 / sqrt(mean((t - mean)^2) + eps); the mean counts as zero for "rms"."""
    t = t - t.mean(-1, keepdim=True) if kind == "layer" else t
    r = torch.rsqrt((t * t).mean(-1, keepdim=True) + eps)
    return t * r, r


def _by_row(gate, rows):
    """A gate for each row: one for all, or one for each run of rows / G rows."""
    return gate.float() if gate.dim() == 1 else gate.float().repeat_interleave(rows // gate.shape[0], 0)


def _join_plain(s):
    u = s["y"].float()
    if s["post_weight"] is not None:
        u = _normed(u, s["kind"])[0] * s["post_weight"].float()
        u = u + s["post_bias"].float() if s["post_bias"] is not None else u
    if s["gate"] is not None:
        u = u * _by_row(s["gate"], u.shape[0])
    z = s["x"].float() + s["residual_scale"] * u
    h = _normed(z, s["kind"])[0] * s["weight"].float()
    return z, h + s["bias_"].float() if s["bias_"] is not None else h


def _norm_grad(hat, r, g, kind):
    """The gradient of hat = (t - mean) * r with respect to t, for the gradient g of hat."""
    g0 = g - g.mean(-1, keepdim=True) if kind == "layer" else g
    return r * (g0 - hat * (g * hat).mean(-1, keepdim=True))


def _join_grad_plain(s):
    """From z (here "x"), y and the gradients of z and h: those of x, y, weight, bias, gate, post_weight and post_bias."""
    a, rows = s["residual_scale"], s["x"].shape[0]
    hat, r = _normed(s["x"].float(), s["kind"])
    gh = s["grad_h"].float()
    dx = s["grad_z"].float() + _norm_grad(hat, r, gh * s["weight"].float(), s["kind"])
    out = {"x": dx, "weight": (gh * hat).sum(0)}
    if s["bias_"] is not None:
        out["bias"] = gh.sum(0)
    du = a * dx
    y = s["y"].float()
    post = s["post_weight"] is not None
    yhat, ry = _normed(y, s["kind"]) if post else (y, None)
    if s["gate"] is not None:
        u = yhat * s["post_weight"].float() if post else y
        u = u + s["post_bias"].float() if s["post_bias"] is not None else u
        each = du * u
        out["gate"] = each.sum(0) if s["gate"].dim() == 1 else each.view(s["gate"].shape[0], -1, each.shape[-1]).sum(1)
        du = du * _by_row(s["gate"], rows)
    if post:
        out["post_weight"] = (du * yhat).sum(0)
        if s["post_bias"] is not None:
            out["post_bias"] = du.sum(0)
        du = _norm_grad(yhat, ry, du * s["post_weight"].float(), s["kind"])
    out["y"] = du
    return out


def _clip_plain(s):
    norm = torch.sqrt(torch.stack([t.float().square().sum() for t in s["grads"]]).sum())
    by = (s["max_norm"] / (norm + 1e-6)).clamp(max=1.0)
    return norm, [o.copy_(t.float() * by) for t, o in zip(s["grads"], s["out"])]


def run(s):
    if own:
        return _run_own(s)
    if s["op"] == "attention":
        dt = s["q"].dtype
        if s["mode"] == "fwd":
            out, lse = _attention_plain(s)
            return {"out": out.to(dt), "lse": lse}
        dq, dk, dv = _attention_grad_plain(s)
        return {"q": dq.to(dt), "k": dk.to(dt), "v": dv.to(dt)}
    if s["op"] == "join":
        dt = s["x"].dtype
        if s["mode"] == "fwd":
            z, h = _join_plain(s)
            return {"z": z.to(dt), "h": h.to(dt)}
        return {n: t.to(dt if n in ("x", "y") else s["weight"].dtype) for n, t in _join_grad_plain(s).items()}
    norm, out = _clip_plain(s)
    return {"norm": norm, "out": out}


def _run_own(s):
    import paper_2507_07149_b200 as daf
    if s["op"] == "attention":
        how = {"causal": s["causal"], "key_lengths": s["key_lengths"]}
        if s["mode"] == "fwd":
            out, lse = daf.attention(s["q"], s["k"], s["v"], **how)
            return {"out": out, "lse": lse}
        dq, dk, dv = daf.attention_grad(s["q"], s["k"], s["v"], s["out"], s["lse"], s["grad_out"], **how)
        return {"q": dq, "k": dk, "v": dv}
    if s["op"] == "join":
        how = {"gate": s["gate"], "post_weight": s["post_weight"], "post_bias": s["post_bias"],
               "residual_scale": s["residual_scale"], "kind": s["kind"]}
        if s["mode"] == "fwd":
            z, h = daf.residual_norm(s["x"], s["y"], s["weight"], s["bias_"], **how)
            return {"z": z, "h": h}
        grads = daf.residual_norm_grad(s["x"], s["y"], s["weight"], s["bias_"], s["grad_z"], s["grad_h"], **how)
        return {n: t for n, t in grads.items() if t is not None}
    norm = daf.clip_grad_norm(s["grads"], s["max_norm"], out=s["out"])
    return {"norm": norm, "out": s["out"]}


# ---------------------------------------------------------------------------------------------------- what a pass costs
def work(case):
    if case["op"] == "attention":
        b, sq, sk, h, kv, d = (case[n] for n in ("batch", "queries", "keys", "heads", "kv_heads", "dim"))
        if case["causal"]:                                         # visible pairs of a sequence of `n` keys: row i sees clip(i + 1 + sk - sq, 0, n)
            pairs = sum(sum(min(n, max(0, i + 1 + sk - sq)) for i in range(sq)) for n in _lengths(case))
        else:
            pairs = sum(sq * n for n in _lengths(case))
        e = _BYTES[case["dtype"]]
        keys = sum(_lengths(case))
        q, k = b * sq * h * d * e, keys * kv * d * e
        if case["mode"] == "fwd":
            return {"bytes": 2 * q + 2 * k + 4 * b * h * sq, "flops": 4 * d * h * pairs}
        return {"bytes": 4 * q + 2 * k + 2 * b * sk * kv * d * e + 4 * b * h * sq, "flops": 10 * d * h * pairs}
    if case["op"] == "join":
        n, c = case["rows"] * case["width"], case["width"]
        e = _BYTES[case["dtype"]]
        vectors = 1 + case["bias"] + case["gates"] + (1 + case["bias"]) * case["post"]
        p = (4 if case["params"] == "f32" else e) * c * vectors
        if case["mode"] == "fwd":
            return {"bytes": 4 * n * e + p, "flops": 12 * n}
        return {"bytes": 6 * n * e + 2 * p, "flops": 30 * n}
    n = sum(math.prod(shape) for shape in _clip_shapes(case))
    return {"bytes": 2 * n * _BYTES[case["dtype"]], "flops": 3 * n}


# ---------------------------------------------------------------------------------------------------- in 64 bits
def _exact_attention(case, s):
    b, sq, sk, h, kv, d = (case[n] for n in ("batch", "queries", "keys", "heads", "kv_heads", "dim"))
    bwd = case["mode"] == "bwd"
    made = {n: torch.zeros(s[n].shape, dtype=torch.float64, device="cuda") for n in ("q", "k", "v")}
    lse = torch.full((b, h, sq), -math.inf, dtype=torch.float64, device="cuda")
    for i, n in enumerate(_lengths(case)):
        for e in range(kv if n else 0):
            k, v = s["k"][i, :n, e].double(), s["v"][i, :n, e].double()
            hs = range(e * (h // kv), (e + 1) * (h // kv))
            for a in hs:
                w = s["q"][i, :, a].double() @ k.t() / math.sqrt(d)
                if case["causal"]:
                    w = w.masked_fill(torch.triu(torch.ones(sq, n, dtype=torch.bool, device="cuda"), 1 + sk - sq), -math.inf)
                if not bwd:
                    lse[i, a] = torch.logsumexp(w, 1)
                    made["q"][i, :, a] = torch.nan_to_num(torch.exp(w - lse[i, a][:, None]), nan=0.0) @ v
                    continue
                p = torch.exp(w - s["lse"][i, a].double()[:, None])
                p = torch.nan_to_num(p, nan=0.0, posinf=0.0)       # rows that see nothing: lse is minus infinity
                g = s["grad_out"][i, :, a].double()
                ds = p * (g @ v.t() - (g * s["out"][i, :, a].double()).sum(1, keepdim=True)) / math.sqrt(d)
                made["q"][i, :, a] = ds @ k
                made["k"][i, :n, e] += ds.t() @ s["q"][i, :, a].double()
                made["v"][i, :n, e] += p.t() @ g
    return made if bwd else {"out": made["q"], "lse": lse}


def _exact_join(case, s):
    def stats(t):
        m = t.mean(1, keepdim=True) if case["kind"] == "layer" else torch.zeros_like(t[:, :1])
        return m, 1 / torch.sqrt(((t - m) ** 2).mean(1, keepdim=True) + 1e-6)

    def vector(n, fill):
        return s[n].double() if s[n] is not None else torch.full((case["width"],), fill, dtype=torch.float64, device="cuda")

    c, rows, a = case["width"], case["rows"], s["residual_scale"]
    x, y, w = s["x"].double(), s["y"].double(), s["weight"].double()
    gate = vector("gate", 1.0)
    per_row = gate.view(-1, 1, c).expand(-1, rows // (gate.numel() // c), c).reshape(-1, c) if gate.dim() == 2 else gate
    w1, b1 = vector("post_weight", 1.0), vector("post_bias", 0.0)
    my, ry = stats(y) if case["post"] else (0.0, 1.0)
    yhat = (y - my) * ry
    if case["mode"] == "fwd":
        z = x + a * per_row * (yhat * w1 + b1)
        m, r = stats(z)
        return {"z": z, "h": (z - m) * r * w + vector("bias_", 0.0)}
    m, r = stats(x)
    hat, gh = (x - m) * r, s["grad_h"].double()
    t = gh * w
    centre = t.sum(1, keepdim=True) / c if case["kind"] == "layer" else 0.0
    dx = s["grad_z"].double() + r * (t - centre - hat * (t * hat).sum(1, keepdim=True) / c)
    out = {"x": dx, "weight": (gh * hat).sum(0)}
    if case["bias"]:
        out["bias"] = gh.sum(0)
    if case["gates"]:
        out["gate"] = (a * dx * (yhat * w1 + b1)).view(case["gates"], -1, c).sum(1).view(gate.shape)
    d = a * per_row * dx
    if case["post"]:
        out["post_weight"] = (d * yhat).sum(0)
        if case["bias"]:
            out["post_bias"] = d.sum(0)
        t = d * w1
        centre = t.sum(1, keepdim=True) / c if case["kind"] == "layer" else 0.0
        d = ry * (t - centre - yhat * (t * yhat).sum(1, keepdim=True) / c)
    out["y"] = d
    return out


def exact(case, seed):
    if case["op"] == "attention" and case["batch"] * case["heads"] > 8192:
        return None
    s = prepare(case, seed)
    if case["op"] == "attention":
        return _exact_attention(case, s)
    if case["op"] == "join":
        return _exact_join(case, s)
    norm = math.sqrt(sum(float(t.double().pow(2).sum()) for t in s["grads"]))
    by = min(1.0, case["max_norm"] / (norm + 1e-6))
    return {"norm": torch.tensor(norm, dtype=torch.float64), "out": [t.double() * by for t in s["grads"]]}
