"""Cases of the operators of a language model's training step: the token embedding and its gradient, norms of queries and
keys for each head with the rotation by position in the same pass and their gradient, and the orthogonalised update.

``listed()`` names the cases, ``draw()`` gives more of the same ranges, ``prepare()`` makes a case's inputs on the GPU,
``run()`` does one pass -- in elementary torch operations, or with ``own`` set through the library's kernels --,
``exact()`` gives the same outputs from the definitions in 64 bits and ``work()`` the bytes and operations of a pass.

  embedding      out[t] = scale * weight[token[t]]; backward: grad_weight[v] = scale * sum of grad_out[t] over the tokens
                 that are v (none for the padding token), zero for rows that no token names.
  rotary         for every token and head, x a row of q or k: n = x / sqrt(mean(x^2) + eps) * weight, then the first
                 `rotary` elements in pairs (i, i + rotary / 2) or (2 i, 2 i + 1) turned by position * base^(-2 i / rotary).
  orthogonal     x = g / (|g| + eps), five times x = a x + (b x x^T + c (x x^T)^2) x: the odd polynomial that takes the
                 singular values of g towards one, for every matrix of a list.
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "f16": 2, "bf16": 2}
_A, _B, _C = 3.4445, -4.7750, 2.0315


def _embedding(name, mode, dtype, table, tokens, vocabulary, width, ids="i64", padding=False, scale=1.0):
    return {"name": name, "op": "embedding", "mode": mode, "dtype": dtype, "table": table, "tokens": tokens,
            "vocabulary": vocabulary, "width": width, "ids": ids, "padding": padding, "scale": scale}


def _rotary(name, mode, dtype, params, batch, tokens, heads, kv_heads, dim, rotary, style="halves", packed=True, positions="row"):
    return {"name": name, "op": "rotary", "mode": mode, "dtype": dtype, "params": params, "batch": batch, "tokens": tokens,
            "heads": heads, "kv_heads": kv_heads, "dim": dim, "rotary": rotary, "style": style, "packed": packed,
            "positions": positions}


def _orthogonal(name, dtype, shapes, layers=1):
    return {"name": name, "op": "orthogonal", "dtype": dtype, "shapes": shapes, "layers": layers}


def listed():
    return [
        # one short prompt of a small model: what a call costs when there is next to nothing to copy
        _embedding("embedding_small_fwd", "fwd", "bf16", "bf16", 61, 4096, 256),
        # the gradient of an ordinary batch (64 sequences of 256 tokens, a tenth of them padding) into a 16-bit table
        _embedding("embedding_batch_bwd", "bwd", "bf16", "bf16", 16384, 32000, 768, padding=True),
        # a large batch and a large table: 16-bit activations from parameters in 32 bits, both directions
        _embedding("embedding_large_fwd", "fwd", "bf16", "f32", 131072, 128000, 2048, ids="i32", scale=math.sqrt(2048)),
        _embedding("embedding_large_bwd", "bwd", "bf16", "f32", 131072, 128000, 2048, ids="i32", scale=math.sqrt(2048)),
        # one new token for each of 32 sequences, every one at a far position of its own
        _rotary("rotary_token_fwd", "fwd", "bf16", "bf16", 32, 1, 16, 4, 128, 128, packed=False, positions="far"),
        # a batch of the ViT-B/16 layout (64 x 197 tokens, 12 heads of 64), slices of one projection: backward
        _rotary("rotary_batch_bwd", "bwd", "bf16", "f32", 64, 197, 12, 12, 64, 64),
        # full precision, an odd length and head size, a part of the head turned, neighbouring pairs: backward
        _rotary("rotary_odd_bwd", "bwd", "f32", "f32", 5, 509, 6, 2, 80, 32, style="pairs", packed=False),
        # long sequences, four query heads to a key head
        _rotary("rotary_long_fwd", "fwd", "bf16", "bf16", 4, 8192, 16, 4, 128, 128),
        # the matrices of the trainer's four blocks (width 256, hidden 1024): many small ones
        _orthogonal("orthogonal_trainer", "bf16", "768x256 256x256 1024x256 256x1024", 4),
        # odd sizes in full precision, a vector among them
        _orthogonal("orthogonal_odd", "f32", "333x1285 1000x512 77x77 1x300 640x640"),
        # a small model's blocks in half precision
        _orthogonal("orthogonal_half", "f16", "2304x768 768x768 768x1536", 2),
        # two blocks of a model of width 2048 and hidden size 8192
        _orthogonal("orthogonal_large", "bf16", "6144x2048 2048x2048 8192x2048 2048x8192", 2),
    ]


def _log_int(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["embedding", "embedding", "rotary", "rotary", "orthogonal"])
    if op == "embedding":
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        width = _log_int(rng, 8, 512) * rng.choice([1, 8, 8, 8]) + rng.choice([0, 0, 0, 1])
        tokens = min(_log_int(rng, 1, 262144), 131072 * 2048 // width)
        case = _embedding("", rng.choice(["fwd", "bwd", "bwd"]), dtype, rng.choice([dtype, "f32"]), tokens,
                          min(_log_int(rng, 2, 262144), 128000 * 2048 // width), width, rng.choice(["i64", "i32"]),
                          rng.random() < 0.5, rng.choice([1.0, math.sqrt(width)]))
    elif op == "rotary":
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        dim = rng.choice([32, 40, 64, 64, 72, 80, 96, 128, 128, 256])
        kv_heads = rng.choice([1, 2, 3, 4, 8, 12])
        heads = kv_heads * rng.choice([1, 1, 2, 4])
        most = 4 * 8192 * 20 * 128 // ((heads + kv_heads) * dim * (2 if dtype == "f32" else 1))
        batch = _log_int(rng, 1, 64)
        tokens = max(1, min(_log_int(rng, 1, 8192), most // batch))
        case = _rotary("", rng.choice(["fwd", "bwd", "bwd"]), dtype, rng.choice(["f32", dtype]), batch, tokens, heads, kv_heads, dim,
                       rng.choice([dim, dim, 8 * rng.randint(1, dim // 8)]), rng.choice(["halves", "halves", "pairs"]), rng.random() < 0.5,
                       rng.choice(["row", "far", "none"]))
    else:
        dtype = rng.choice(["bf16", "bf16", "bf16", "f16", "f32"])
        most = 2048 if dtype == "bf16" else 1024
        shapes = []
        for _ in range(rng.randint(1, 4)):
            small, ratio = _log_int(rng, 1, most), math.exp(rng.uniform(0, math.log(4)))
            wide = (small, max(1, int(small * ratio)))
            shapes.append("%dx%d" % (wide if rng.random() < 0.5 else wide[::-1]))
        case = _orthogonal("", dtype, " ".join(shapes), 1 if dtype != "bf16" else rng.randint(1, 2))
    return {k: v for k, v in case.items() if k != "name"}


# ---------------------------------------------------------------------------------------------------- inputs
def _randn(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * scale).to(dtype)


def _tokens(case, g):
    """Tokens as text has them: the word of rank r about 1 / r as often as the first one, a tenth of them padding where there is any."""
    n, v = case["tokens"], case["vocabulary"]
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    rank = (torch.exp(u * math.log(v)) - 1).long().clamp_(0, v - 1)
    order = torch.randperm(v, generator=g, device="cuda")                     # which token has which rank
    t = order[rank]
    if case["padding"]:
        t = torch.where(torch.rand(n, generator=g, device="cuda") < 0.1, 0, t)
    return t.to(torch.int32 if case["ids"] == "i32" else torch.int64)


def _shapes(case):
    return [tuple(int(n) for n in s.split("x")) for s in case["shapes"].split()] * case["layers"]


def _update(g, shape, dtype):
    """What an update looks like: sums of outer products over a batch, some directions far stronger than others, and noise."""
    r, c = shape
    k = max(1, min(r, c) // 4)
    strong = _randn(g, (r, k), torch.float32) / (1 + torch.arange(k, device="cuda"))
    return (0.01 * (strong @ _randn(g, (k, c), torch.float32) + 0.1 * _randn(g, shape, torch.float32))).to(dtype)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    s = dict(case)
    dt = _TYPES[case["dtype"]]
    if case["op"] == "embedding":
        s["ids_"] = _tokens(case, g)
        s["table_type"] = _TYPES[case["table"]]
        if case["mode"] == "fwd":
            s["weight"] = _randn(g, (case["vocabulary"], case["width"]), s["table_type"], 0.02)
        else:
            s["grad_out"] = _randn(g, (case["tokens"], case["width"]), dt, 0.1)
    elif case["op"] == "rotary":
        b, n, h, kv, d = (case[x] for x in ("batch", "tokens", "heads", "kv_heads", "dim"))
        pt = torch.float32 if case["params"] == "f32" else dt
        if case["packed"]:                                          # slices of one projection's output
            s["q"], s["k"], _ = _randn(g, (b, n, h + 2 * kv, d), dt).split((h, kv, kv), 2)
        else:
            s["q"], s["k"] = _randn(g, (b, n, h, d), dt, 2.0), _randn(g, (b, n, kv, d), dt, 0.5)
        s["q_weight"], s["k_weight"] = ((1 + 0.2 * _randn(g, (d,), torch.float32)).to(pt) for _ in range(2))
        at = torch.arange(n, device="cuda", dtype=torch.int32).expand(b, n)
        if case["positions"] == "far":                              # every sequence starts at a place of its own
            at = at + torch.randint(0, 1 << 20, (b, 1), generator=g, device="cuda", dtype=torch.int32)
        s["at"] = None if case["positions"] == "none" else at.contiguous()
        if case["mode"] == "bwd":
            s["grad_q"], s["grad_k"] = _randn(g, (b, n, h, d), dt), _randn(g, (b, n, kv, d), dt)
    else:
        s["updates"] = [_update(g, shape, dt) for shape in _shapes(case)]
    return s


# ---------------------------------------------------------------------------------------------------- the plain forms
def _embedding_plain(s):
    ids = s["ids_"].long()
    if s["mode"] == "fwd":
        return {"out": (s["weight"][ids].float() * s["scale"]).to(_TYPES[s["dtype"]])}
    grad = torch.zeros((s["vocabulary"], s["width"]), dtype=torch.float32, device="cuda")
    grad.index_add_(0, ids, s["grad_out"].float())
    if s["padding"]:
        grad[0] = 0
    return {"weight": (grad * s["scale"]).to(s["table_type"])}


def _turns(s):
    """Cosine and sine of every token's angles, [B, S, 1, rotary / 2]: angles of far positions need 64 bits."""
    b, n = s["q"].shape[:2]
    at = s["at"] if s["at"] is not None else torch.arange(n, device="cuda").expand(b, n)
    r = s["rotary"]
    angle = at.double()[:, :, None, None] * 10000.0 ** (-torch.arange(0, r, 2, device="cuda", dtype=torch.float64) / r)
    return torch.cos(angle).float(), torch.sin(angle).float()


def _turn(x, cos, sin, style):
    """The first elements of each row, in pairs, as complex numbers times cos + i sin; the others as they are."""
    r = 2 * cos.shape[-1]
    head = x[..., :r]
    a, b = head.chunk(2, -1) if style == "halves" else (head[..., 0::2], head[..., 1::2])
    a, b = a * cos - b * sin, a * sin + b * cos
    head = torch.cat((a, b), -1) if style == "halves" else torch.stack((a, b), -1).flatten(-2)
    return torch.cat((head, x[..., r:]), -1)


def _rotary_plain(s, eps=1e-6):
    cos, sin = _turns(s)
    out = {}
    for n in "qk":
        x, w = s[n].float(), s[n + "_weight"].float()
        hat = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + eps)
        if s["mode"] == "fwd":
            out[n] = _turn(hat * w, cos, sin, s["style"]).to(s[n].dtype)
            continue
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + eps)
        g = _turn(s["grad_" + n].float(), cos, -sin, s["style"])     # turned back
        out[n + "_weight"] = (g * hat).sum((0, 1, 2)).to(s[n + "_weight"].dtype)
        g = g * w
        out[n] = (r * (g - hat * (g * hat).mean(-1, keepdim=True))).to(s[n].dtype)
    return out


def _orthogonal_plain(g, eps=1e-7):
    wide = g.shape[0] <= g.shape[1]
    x = g.float() if wide else g.float().t()
    x = x / (g.double().square().sum().sqrt() + eps).float()
    for _ in range(5):
        gram = x @ x.t()
        x = _A * x + (_B * gram + _C * (gram @ gram)) @ x
    return (x if wide else x.t()).to(g.dtype).contiguous()


def run(s):
    if own:
        return _run_own(s)
    if s["op"] == "embedding":
        return _embedding_plain(s)
    if s["op"] == "rotary":
        return _rotary_plain(s)
    return [_orthogonal_plain(g) for g in s["updates"]]


def _run_own(s):
    import paper_2507_07149_b200 as daf
    if s["op"] == "embedding":
        if s["mode"] == "fwd":
            return {"out": daf.embedding(s["ids_"], s["weight"], scale=s["scale"], dtype=_TYPES[s["dtype"]])}
        return {"weight": daf.embedding_grad(s["ids_"], s["grad_out"], s["vocabulary"], scale=s["scale"],
                                             padding=0 if s["padding"] else None, dtype=s["table_type"])}
    if s["op"] == "rotary":
        how = {"positions": s["at"], "rotary_dim": s["rotary"], "style": s["style"]}
        if s["mode"] == "fwd":
            q, k = daf.rotary_norm(s["q"], s["k"], s["q_weight"], s["k_weight"], **how)
            return {"q": q, "k": k}
        gq, gk, gqw, gkw = daf.rotary_norm_grad(s["q"], s["k"], s["q_weight"], s["k_weight"], s["grad_q"], s["grad_k"], **how)
        return {"q": gq, "k": gk, "q_weight": gqw, "k_weight": gkw}
    return daf.orthogonalize(s["updates"])


# ---------------------------------------------------------------------------------------------------- what a pass costs
def work(case):
    if case["op"] == "embedding":
        n, v, c = case["tokens"], case["vocabulary"], case["width"]
        e, t = _BYTES[case["dtype"]], _BYTES[case["table"]]
        ids = n * (4 if case["ids"] == "i32" else 8)
        # rows that n draws name, of v whose r-th comes with a probability of log((r + 2) / (r + 1)) / log(v) or so
        named = v if v <= 2 else sum(d * (1 - (1 - math.log((m + 2) / (m + 1)) / math.log(v)) ** n) for m, d in _ranks(v))
        if case["mode"] == "fwd":
            return {"bytes": ids + int(named) * c * t + n * c * e, "flops": n * c}
        return {"bytes": ids + n * c * e + v * c * t, "flops": n * c}
    if case["op"] == "rotary":
        rows = case["batch"] * case["tokens"] * (case["heads"] + case["kv_heads"])
        n = rows * case["dim"] * _BYTES[case["dtype"]]
        at = 0 if case["positions"] == "none" else 4 * case["batch"] * case["tokens"]
        if case["mode"] == "fwd":
            return {"bytes": 2 * n + at, "flops": 7 * rows * case["dim"]}
        return {"bytes": 3 * n + at, "flops": 16 * rows * case["dim"]}
    flops = bytes_ = 0
    for r, c in _shapes(case):
        m, n = min(r, c), max(r, c)
        flops += 5 * (m * (m + 1) * n + m * (m + 1) * m + 2 * m * m * n)      # the first two products are symmetric
        bytes_ += 2 * m * n * _BYTES[case["dtype"]]
    return {"bytes": bytes_, "flops": flops}


def _ranks(v):
    """Ranks 0 .. v - 1 in runs of growing length: (a rank in the middle, the run's length)."""
    r = 0
    while r < v:
        d = min(v - r, max(1, r // 8))
        yield r + d // 2, d
        r += d


# ---------------------------------------------------------------------------------------------------- in 64 bits
def _exact_embedding(case, s):
    v, c = case["vocabulary"], case["width"]
    ids = s["ids_"].to(torch.int64)
    if case["mode"] == "fwd":
        return {"out": torch.index_select(s["weight"], 0, ids).double().mul_(case["scale"])}
    made = torch.zeros((v, c), dtype=torch.float64, device="cuda")
    order = torch.argsort(ids, stable=True)
    words, counts = torch.unique_consecutive(ids[order], return_counts=True)
    ends = torch.cumsum(counts, 0)
    for lo in range(0, c, 256):                                     # sums of runs as differences of running sums
        run_ = torch.cumsum(s["grad_out"][:, lo:lo + 256].double()[order], 0)[ends - 1]
        made[words, lo:lo + 256] = torch.diff(run_, dim=0, prepend=torch.zeros_like(run_[:1])) * case["scale"]
    if case["padding"]:
        made[0] = 0.0
    return {"weight": made}


def _exact_rotary(case, s):
    b, n, d, r = (case[x] for x in ("batch", "tokens", "dim", "rotary"))
    first, second = (list(range(r // 2)), list(range(r // 2, r))) if case["style"] == "halves" else (list(range(0, r, 2)), list(range(1, r, 2)))
    at = s["at"].double() if s["at"] is not None else torch.arange(n, dtype=torch.float64, device="cuda").repeat(b, 1)
    inv = torch.tensor([10000.0 ** (-2.0 * i / r) for i in range(r // 2)], dtype=torch.float64, device="cuda")
    phase = torch.exp(1j * at[:, :, None, None] * inv)
    made = {}
    for name in ("q", "k"):
        x, w = s[name].double(), s[name + "_weight"].double()
        size = (x.pow(2).sum(-1, keepdim=True) / d + 1e-6).sqrt()
        if case["mode"] == "fwd":
            y = x / size * w
            z = torch.complex(y[..., first], y[..., second]) * phase
            y[..., first], y[..., second] = z.real, z.imag
            made[name] = y
            continue
        g = s["grad_" + name].double()
        z = torch.complex(g[..., first], g[..., second]) * phase.conj()
        g[..., first], g[..., second] = z.real, z.imag
        unit = x / size
        made[name + "_weight"] = torch.einsum("bshd,bshd->d", g, unit)
        gw = g * w
        made[name] = (gw - unit * (torch.einsum("bshd,bshd->bsh", gw, unit) / d)[..., None]) / size
    return made


def _exact_orthogonal(g):
    x = g.double()
    x = x / (torch.linalg.matrix_norm(x) + 1e-7)
    for _ in range(5):
        if x.shape[0] <= x.shape[1]:
            p = torch.mm(x, x.mT)
            x = torch.addmm(x, torch.addmm(p, p, p, beta=_B, alpha=_C), x, beta=_A)
        else:
            p = torch.mm(x.mT, x)
            x = torch.addmm(x, x, torch.addmm(p, p, p, beta=_B, alpha=_C), beta=_A)
    return x


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "embedding":
        return _exact_embedding(case, s)
    if case["op"] == "rotary":
        return _exact_rotary(case, s)
    return [_exact_orthogonal(g) for g in s["updates"]]
