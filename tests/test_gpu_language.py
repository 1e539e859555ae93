"""The operators of a language model's step as differentiable functions, layers and an optimizer: against torch's autograd on the
formulas written out in float64, and together in a training step, with and without compressed activations."""
import math

import pytest

import paper_2507_07149_b200 as daf

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2507_07149_b200 import transformer as tr  # noqa: E402
from paper_2507_07149_b200.autograd import saved_activation_compression  # noqa: E402


def near(got, want, rel):
    assert (got.double() - want).norm() <= rel * want.norm(), float((got.double() - want).norm() / want.norm())


def turned(x, positions, base=10000.0):
    d = x.shape[-1]
    a = positions.double()[..., None, None] * base ** (-torch.arange(0, d, 2, device=x.device, dtype=torch.float64) / d)
    p, q = x.chunk(2, -1)
    return torch.cat((p * a.cos() - q * a.sin(), p * a.sin() + q * a.cos()), -1)


def normed(x, w, eps=1e-6):
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + eps) * w


# float32: sums of a few hundred binary32 terms, 2^-24 each: 2^-16 of the results' size
def test_embedding_through_autograd():
    torch.manual_seed(0)
    layer = tr.Embedding(50, 24, scale=3.0, padding=7, device="cuda")
    t = torch.randint(50, (4, 9), device="cuda")
    t[0, :3] = 7
    g = torch.randn(4, 9, 24, device="cuda")
    (layer(t) * g).sum().backward()
    w = layer.weight.detach().double().requires_grad_()
    ((3.0 * w[t]) * g).sum().backward()
    w.grad[7] = 0
    near(layer.weight.grad, w.grad, 2.0 ** -16)
    mixed = tr.embedding(t, layer.weight, dtype=torch.bfloat16)
    assert mixed.dtype == torch.bfloat16
    layer.weight.grad = None
    mixed.float().sum().backward()
    assert torch.equal(layer.weight.grad.sum(1), 24.0 * torch.bincount(t.flatten(), minlength=50).float())


@pytest.mark.parametrize("use", ["both", "q", "k", "alone"])
def test_rotary_norm_through_autograd(use):
    torch.manual_seed(1)
    x = torch.randn(2, 13, 6 * 16, device="cuda", requires_grad=True)
    wq, wk = (torch.nn.Parameter(1 + 0.2 * torch.randn(16, device="cuda")) for _ in range(2))
    gq, gk = torch.randn(2, 13, 4, 16, device="cuda"), torch.randn(2, 13, 2, 16, device="cuda")
    at = torch.randint(0, 5000, (2, 13), device="cuda")

    def heads(t):
        return t.view(2, 13, 6, 16).split((4, 2), 2)
    q, k = heads(x)
    if use == "alone":
        loss = (tr.rotary_norm(q, None, wq, positions=at) * gq).sum()
    else:
        a, b = tr.rotary_norm(q, k, wq, wk, positions=at)
        loss = ((a * gq).sum() if use != "k" else 0) + ((b * gk).sum() if use != "q" else 0)
    loss.backward()
    y, vq, vk = (t.detach().double().requires_grad_() for t in (x, wq, wk))
    q, k = heads(y)
    want = ((turned(normed(q, vq), at) * gq).sum() if use != "k" else 0) + ((turned(normed(k, vk), at) * gk).sum() if use in ("both", "k") else 0)
    want.backward()
    near(x.grad, y.grad, 2.0 ** -16)
    for got, ref in ((wq.grad, vq.grad), (wk.grad, vk.grad)):
        if ref is None:
            assert got is None or not got.any()
        else:
            near(got, ref, 2.0 ** -16)


def test_second_derivatives_are_errors():
    w = torch.randn(9, 16, device="cuda", requires_grad=True)
    g, = torch.autograd.grad(tr.embedding(torch.tensor([1, 2], device="cuda"), w).square().sum(), w, create_graph=True)
    with pytest.raises(RuntimeError):
        g.sum().backward()
    q = torch.randn(1, 2, 1, 16, device="cuda", requires_grad=True)
    g, = torch.autograd.grad(tr.rotary_norm(q, None).square().sum(), q, create_graph=True)
    with pytest.raises(RuntimeError):
        g.sum().backward()


def test_tokens_or_positions_that_change_between_the_passes_are_an_error():
    w, t = torch.randn(9, 16, device="cuda", requires_grad=True), torch.tensor([1, 2], device="cuda")
    out = tr.embedding(t, w)
    t.add_(1)
    with pytest.raises(RuntimeError):
        out.sum().backward()
    q, at = torch.randn(1, 2, 1, 16, device="cuda", requires_grad=True), torch.tensor([[1, 2]], device="cuda")
    out = tr.rotary_norm(q, None, positions=at)
    at.add_(1)
    with pytest.raises(RuntimeError):
        out.sum().backward()


def model_in_64_bits(net, tokens, lengths):
    """The language model's scores from its parameters in float64."""
    p = {n: t.detach().double().requires_grad_() for n, t in net.named_parameters()}
    x = p["embed.weight"][tokens]
    ln = torch.nn.functional.layer_norm
    h = ln(x, x.shape[-1:], p["first.weight"], p["first.bias"], 1e-5)
    b, s, width = x.shape
    at = torch.arange(s, device="cuda").expand(b, s)
    see = (at[0][None, :] <= at[0][:, None])[None, None] & (at[0][None] < lengths[:, None])[:, None, None]
    for i, block in enumerate(net.blocks):
        w = {n[len(f"blocks.{i}."):]: t for n, t in p.items() if n.startswith(f"blocks.{i}.")}
        qkv = (h @ w["qkv.weight"].t() + w["qkv.bias"]).view(b, s, -1, block.dim)
        q, k, v = qkv.split((block.heads, block.kv_heads, block.kv_heads), 2)
        q, k = turned(normed(q, w["q_norm"]), at), turned(normed(k, w["k_norm"]), at)
        k, v = (t.repeat_interleave(block.heads // block.kv_heads, 2) for t in (k, v))
        scores = (torch.einsum("bqhd,bkhd->bhqk", q, k) / math.sqrt(block.dim)).masked_fill(~see, float("-inf"))
        a = torch.einsum("bhqk,bkhd->bqhd", torch.softmax(scores, -1), v).reshape(b, s, -1)
        for join, y in (("join1", a @ w["out.weight"].t() + w["out.bias"]), ("join2", None)):
            if y is None:
                y = torch.nn.functional.gelu(h @ w["up.weight"].t() + w["up.bias"]) @ w["down.weight"].t() + w["down.bias"]
            x = x + w[join + ".gate"] * y
            h = ln(x, x.shape[-1:], w[join + ".weight"], w[join + ".bias"], 1e-6)
    return h @ p["head.weight"].t(), p


def test_a_step_of_the_language_model():
    """float32 throughout: some hundred binary32 roundings in sequence (two blocks' products in full precision), each result's
    relative error below 1e-4."""
    torch.manual_seed(4)
    torch.backends.cuda.matmul.allow_tf32 = False
    net = tr.LanguageModel(97, 64, 4, 2, 128, padding=0, kv_heads=2, gate_init=0.5).cuda()
    tokens = torch.randint(97, (3, 21), device="cuda")
    lengths = torch.tensor([21, 5, 13], dtype=torch.int32, device="cuda")
    here = torch.arange(21, device="cuda") < lengths[:, None]
    tokens = tokens.where(here, 0)
    g = torch.randn(3, 21, 97, device="cuda") * here[..., None]
    out = net(tokens, lengths)
    (out * g).sum().backward()
    want, p = model_in_64_bits(net, tokens, lengths)
    (want * g).sum().backward()
    p["embed.weight"].grad[0] = 0
    near(out * here[..., None], want.detach() * here[..., None], 1e-4)
    for n, t in net.named_parameters():
        near(t.grad, p[n].grad, 1e-4)
    daf.check_device()


def test_muon_steps_by_its_formula():
    """Two steps: momentum and the steps in float64, but for the update's rounding to bfloat16 (2^-9 on average of a direction) and the
    orthogonalisation's own (see its test): 2e-2 of the step's size."""
    torch.manual_seed(5)
    ps = [torch.nn.Parameter(torch.randn(*s, device="cuda")) for s in ((96, 64), (64, 96), (32, 4, 3, 3))]
    start = [p.detach().double().clone() for p in ps]
    opt = tr.Muon(ps, 0.1, momentum=0.9, weight_decay=0.01)
    gs = [[torch.randn_like(p) for p in ps] for _ in range(2)]
    want, buf = [s.clone() for s in start], [torch.zeros_like(s) for s in start]
    for step in range(2):
        for p, g in zip(ps, gs[step]):
            p.grad = g.clone()
        before = [w.clone() for w in want]
        opt.step()
        for i, g in enumerate(gs[step]):
            buf[i] = 0.9 * buf[i] + g.double()
            u = (g.double() + 0.9 * buf[i]).flatten(1)
            x = u / (u.norm() + 1e-7)
            tall = x.shape[0] > x.shape[1]
            x = x.t() if tall else x
            for _ in range(5):
                a = x @ x.t()
                x = 3.4445 * x + (-4.7750 * a + 2.0315 * a @ a) @ x
            x = (x.t() if tall else x).reshape(g.shape)
            want[i] = (1 - 0.1 * 0.01) * before[i] - 0.1 * math.sqrt(max(1.0, u.shape[0] / u.shape[1])) * x
        for p, w, b in zip(ps, want, before):
            assert (p.double() - w).norm() <= 2e-2 * (w - b).norm() * (step + 1)
    with pytest.raises(ValueError):
        tr.Muon([torch.nn.Parameter(torch.zeros(4, device="cuda"))])


def test_muon_keeps_its_momentum_in_32_bits_through_a_checkpoint():
    torch.manual_seed(8)
    ps = [torch.nn.Parameter(torch.randn(16, 24, device="cuda").bfloat16()) for _ in range(2)]
    opt = tr.Muon(ps, 0.1)
    ps[0].grad = torch.randn_like(ps[0])                            # the other one has no gradient yet
    for _ in range(3):
        opt.step()
    kept = opt.state[ps[0]]["momentum"].clone()
    assert kept.dtype == torch.float32 and ps[1] not in opt.state
    other = tr.Muon(ps, 0.5)
    other.load_state_dict(opt.state_dict())
    got = other.state[ps[0]]["momentum"]
    assert got.dtype == torch.float32 and torch.equal(got, kept) and got.data_ptr() != opt.state[ps[0]]["momentum"].data_ptr()
    assert other.param_groups[0]["lr"] == 0.1
    other.step()


@pytest.mark.parametrize("bits", [None, 8.0, 4.0])
def test_training_runs(bits):
    losses = tr.train_language(3, compressed=bits is not None, bit_budget=bits or 8.0, batch=5, tokens=64, vocabulary=300)
    assert len(losses) == 3 and all(math.isfinite(a) and math.isfinite(b) and b > 0 for a, b in losses)


def test_gradients_under_compression_are_those_of_the_restored_queries_and_keys():
    torch.manual_seed(6)
    q, k = (torch.randn(2, 64, n, 64, device="cuda", requires_grad=True) for n in (4, 2))
    w = torch.ones(64, device="cuda", requires_grad=True)
    ctx = saved_activation_compression(group_size=256, bit_budget=8.0, seed=1)
    gq, gk = torch.randn_like(q), torch.randn_like(k)
    with ctx:
        a, b = tr.rotary_norm(q, k, w, w)
    torch.autograd.backward((a, b), (gq, gk))
    exact = daf.rotary_norm_grad(q.detach(), k.detach(), w.detach(), w.detach(), gq, gk)
    # 8 bits of a group of 256: a step is its range / 255, about 6 / 255 of the deviation; stochastic rounding is off by 0.4 of that
    near(q.grad, exact[0].double(), 2e-2)
    near(k.grad, exact[1].double(), 2e-2)
    assert not torch.equal(q.grad, exact[0])


def test_a_captured_step():
    """Forward and backward of a block in a graph, replayed on other inputs."""
    torch.manual_seed(7)
    emb = tr.Embedding(40, 64, device="cuda")
    block = tr.Block(64, 2, 128, causal=True, rotary=True).cuda()
    params = [*emb.parameters(), *block.parameters()]
    tokens = torch.randint(40, (2, 10), device="cuda")

    def step():
        x = emb(tokens)
        z, h = block(x, x)
        return torch.autograd.grad((z * z).sum() + h.sum(), params)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        made = step()
    tokens.copy_(torch.randint(40, (2, 10), device="cuda"))
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(made, step()):
        assert torch.equal(a, b) or (a - b).norm() <= 1e-5 * b.norm()     # cuBLAS may take another algorithm
