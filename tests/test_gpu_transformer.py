"""The operators as differentiable functions and layers: against torch's autograd on the formulas written out in float64,
and together in a training step, with and without compressed activations."""
import pytest

import paper_2507_07149_b200 as daf

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2507_07149_b200 import transformer as tr  # noqa: E402
from paper_2507_07149_b200.autograd import saved_activation_compression  # noqa: E402


def test_attention_through_autograd_with_shared_heads_and_a_packed_projection():
    """float32 inputs: the kernels' sums are binary32 (relative 2^-16 of the results' size is generous, see the operator's test)."""
    torch.manual_seed(0)
    x = torch.randn(2, 70, (4 + 2 * 2) * 16, device="cuda", requires_grad=True)

    def heads(t):
        return t.view(2, 70, 8, 16).split((4, 2, 2), 2)
    q, k, v = heads(x)
    lens = torch.tensor([70, 33], dtype=torch.int32, device="cuda")
    out = tr.attention(q, k, v, causal=True, key_lengths=lens)
    g = torch.randn_like(out)
    out.backward(g)
    y = x.detach().double().requires_grad_()
    q, k, v = heads(y)
    k, v = (t.repeat_interleave(2, 2) for t in (k, v))
    s = torch.einsum("bqhd,bkhd->bhqk", q, k) / 4
    i = torch.arange(70, device="cuda")
    see = (i[None, :] <= i[:, None])[None, None] & (i[None] < lens[:, None])[:, None, None]
    want = torch.einsum("bhqk,bkhd->bqhd", torch.softmax(s.masked_fill(~see, float("-inf")), -1), v)
    want.backward(g.double())
    for a, b in ((out, want), (x.grad, y.grad)):
        assert (a.double() - b).norm() <= 2.0 ** -16 * b.norm()


@pytest.mark.parametrize("use", ["both", "z", "h"])
def test_join_through_autograd(use):
    torch.manual_seed(1)
    layer = tr.ResidualNorm(96, gate_init=0.3, post=True, residual_scale=0.5, device="cuda")
    with torch.no_grad():
        for p in layer.parameters():
            p.add_(0.1 * torch.randn_like(p))
    x, y = (torch.randn(3, 11, 96, device="cuda", requires_grad=True) for _ in range(2))
    gz, gh = torch.randn(3, 11, 96, device="cuda"), torch.randn(3, 11, 96, device="cuda")

    def loss(z, h):
        return (0 if use == "h" else (z * gz.to(z.dtype)).sum()) + (0 if use == "z" else (h * gh.to(h.dtype)).sum())
    loss(*layer(x, y)).backward()
    p = {n: t.detach().double().requires_grad_() for n, t in layer.named_parameters()}
    a, b = x.detach().double().requires_grad_(), y.detach().double().requires_grad_()
    u = torch.nn.functional.layer_norm(b, (96,), p["post_weight"], p["post_bias"], 1e-6)
    z = a + 0.5 * p["gate"] * u
    loss(z, torch.nn.functional.layer_norm(z, (96,), p["weight"], p["bias"], 1e-6)).backward()
    for got, want in [(x.grad, a.grad), (y.grad, b.grad)] + [(t.grad, p[n].grad) for n, t in layer.named_parameters()]:
        want = torch.zeros_like(got) if want is None else want
        assert (got.double() - want).norm() <= 2.0 ** -16 * want.norm() + 1e-6


def test_clipping_parameters():
    torch.manual_seed(2)
    ps = [torch.nn.Parameter(torch.randn(n, device="cuda")) for n in (5, 1000, 3)] + [torch.nn.Parameter(torch.randn(4, 6, device="cuda"))]
    for p in ps[:2]:
        p.grad = torch.randn_like(p)
    ps[3].grad = torch.randn(6, 4, device="cuda").t()               # not contiguous
    want = torch.cat([p.grad.reshape(-1) for p in ps if p.grad is not None]).double()
    norm = tr.clip_grad_norm_(ps, 0.5)
    got = torch.cat([p.grad.reshape(-1) for p in ps if p.grad is not None]).double()
    assert abs(float(norm) - float(want.norm())) <= 2.0 ** -16 * float(want.norm()) and ps[2].grad is None
    assert (got - want * 0.5 / (want.norm() + 1e-6)).norm() <= 2.0 ** -16 * 0.5


def test_what_attention_and_the_join_keep_is_compressed():
    """Inside the hooks q, k, v and the output are kept compressed, the row statistics are not; the gradients are those of the
    restored tensors."""
    torch.manual_seed(3)
    q, k, v = (torch.randn(2, 128, 4, 64, device="cuda", requires_grad=True) for _ in range(3))
    ctx = saved_activation_compression(group_size=256, bit_budget=8.0, seed=1)
    with ctx:
        out = tr.attention(q, k, v)
    assert ctx.stats["tensors"] == 4 and ctx.stats["passed_through"] == 0
    g = torch.randn_like(out)
    out.backward(g)
    kept = [daf.decompress(daf.compress(t.detach().reshape(-1), 256, (1, 2, 4, 8), 8.0, seed=1, elem_index_base=65536 * i)).view(t.shape)
            for i, t in enumerate((q, k, v, out))]
    _, lse = daf.attention(q.detach(), k.detach(), v.detach())
    want = daf.attention_grad(*kept, lse, g)
    for t, w in zip((q, k, v), want):
        assert torch.equal(t.grad, w)


def test_training_with_and_without_compressed_activations():
    """The task separates after a few steps; compressed at 8 bits the loss follows the uncompressed one."""
    plain = tr.train(25, compressed=False, batch=32, tokens=65)
    packed = tr.train(25, compressed=True, batch=32, tokens=65)
    assert all(torch.isfinite(torch.tensor(x)).all() for x in (plain, packed))
    first, last, kept = plain[0][0], sum(x[0] for x in plain[-5:]) / 5, sum(x[0] for x in packed[-5:]) / 5
    assert last < 0.7 * first and kept < 0.7 * first and abs(kept - last) < 0.25 * first
