"""Attention inside saved_activation_compression below 8 bits: the gradients are those of the formula at the restored q, k and v.

q and k have standard deviation 2, so the scores have 4 (64 elements): restored from 4 bits they are off by several units, and
probabilities with the statistics of the exact scores sum to anything."""
import pytest

import paper_2507_07149_b200 as daf

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_attention import reference  # noqa: E402

from paper_2507_07149_b200 import transformer as tr  # noqa: E402
from paper_2507_07149_b200.autograd import saved_activation_compression  # noqa: E402


def through(ctx, dtype=torch.float32, causal=False, size=2.0, tokens=256):
    torch.manual_seed(3)
    q, k, v = ((size * torch.randn(2, tokens, 4, 64, device="cuda")).to(dtype).requires_grad_() for _ in range(3))
    with ctx:
        out = tr.attention(q, k, v, causal=causal)
    g = torch.randn_like(out)
    out.backward(g)
    return q, k, v, g


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("bits", [2.0, 4.0])
@pytest.mark.parametrize("causal", [False, True])
def test_gradients_are_those_of_the_restored_tensors(dtype, bits, causal):
    """Relative errors of the whole gradients: 2^-6 is four roundings to bfloat16 of every factor, 2^-9 of float16; binary32 as in
    test_attention_through_autograd."""
    ctx = saved_activation_compression(group_size=256, bit_budget=bits, seed=1)
    q, k, v, g = through(ctx, dtype, causal)
    assert ctx.stats["tensors"] == 3 and ctx.stats["passed_through"] == 0      # the output is not kept
    kept = [daf.decompress(daf.compress(t.detach().reshape(-1), 256, (1, 2, 4, 8), bits, seed=1, elem_index_base=t.numel() * i)).view(t.shape)
            for i, t in enumerate((q, k, v))]
    out, lse = daf.attention(*kept, causal=causal)
    for t, w in zip((q, k, v), daf.attention_grad(*kept, out, lse, g, causal=causal)):
        assert torch.equal(t.grad, w)
    r, _, L = reference(*kept, g, 0.125, causal, None)
    want, _, _ = reference(*kept, g, 0.125, causal, None, r["out"], L)
    tol = {torch.float32: 2.0 ** -16, torch.float16: 2.0 ** -9, torch.bfloat16: 2.0 ** -6}[dtype]
    for n, t in zip("qkv", (q, k, v)):
        assert (t.grad.double() - want[n]).norm() <= tol * want[n].norm(), n


def test_a_store_that_drops_what_attention_kept():
    """Dropped tensors come back as zeros: uniform probabilities over the keys, no gradient of q and k, finite ones of v."""
    ctx = saved_activation_compression(group_size=256, bit_budget=8, mem_budget=1 << 16, seed=1)
    q, k, v, g = through(ctx, size=3.0)
    assert ctx.stats["dropped"] > 0
    assert (q.grad == 0).all() and (k.grad == 0).all()
    want = (g.double().sum(1, keepdim=True) / 256).expand_as(g)
    assert (v.grad.double() - want).norm() <= 2.0 ** -16 * want.norm()


def test_other_hooks_keep_what_they_are_given():
    """Hooks that restore exactly (and none at all) keep the statistics; inside and outside of a compressing context."""
    plain = through(torch.autograd.graph.saved_tensors_hooks(lambda t: t, lambda t: t))
    seen = []
    both = through(torch.autograd.graph.saved_tensors_hooks(lambda t: seen.append(t) or t, lambda t: t))
    assert len(seen) == 4
    for a, b in zip(plain[:3], both[:3]):
        assert torch.equal(a.grad, b.grad)


def test_the_trainer_at_the_default_budget():
    losses = tr.train(25, compressed=True, bit_budget=4.0, batch=32, tokens=64)
    first, last = losses[0][0], sum(x[0] for x in losses[-5:]) / 5
    assert last < 0.8 * first and all(b < 1e4 for _, b in losses)
