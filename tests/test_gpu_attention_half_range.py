"""Attention's backward pass in float16, whose range is the narrowest: gradients that differ by orders of magnitude between rows, long
values, probabilities far below the smallest normal number."""
import pytest

import paper_2507_07149_b200 as daf

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_attention import reference  # noqa: E402

HALF = torch.float16


def tensors(Sq, Sk, H, Hkv, D, seed=0, v_size=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    q, g = (torch.randn((1, Sq, H, D), generator=gen, device="cuda") for _ in range(2))
    k, v = (torch.randn((1, Sk, Hkv, D), generator=gen, device="cuda") for _ in range(2))
    return q.to(HALF), k.to(HALF), (v_size * v).to(HALF), g


def both(q, k, v, g, causal):
    out, lse = daf.attention(q, k, v, causal=causal)
    got = daf.attention_grad(q, k, v, out, lse, g, causal=causal)
    want, _, _ = reference(q, k, v, g, q.shape[3] ** -0.5, causal, None, out, lse)
    return got, want


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("D,Sk", [(64, 1024), (80, 700), (128, 1024)])
def test_rows_of_small_gradients_beside_large_ones(causal, D, Sk):
    """grad_out of one row in fifty is 2^17 times that of the others, as with a loss on a few tokens.  dq of every row on its own:
    dS and the result are rounded to 2^-11 each, elements of random signs; 2^-10 of the row's norm, and results below 2^-14
    lose 2^-25 each."""
    q, k, v, g = tensors(300, Sk, 2, 1, D)
    size = torch.full((300, 1, 1), 2.0 ** -7, device="cuda")
    size[::50] = 2.0 ** 10
    g = (g * size).to(HALF)
    (gq, gk, gv), want = both(q, k, v, g, causal)
    off = (gq.double() - want["q"]).norm(dim=3)
    assert (off <= 2.0 ** -10 * want["q"].norm(dim=3) + 2.0 ** -25 * D ** 0.5).all(), float((off / want["q"].norm(dim=3)).max())
    for t, n in ((gk, "k"), (gv, "v")):
        assert (t.double() - want[n]).norm() <= 2.0 ** -10 * want[n].norm()


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("v_size,keys", [(300.0, 300), (3000.0, 300), (300.0, 4), (3000.0, 3)])
def test_long_values(causal, D, v_size, keys):
    """|v| of 2400 to 34000 with gradients that keep every result inside the type; few keys have large probabilities."""
    q, k, v, g = tensors(200, keys, 2, 2, D, seed=1, v_size=v_size)
    g = (g * (4.0 / v_size)).to(HALF)
    got, want = both(q, k, v, g, causal)
    for t, n in zip(got, "qkv"):
        assert torch.isfinite(t).all(), n
        assert (t.double() - want[n]).norm() <= 2.0 ** -10 * want[n].norm() + 2.0 ** -25 * t.numel() ** 0.5, n


@pytest.mark.parametrize("keys", [50000, 400000, 483000, 3000001])
def test_probabilities_below_the_smallest_normal_number(keys):
    """Uniform probabilities of 2^-15.6 to 2^-21.5: dv is their product with a sum over the rows, two roundings of 2^-11."""
    q = torch.zeros(1, 64, 1, 8, device="cuda", dtype=HALF)
    k, v = (torch.randn(1, keys, 1, 8, device="cuda").to(HALF) for _ in range(2))
    g = torch.full_like(q, 1000.0)
    out, lse = daf.attention(q, k, v)
    gv = daf.attention_grad(q, k, v, out, lse, g)[2]
    want = 64 * 1000.0 / keys
    assert ((gv.double() / want - 1).abs() <= 2.0 ** -10 + 2.0 ** -12).all(), float((gv.double() / want - 1).abs().max())


@pytest.mark.parametrize("D", [64, 128])
def test_long_values_along_the_gradient(D):
    """grad_out along one of two long values: dP reaches |grad_out| |v|, the largest there is."""
    q, k, v, _ = tensors(130, 2, 1, 1, D, seed=2, v_size=3000.0)
    g = (v[:, :1].float() * 2.0 ** -24).to(HALF).expand(1, 130, 1, D).contiguous()
    got, want = both(q, k, v, g, False)
    for t, n in zip(got, "qkv"):
        assert torch.isfinite(t).all(), n
        assert (t.double() - want[n]).norm() <= 2.0 ** -10 * want[n].norm() + 2.0 ** -25 * t.numel() ** 0.5, n
