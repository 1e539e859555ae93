"""Attention rows whose maximum moves while the keys are walked: the running reference, its sum and the accumulated output all
have to follow it.  Against the definition in 64 bits, with the bounds of test_gpu_attention.

The scores are step * blk * sign in units of log2 (blk: the 64 keys' or 128 keys' block, counted from the middle; sign: 1, 0 or
-1, mixed within every warp's rows) plus a little noise.  |s| stays below the 30 that those bounds assume."""
import math

import pytest

import paper_2507_07149_b200 as daf

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_attention import check, reference  # noqa: E402


def moving(dtype, B, Sq, Sk, H, Hkv, D, causal, step, block, lengths=None, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    scale = step / 1.4426950408889634

    def rnd(*shape, size=1.0):
        return torch.randn(shape, generator=gen, device="cuda") * size
    q, k = rnd(B, Sq, H, D, size=0.01), rnd(B, Sk, Hkv, D, size=0.01)
    q[..., 0] = torch.randint(-1, 2, (B, Sq, H), generator=gen, device="cuda").float()
    blocks = (Sk + block - 1) // block
    k[..., 0] = (torch.arange(Sk, device="cuda") // block - blocks // 2).float()[None, :, None]
    q, k, v, g = q.to(dtype), k.to(dtype), rnd(B, Sk, Hkv, D).to(dtype), rnd(B, Sq, H, D).to(dtype)
    lens = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    out, lse = daf.attention(q, k, v, causal=causal, scale=scale, key_lengths=lens)
    want, bound, L = reference(q, k, v, g, scale, causal, lengths)
    check(out, want["out"], bound["out"], "out")
    fin = ~torch.isinf(L)
    assert torch.equal(torch.isinf(lse), ~fin) and ((lse.double() - L)[fin].abs() <= 2.0 ** -20 * (4 + L[fin].abs())).all(), "lse"
    grads = daf.attention_grad(q, k, v, out, lse, g, causal=causal, scale=scale, key_lengths=lens)
    want, bound, _ = reference(q, k, v, g, scale, causal, lengths, out, lse)
    for n, t in zip("qkv", grads):
        check(t, want[n], bound[n], f"grad_{n}")
    again, again_lse = daf.attention(q, k, v, causal=causal, scale=scale, key_lengths=lens)
    assert torch.equal(again, out) and torch.equal(again_lse, lse)


@pytest.mark.parametrize("step", [0.9, 7.9])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_maxima_that_move_with_every_block_binary32(step, D, causal):
    """Blocks of 64 keys: the two warps of a row tell each other another maximum in every block."""
    moving(torch.float32, 2, 300, 450, 4, 2, D, causal, step, 64, lengths=[450, 333])
