"""Attention rows whose maximum moves while the keys are walked: the running reference, its sum and the accumulated output all
have to follow it.  Against the definition in 64 bits, with the bounds of test_gpu_attention.

The scores are step * blk * sign in units of log2 (blk: the 64 keys' or 128 keys' block, counted from the middle; sign: 1, 0 or
-1, mixed within every warp's rows) plus a little noise.  |s| stays below the 30 that those bounds assume."""
import math

import pytest

import paper_2507_07149_b200 as daf

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_attention import DTYPES, check, reference  # noqa: E402


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


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("step", [7.9, 8.1])
@pytest.mark.parametrize("D", [40, 64, 80, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_maxima_that_pass_the_references_bound(dtype, step, D, causal):
    """Blocks of 128 keys whose maxima rise by just less and just more than the 8 units of log2 that the 16-bit kernel lets a
    maximum pass its reference by before it scales what it has (two steps of 7.9 make it move, too)."""
    moving(dtype, 2, 300, 700, 4, 2, D, causal, step, 128)
    moving(dtype, 3, 257, 900, 2, 1, D, causal, step, 128, lengths=[900, 0, 641], seed=1)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("step", [0.75, 2.5])
def test_maxima_that_move_in_calls_split_over_the_keys(dtype, step):
    """Few rows over many keys: the splits' maxima differ, and move inside a split, too."""
    moving(dtype, 1, 5, 2100, 2, 1, 64, False, step, 128)
    moving(dtype, 2, 3, 2100, 1, 1, 128, True, step, 128, lengths=[2100, 1290], seed=2)


@pytest.mark.parametrize("dtype", DTYPES)
def test_one_key_above_all_that_came_before(dtype):
    """A single late key takes over, in one row of a warp alone: the others' sums keep their bits."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    q, k, v = (torch.randn((1, S, 1, 64), generator=gen, device="cuda").to(dtype) for S in (128, 640, 640))
    q[..., 0], k[..., 0] = 0, 0
    want, want_lse = daf.attention(q, k, v)
    q[0, 77, 0, 0], k[0, 600, 0, 0] = 16, 16                        # 256 / 8 = 32 more for one pair
    out, lse = daf.attention(q, k, v)
    rest = torch.arange(128, device="cuda") != 77
    tell = 2.0 ** -20 * (4 + want_lse.abs())
    assert ((lse - want_lse).abs() <= tell)[:, :, rest].all() and (lse[0, 0, 77] - (q[0, 77, 0].double() @ k[0, 600, 0].double() / 8)).abs() <= 1e-3
    u = {torch.float32: 2.0 ** -16, torch.float16: 2.0 ** -10, torch.bfloat16: 2.0 ** -7}[dtype]
    assert ((out - want).abs()[:, rest] <= u).all() and ((out - v[:, 600:601]).abs()[:, 77] <= u * v[:, 600].abs() + 1e-5).all()
