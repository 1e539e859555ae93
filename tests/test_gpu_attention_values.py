"""What attention makes of values that are not numbers, and of rows that see nothing but hold such values.

The definition: a visible score that is NaN or +inf makes its row's output and logarithm NaN; one that is -inf has weight zero
(binary32 inputs: an infinite element of q or k counts as NaN); a visible value that is not a number reaches the outputs of
the rows that see it; 0 and -inf mean a row that sees no key, and nothing else."""
import math

import pytest

import paper_2507_07149_b200 as daf

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_attention import DTYPES, check, reference  # noqa: E402


def inputs(dtype, Sq, Sk, H, D, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn((1, S, H, D), generator=gen, device="cuda").to(dtype) for S in (Sq, Sk, Sk)]


# few rows over many keys: the call is split over the keys (16-bit types)
SHAPES = [(100, 70, 2, 64), (200, 300, 1, 128), (5, 4100, 1, 64), (3, 5000, 2, 80)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("Sq,Sk,H,D", SHAPES)
@pytest.mark.parametrize("at", [0, 0.5, 1])
def test_nan_in_a_visible_key_reaches_every_row(dtype, Sq, Sk, H, D, at):
    q, k, v = inputs(dtype, Sq, Sk, H, D)
    k[0, int(at * (Sk - 1)), 0, 3] = math.nan
    out, lse = daf.attention(q, k, v)
    assert out[:, :, 0].isnan().all() and lse[:, 0].isnan().all()
    assert out[:, :, 1:].isfinite().all() and lse[:, 1:].isfinite().all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("Sq,Sk,H,D", SHAPES)
def test_nan_in_a_query_reaches_its_row_alone(dtype, Sq, Sk, H, D):
    q, k, v = inputs(dtype, Sq, Sk, H, D)
    want, want_lse = daf.attention(q, k, v)
    q[0, 2, 0, 5] = math.nan
    out, lse = daf.attention(q, k, v)
    assert out[0, 2, 0].isnan().all() and lse[0, 0, 2].isnan()
    keep = torch.ones_like(out[..., 0], dtype=torch.bool)
    keep[0, 2, 0] = False
    assert torch.equal(out[keep], want[keep]) and torch.equal(lse[keep.transpose(1, 2)], want_lse[keep.transpose(1, 2)])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("Sq,Sk,H,D", SHAPES)
@pytest.mark.parametrize("scale", [0.125, -0.125])
def test_infinite_scores(dtype, Sq, Sk, H, D, scale):
    """+inf is NaN; -inf is a weight of zero, all of them -inf nothing to divide by: NaN beside a logarithm of -inf."""
    q, k, v = inputs(dtype, Sq, Sk, H, D)
    q = q.abs() + 0.5                                               # no zeros, one sign: q . k with an infinity in k has its sign
    k[0, Sk // 2, 0] = math.inf if scale > 0 else -math.inf
    out, lse = daf.attention(q, k, v, scale=scale)
    assert out[:, :, 0].isnan().all() and lse[:, 0].isnan().all() and out[:, :, 1:].isfinite().all()
    if dtype == torch.float32:
        return
    k[0, Sk // 2, 0] = -math.inf if scale > 0 else math.inf
    out, lse = daf.attention(q, k, v, scale=scale)
    others = torch.arange(Sk, device="cuda") != Sk // 2
    want, bound, L = reference(q, k[:, others], v[:, others], q, scale, False, None)
    check(out[:, :, :1], want["out"][:, :, :1], bound["out"][:, :, :1] + 2.0 ** -20, "out")
    assert ((lse[:, 0].double() - L[:, 0]).abs() <= 2.0 ** -20 * (4 + L[:, 0].abs())).all()
    k[0, :, 0] = -math.inf if scale > 0 else math.inf
    out, lse = daf.attention(q, k, v, scale=scale)
    assert out[:, :, 0].isnan().all() and (lse[:, 0] == -math.inf).all() and out[:, :, 1:].isfinite().all()


@pytest.mark.parametrize("dtype,size", [(torch.float32, 1e16), (torch.float32, 1e18), (torch.float16, 1e3), (torch.bfloat16, 1e3)])
def test_scores_far_below_zero(dtype, size):
    """Finite scores, however low, are scores: the row is not one that sees nothing."""
    q = torch.full((1, 40, 1, 64), size, device="cuda", dtype=dtype)
    k = torch.full((1, 150, 1, 64), -size, device="cuda", dtype=dtype)
    v = torch.randn(1, 150, 1, 64, device="cuda").to(dtype)
    out, lse = daf.attention(q, k, v, scale=1.0)
    want = v.double().mean(1, keepdim=True).expand_as(out)
    score = float(q[0, 0, 0, 0].double() * k[0, 0, 0, 0].double()) * 64
    assert (out.double() - want).abs().max() <= 2.0 ** -7 and ((lse / score) - 1).abs().max() <= 2.0 ** -20


@pytest.mark.parametrize("size", [1e16, 1e18])
def test_16_bit_scores_out_of_range_are_not_an_empty_row(size):
    """Beyond 2^27 the exponent's rounding no longer fits a power: the output says NaN instead of 0, or is right."""
    q = torch.full((1, 40, 1, 64), size, device="cuda", dtype=torch.bfloat16)
    v = torch.ones(1, 150, 1, 64, device="cuda", dtype=torch.bfloat16)
    out, _ = daf.attention(q, -q[:, :1].expand(1, 150, 1, 64), v, scale=1.0)
    assert (out.isnan() | (out == 1)).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("Sq,Sk,H,D", SHAPES)
def test_values_that_are_not_numbers(dtype, Sq, Sk, H, D):
    q, k, v = inputs(dtype, Sq, Sk, H, D)
    v[0, Sk - 1, 0, 7] = math.nan
    out, lse = daf.attention(q, k, v)
    assert out[:, :, 0, 7].isnan().all() and lse.isfinite().all()
    rest = torch.ones_like(out, dtype=torch.bool)
    rest[:, :, 0, 7] = False
    assert out[rest].isfinite().all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_backward_follows(dtype):
    """Rows whose output is NaN give NaN gradients (a loss scaler sees them); heads without one stay finite."""
    q, k, v = inputs(dtype, 150, 150, 2, 64)
    k[0, 30, 0, 0] = math.nan
    out, lse = daf.attention(q, k, v)
    for t in daf.attention_grad(q, k, v, out, lse, torch.ones_like(out)):
        assert t[:, :, 0].isnan().any() and t[:, :, 1].isfinite().all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Sq,Sk,lengths", [(300, 100, None), (130, 1, None), (200, 150, [150, 0])])
def test_whatever_a_row_that_sees_nothing_holds(dtype, D, Sq, Sk, lengths):
    """Causal rows ahead of the first key, sequences without keys: NaN and infinities in their q, out and grad_out change nothing."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    B = 1 if lengths is None else len(lengths)
    q, g = (torch.randn((B, Sq, 2, D), generator=gen, device="cuda").to(dtype) for _ in range(2))
    k, v = (torch.randn((B, Sk, 1, D), generator=gen, device="cuda").to(dtype) for _ in range(2))
    lens = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    out, lse = daf.attention(q, k, v, causal=True, key_lengths=lens)
    want = daf.attention_grad(q, k, v, out, lse, g, causal=True, key_lengths=lens)
    dead = torch.zeros(B, Sq, dtype=torch.bool, device="cuda")
    dead[:, :Sq - Sk] = True
    if lengths is not None:
        dead[1] = True
    assert dead.any()
    for bad in (math.nan, math.inf):
        q2, g2, out2 = (t.clone() for t in (q, g, out))
        q2[dead], g2[dead], out2[dead] = bad, bad, bad
        a, b = daf.attention(q2, k, v, causal=True, key_lengths=lens)
        assert torch.equal(a, out) and torch.equal(b, lse)
        got = daf.attention_grad(q2, k, v, out2, lse, g2, causal=True, key_lengths=lens)
        for t, w in zip(got, want):
            assert torch.equal(t, w)
    # and keys that are not numbers reach the rows that see them, not these
    if Sk > 1 and lengths is None:
        k2 = k.clone()
        k2[:, -1] = math.nan
        a, b = daf.attention(q, k2, v, causal=True)
        gq, _, _ = daf.attention_grad(q, k2, v, a, b, g, causal=True)
        assert (gq[dead] == 0).all() and (a[dead] == 0).all() and (b.transpose(1, 2)[dead] == -math.inf).all()


@pytest.mark.parametrize("batch,queries,keys", [(0, 5, 5), (2, 0, 5), (2, 0, 0), (2, 5, 0)])
def test_a_call_without_work_leaves_a_status_too(batch, queries, keys):
    """The workspace holds the status word behind every call that returned DAF_OK, whatever lay there before."""
    import ctypes
    p = daf.daf_attention_params(ctypes.sizeof(daf.daf_attention_params), daf.BF16, batch, queries, keys, 2, 2, 64, 0, 0.125)
    for name, n in (("q", queries), ("k", keys), ("v", keys), ("out", queries), ("grad_out", queries), ("grad_q", queries), ("grad_k", keys), ("grad_v", keys)):
        getattr(p, name + "_stride")[:] = (max(n, 1) * 128, 128, 64)
    x = torch.zeros(2, 5, 2, 64, dtype=torch.bfloat16, device="cuda")
    y, lse = torch.zeros_like(x), torch.zeros(2, 2, 5, device="cuda")
    ws = torch.full((max(daf.daf_attention_workspace(p), daf.daf_attention_grad_workspace(p), 256),), 0xFF, dtype=torch.uint8, device="cuda")
    daf.daf_attention(p, x, x, x, None, y, lse, ws, ws.numel())
    assert daf.daf_poll_status(ws) == daf.OK
    ws.fill_(0xFF)
    daf.daf_attention_grad(p, x, x, x, None, x, lse, x, y, y, y, ws, ws.numel())
    assert daf.daf_poll_status(ws) == daf.OK
