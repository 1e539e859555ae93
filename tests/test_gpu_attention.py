"""Attention and its recomputing backward pass against the definition in 64 bits.

Bounds, derived from the arithmetic (u = 2^-8 / 2^-11 the rounding unit of bfloat16 / float16 results, 0 extra for
binary32 inputs, whose products stay in binary32): a result r = sum of w_j t_j with weights rounded to the input type is
off by at most u |r| (its own rounding) + u sum |w_j t_j| (the weights') + 2^-16 sum |w_j t_j| (binary32 sums, the
exponential's argument |s| <= 30 at 2^-24 each side); float16 weights below 2^-14 are off by 2^-25 absolutely.  For the
score gradients, p (dp - delta), the last term takes |dp| + |delta| in place of their difference."""
import math

import pytest

import paper_2507_07149_b200 as daf

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
UW = {torch.float32: 0.0, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 0.0, torch.float16: 2.0 ** -24, torch.bfloat16: 0.0}
F32 = 2.0 ** -16


def visible(Sq, Sk, causal, n):
    j = torch.arange(Sk, device="cuda")
    see = (j < n)[None, :].expand(Sq, Sk)
    if causal:
        see = see & (j[None, :] <= torch.arange(Sq, device="cuda")[:, None] + Sk - Sq)
    return see


def reference(q, k, v, g, scale, causal, lengths, out=None, lse=None):
    """Everything in float64, with the bound of each result beside it.  The backward pass starts from the given out and lse."""
    B, Sq, H, D = q.shape
    Sk, Hkv = k.shape[1], k.shape[2]
    dt = q.dtype
    u, uw, tiny = U[dt], UW[dt], TINY[dt]
    r = {n: torch.zeros(s, dtype=torch.float64, device="cuda") for n, s in
         (("out", q.shape), ("q", q.shape), ("k", k.shape), ("v", v.shape))}
    bound = {n: torch.zeros_like(t) for n, t in r.items()}
    L = torch.full((B, H, Sq), -math.inf, dtype=torch.float64, device="cuda")
    for b in range(B):
        n = Sk if lengths is None else min(max(int(lengths[b]), 0), Sk)
        for h in range(H):
            e = h // (H // Hkv)
            see = visible(Sq, Sk, causal, n)[:, :n]
            Q, K, V, G = q[b, :, h].double(), k[b, :n, e].double(), v[b, :n, e].double(), g[b, :, h].double()
            if n == 0 or Sq == 0:
                continue
            s = (Q @ K.t() * scale).masked_fill(~see, -math.inf)
            L[b, h] = torch.logsumexp(s, 1)
            some = see.any(1, keepdim=True)
            p = torch.where(some, torch.exp(s - torch.where(some, L[b, h][:, None], 0.0)), 0.0)
            r["out"][b, :, h] = p @ V
            bound["out"][b, :, h] = (uw + F32) * (p @ V.abs()) + tiny * V.abs().sum(0)
            if lse is None:
                continue
            given = lse[b, h].double()[:, None]
            p = torch.where(see, torch.exp(torch.where(see, s, 0.0) - torch.where(some, given, 0.0)), 0.0)
            dp, delta = G @ V.t(), (G * out[b, :, h].double()).sum(1, keepdim=True)
            ds = p * (dp - delta)
            wide = p * (G.abs() @ V.t().abs() + (G * out[b, :, h].double()).abs().sum(1, keepdim=True))
            r["q"][b, :, h] = ds @ K * scale
            r["k"][b, :n, e] += ds.t() @ Q * scale
            r["v"][b, :n, e] += p.t() @ G
            w = uw * ds.abs() + F32 * wide + tiny * see
            bound["q"][b, :, h] = w @ K.abs() * abs(scale)
            bound["k"][b, :n, e] += w.t() @ Q.abs() * abs(scale)
            bound["v"][b, :n, e] += ((uw + F32) * p + tiny * see).t() @ G.abs()
    for n in r:
        bound[n] += 1.01 * u * r[n].abs() + tiny
    return r, bound, L


def check(got, want, bound, what):
    assert torch.isfinite(got).all(), f"{what}: not finite"
    off = (got.double() - want).abs()
    worst = (off / (bound + 1e-30)).max() if off.numel() else torch.tensor(0.0)
    assert (off <= bound + 1e-30).all(), f"{what}: {float(worst):.2f} times its bound, off by {float(off.max()):.3g}"


def run_case(dtype, B, Sq, Sk, H, Hkv, D, causal, lengths=None, scale=None, packed=False, poison=False, size=1.0, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def rnd(*shape):
        return (torch.randn(shape, generator=gen, device="cuda") * size).to(dtype)
    if packed:
        q, k, v = rnd(B, Sq, 3, H, D).unbind(2)
    else:
        q, k, v = rnd(B, Sq, H, D), rnd(B, Sk, Hkv, D), rnd(B, Sk, Hkv, D)
    g = rnd(B, Sq, H, D)
    lens = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    if poison:                                                     # what lies behind a sequence's end is nobody's business
        for b in range(B):
            n = min(max(lengths[b], 0), Sk)
            k[b, n:], v[b, n:] = float("nan"), float("inf")
    scale_ = D ** -0.5 if scale is None else scale
    out, lse = daf.attention(q, k, v, causal=causal, scale=scale, key_lengths=lens)
    want, bound, L = reference(q, k, v, g, scale_, causal, lengths)
    check(out, want["out"], bound["out"], "out")
    assert torch.equal(torch.isinf(lse), torch.isinf(L)) and not torch.isnan(lse).any()
    fin = ~torch.isinf(L)
    assert ((lse.double() - L)[fin].abs() <= 2.0 ** -20 * (4 + L[fin].abs())).all(), "lse"
    grads = daf.attention_grad(q, k, v, out, lse, g, causal=causal, scale=scale, key_lengths=lens)
    want, bound, _ = reference(q, k, v, g, scale_, causal, lengths, out, lse)
    for n, t in zip("qkv", grads):
        check(t, want[n], bound[n], f"grad_{n}")
    return q, k, v, g, out, lse, grads


DTYPES = [torch.float32, torch.float16, torch.bfloat16]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B,Sq,Sk,H,Hkv,D,causal", [
    (1, 1, 1, 1, 1, 8, False), (2, 1, 300, 4, 2, 64, False), (1, 1, 65, 2, 2, 128, True), (2, 64, 64, 2, 2, 64, False),
    (1, 63, 63, 3, 1, 40, True), (2, 128, 128, 2, 1, 128, True), (1, 129, 129, 2, 2, 72, True), (3, 197, 197, 4, 4, 64, False),
    (1, 257, 100, 2, 1, 96, True), (1, 100, 257, 4, 1, 32, True), (1, 400, 390, 2, 2, 128, True), (2, 130, 1, 2, 1, 16, False),
    (1, 513, 700, 4, 2, 80, False), (1, 1000, 1000, 2, 1, 128, True)])
def test_both_directions(dtype, B, Sq, Sk, H, Hkv, D, causal):
    run_case(dtype, B, Sq, Sk, H, Hkv, D, causal)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("causal", [False, True])
def test_key_lengths_with_anything_behind_them(dtype, causal):
    """Lengths of none, one, inside and at the end of a tile, all, more than all; NaN and infinities behind them."""
    run_case(dtype, 8, 200, 200, 2, 1, 64, causal, lengths=[0, 1, 63, 64, 65, 199, 200, 1000], poison=True)
    run_case(dtype, 3, 70, 300, 2, 2, 128, causal, lengths=[-5, 129, 256], poison=True, seed=1)


@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_that_see_nothing_give_and_take_nothing(dtype):
    q, k, v, g, out, lse, (gq, gk, gv) = run_case(dtype, 1, 300, 100, 2, 1, 64, True)      # rows 0 .. 199 see no key
    assert (out[:, :200] == 0).all() and (lse[:, :, :200] == -math.inf).all() and (gq[:, :200] == 0).all()
    out0, lse0 = daf.attention(q, k[:, :0], v[:, :0])
    assert (out0 == 0).all() and (lse0 == -math.inf).all()
    a, b, c = daf.attention_grad(q, k[:, :0], v[:, :0], out0, lse0, g)
    assert (a == 0).all() and b.numel() == 0 and c.numel() == 0
    a, b, c = daf.attention_grad(q[:, :0], k, v, out[:, :0], lse[:, :, :0].contiguous(), g[:, :0])
    assert a.numel() == 0 and (b == 0).all() and (c == 0).all()
    assert daf.attention(q[:, :0], k, v)[0].numel() == 0 and daf.attention(q[:0], k[:0], v[:0])[0].numel() == 0


@pytest.mark.parametrize("dtype", DTYPES)
def test_strides_offsets_and_orders(dtype):
    run_case(dtype, 2, 150, 150, 3, 3, 64, True, packed=True)
    # [B, H, S, D] in memory, a slice of a wider head, a misaligned start (copied), a broadcast key head (copied)
    gen = torch.Generator(device="cuda").manual_seed(3)
    base = torch.randn((2, 3, 150, 3, 72), generator=gen, device="cuda").to(dtype)
    q, k, v = (t.transpose(1, 2)[..., :64] for t in base.permute(1, 0, 3, 2, 4))
    plain = [t.contiguous() for t in (q, k, v)]
    out, lse = daf.attention(*plain, causal=True)
    got, got_lse = daf.attention(q, k, v, causal=True)
    assert torch.equal(got, out) and torch.equal(got_lse, lse)
    flat = torch.randn(2 * 150 * 3 * 64 + 1, generator=gen, device="cuda").to(dtype)[1:].view(2, 150, 3, 64)
    assert torch.equal(daf.attention(flat, k, v)[0], daf.attention(flat.clone(), plain[1], plain[2])[0])
    shared = plain[1][:, :, :1].expand(2, 150, 3, 64)
    assert torch.equal(daf.attention(q, shared, shared)[0], daf.attention(q, shared.contiguous(), shared.contiguous())[0])
    # gradients into the slices of one packed tensor
    g = torch.randn((2, 150, 3, 64), generator=gen, device="cuda").to(dtype)
    want = daf.attention_grad(*plain, out, lse, g, causal=True)
    packed = torch.full((2, 150, 3, 3, 64), 7.0, dtype=dtype, device="cuda")
    daf.attention_grad(q, k, v, out, lse, g, causal=True, grads=packed.unbind(2))
    for t, w in zip(packed.unbind(2), want):
        assert torch.equal(t, w)


@pytest.mark.parametrize("dtype", DTYPES)
def test_large_scores_negative_scale_and_repeated_calls(dtype):
    run_case(dtype, 1, 130, 130, 2, 2, 64, False, scale=-0.05, size=1.5, seed=5)
    q, k, v, g, out, lse, grads = run_case(dtype, 2, 300, 300, 4, 2, 64, True, seed=6)
    again = daf.attention_grad(q, k, v, out, lse, g, causal=True)
    for a, b in zip(grads, again):                                  # no atomics: the same bits
        assert torch.equal(a, b)
    # scores far apart: every row is one key's value
    q = torch.zeros((1, 64, 1, 64), device="cuda", dtype=dtype)
    q[0, torch.arange(64), 0, torch.arange(64)] = 100.0
    v = torch.randn((1, 64, 1, 64), device="cuda").to(dtype)
    out, lse = daf.attention(q, q, v, scale=1.0)
    assert torch.equal(out, v) and torch.allclose(lse, torch.full_like(lse, 1e4))


def test_another_stream_and_results_beside_what_belongs_to_others():
    """Work goes to the stream it is given; rows and heads beside the written ones keep their values."""
    s = torch.cuda.Stream()
    q, k, v = (torch.randn((1, 100, 2, 64), device="cuda").bfloat16() for _ in range(3))
    want, _ = daf.attention(q, k, v)
    room = torch.full((1, 102, 4, 64), 3.0, device="cuda", dtype=torch.bfloat16)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        daf.attention(q, k, v, out=room[:, 1:101, 1:3])
    s.synchronize()
    assert torch.equal(room[:, 1:101, 1:3], want)
    room[:, 1:101, 1:3] = 3.0
    assert (room == 3.0).all()


def test_gradients_against_differences():
    """f = sum(out * g) along a random direction, central differences at 1/64: the truncation error is (1/64)^2 / 6 times a
    third derivative of the order of f itself, the differences' rounding 2^-23 |f| 64; 2% of the gradient's size covers both."""
    torch.manual_seed(0)
    q, k, v, g = (torch.randn(1, 90, 2, 64, device="cuda") for _ in range(4))
    out, lse = daf.attention(q, k, v, causal=True)
    grads = daf.attention_grad(q, k, v, out, lse, g, causal=True)
    for i in range(3):
        d = torch.randn_like(q)
        x = [q, k, v]
        f = []
        for sign in (1, -1):
            y = list(x)
            y[i] = x[i] + sign / 64 * d
            f.append((daf.attention(*y, causal=True)[0].double() * g.double()).sum())
        slope, want = float(f[0] - f[1]) * 32, float((grads[i].double() * d.double()).sum())
        assert abs(slope - want) <= 0.02 * float(grads[i].double().norm()), (i, slope, want)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", [2.0 ** -13, 2.0 ** 10])
def test_gradients_far_from_one(dtype, size):
    """Gradients scale with grad_out: a power of two more or less in every element of grad_out is the same power of two in
    every gradient, up to the results' own subnormals (float16 results are kept normal by the other inputs)."""
    gen = torch.Generator(device="cuda").manual_seed(11)
    q, k, v, g = (torch.randn((2, 300, 2, 64), generator=gen, device="cuda").to(dtype) for _ in range(4))
    g = (g.float().clamp(-4, 4) + 0.0).to(dtype)
    out, lse = daf.attention(q, k, v)
    base = daf.attention_grad(q, k, v, out, lse, g)
    got = daf.attention_grad(q, k, v, out, lse, (g.float() * size).to(dtype))
    tiny = 2.0 ** -24 if dtype == torch.float16 else 0.0           # half an ulp of a subnormal result
    u = 0.0 if dtype != torch.float16 else 2.0 ** -10               # g * 2^-13 rounds where it falls below 2^-14
    for a, b in zip(got, base):
        a, b = a.double(), b.double() * size
        assert torch.isfinite(a).all() and (a - b).norm() <= u * b.norm() + tiny * math.sqrt(b.numel())


def test_a_stream_by_argument_takes_the_copies_along():
    """Work that is asked for on a stream happens there, the copies of tensors the kernels cannot address included: that stream
    holds everything up, the current one does not."""
    s = torch.cuda.Stream()
    base = torch.randn(2 * 90 * 2 * 64 + 1, device="cuda").bfloat16()
    q = base[1:].view(2, 90, 2, 64)                                 # off its 16-byte boundary
    want, want_lse = daf.attention(q, q, q, causal=True)
    g = torch.randn(2, 90, 2, 64, device="cuda").bfloat16()
    grads = daf.attention_grad(q, q, q, want, want_lse, g, causal=True)
    torch.cuda.synchronize()
    later = torch.zeros_like(base)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
        later.copy_(base)
    q = later[1:].view(2, 90, 2, 64)
    out, lse = daf.attention(q, q, q, causal=True, stream=s)
    got = daf.attention_grad(q, q, q, out, lse, g, causal=True, stream=s)
    s.synchronize()
    assert torch.equal(out, want) and torch.equal(lse, want_lse) and all(torch.equal(a, b) for a, b in zip(got, grads))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B,Sq,Sk,H,Hkv,D,causal,lengths", [
    (1, 1, 8000, 2, 1, 128, False, None), (3, 5, 4100, 2, 2, 64, True, [0, 4100, 130]), (1, 300, 3000, 1, 1, 80, True, None),
    (2, 1, 1153, 1, 1, 40, False, [1153, 1])])
def test_few_rows_over_many_keys(dtype, B, Sq, Sk, H, Hkv, D, causal, lengths):
    """Calls that leave most of the GPU idle are split over the keys and joined; the same bounds, and the same bits twice."""
    q, k, v, g, out, lse, _ = run_case(dtype, B, Sq, Sk, H, Hkv, D, causal, lengths=lengths, poison=lengths is not None)
    lens = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    again, again_lse = daf.attention(q, k, v, causal=causal, key_lengths=lens)
    assert torch.equal(again, out) and torch.equal(again_lse, lse)
