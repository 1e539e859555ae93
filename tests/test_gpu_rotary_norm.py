"""Norms of queries and keys with the rotation by position, and their gradients, against the definitions in 64 bits."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
import paper_2507_07149_b200 as daf  # noqa: E402

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SMALLEST = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -133}


def angles(positions, pairs, rotary, base=10000.0, frequencies=None):
    f = torch.tensor([base ** (-2.0 * i / rotary) for i in range(pairs)] if frequencies is None else frequencies, dtype=torch.float64, device="cuda")
    return positions.double()[..., None, None] * f                  # [B, S, 1, pairs]


def pairs_of(rotary, style):
    i = torch.arange(rotary // 2, device="cuda")
    return (i, i + rotary // 2) if style == "halves" else (2 * i, 2 * i + 1)


def turned(x, angle, first, second):
    y = x.clone()
    c, s = torch.cos(angle), torch.sin(angle)
    y[..., first] = x[..., first] * c - x[..., second] * s
    y[..., second] = x[..., first] * s + x[..., second] * c
    return y


def spread(x, first, second):
    """|a| + |b| of each pair, |x| of what is not turned: what an error of the cosines and sines is multiplied with."""
    y = x.abs()
    y[..., first] = x[..., first].abs() + x[..., second].abs()
    y[..., second] = y[..., first]
    return y


# Relative error of a product with a cosine or sine: theirs (binary32: two units in the last place, 2^-22, of at most one; 16-bit: 2^-21.1 in
# absolute terms) and the angle's (its fraction of a turn is cut at 2^-32 turns and rounded to 24 bits: pi 2^-24 + 2 pi 2^-32), and two
# roundings; of the norm: D / 2 + 6 roundings (sum of squares of D terms, halved by the root; two units of the root itself).
def slack(dtype, d, more=0):
    turn = (2.0 ** -22 if dtype == torch.float32 else 2.0 ** -21.0) + math.pi * 2.0 ** -24 + 2.0 ** -28
    return turn + (d / 2 + 10 + more) * 2.0 ** -24


def near(got, want, off_by):
    half = torch.finfo(got.dtype).eps / 2
    bound = off_by + half * (want.abs() + off_by) + SMALLEST[got.dtype] / 2
    off = (got.double() - want).abs()
    assert (off <= bound).all(), f"off by {off.max().item()}, {(off / bound).max().item()} of the bound"


def forward(x, w, positions, rotary, style, eps, **how):
    first, second = pairs_of(rotary, style)
    x, w = x.double(), 1.0 if w is None else w.double()
    n = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w
    angle = angles(positions, rotary // 2, rotary, **how) if rotary else None
    return (turned(n, angle, first, second) if rotary else n), spread(n, first, second)


def backward(x, w, g, positions, rotary, style, eps, **how):
    """dx, dw and what their errors are proportional to."""
    first, second = pairs_of(rotary, style)
    d = x.shape[-1]
    x, g, w = x.double(), g.double(), torch.ones(d, dtype=torch.float64, device="cuda") if w is None else w.double()
    r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    hat = x * r
    back = turned(g, -angles(positions, rotary // 2, rotary, **how), first, second) if rotary else g
    size = spread(g, first, second)
    dx = r * (back * w - hat * (back * w * hat).mean(-1, keepdim=True))
    dx_size = r * (size * w.abs() + hat.abs() * (size * w.abs() * hat.abs()).mean(-1, keepdim=True))
    return dx, (back * hat).sum((0, 1, 2)), dx_size, (size * hat.abs()).sum((0, 1, 2))


CASES = [  # dtype, params, B, S, H, Hkv, D, rotary, style
    ("bf16", "bf16", 1, 1, 1, 1, 8, 8, "halves"), ("bf16", "f32", 3, 7, 4, 2, 64, 64, "halves"), ("f16", "f16", 2, 33, 6, 6, 80, 80, "halves"),
    ("f16", "f32", 1, 130, 5, 1, 72, 72, "pairs"), ("f32", "f32", 2, 19, 3, 3, 40, 40, "halves"), ("f32", "f32", 1, 61, 12, 4, 128, 64, "pairs"),
    ("bf16", "bf16", 1, 257, 16, 4, 128, 128, "halves"), ("bf16", "f32", 2, 40, 9, 3, 256, 128, "halves"), ("bf16", "bf16", 4, 5, 20, 1, 96, 24, "pairs"),
    ("f16", "f32", 1, 300, 3, 2, 112, 0, "halves"), ("f32", "f32", 5, 1, 17, 17, 256, 256, "halves"), ("bf16", "f32", 64, 40, 12, 12, 64, 64, "halves"),
    ("f32", "f32", 1, 2000, 24, 8, 32, 16, "halves"), ("bf16", "bf16", 2, 9, 1, 1, 24, 16, "pairs")]


def made(case, seed, packed):
    dtype, params, b, s, h, kv, d, rotary, style = case
    dt, pt = TYPES[dtype], TYPES[params]
    g = torch.Generator(device="cuda").manual_seed(seed)
    if packed:
        q, k, _ = torch.randn((b, s, h + 2 * kv, d), generator=g, device="cuda").to(dt).split((h, kv, kv), 2)
    else:
        q, k = (torch.randn((b, s, n, d), generator=g, device="cuda").to(dt) * 3 for n in (h, kv))
    w = [(1 + 0.3 * torch.randn(d, generator=g, device="cuda")).to(pt) for _ in range(2)]
    grads = [torch.randn((b, s, n, d), generator=g, device="cuda").to(dt) for n in (h, kv)]
    at = torch.randint(-50, 1 << 20, (b, s), generator=g, device="cuda", dtype=torch.int32 if b % 2 else torch.int64)
    return q, k, w, grads, at


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_forward_and_gradient(case, packed):
    rotary, style, d = case[7], case[8], case[6]
    q, k, w, grads, at = made(case, 11, packed)
    how = dict(positions=at, rotary_dim=rotary, style=style)
    out = daf.rotary_norm(q, k, *w, **how)
    got = daf.rotary_norm_grad(q, k, *w, *grads, **how)
    assert all(torch.equal(a, b) for a, b in zip(got, daf.rotary_norm_grad(q, k, *w, *grads, **how)))
    for i, x in enumerate((q, k)):
        want, size = forward(x, w[i], at, rotary, style, 1e-6)
        near(out[i], want, slack(x.dtype, d) * size)
        dx, dw, dx_size, dw_size = backward(x, w[i], grads[i], at, rotary, style, 1e-6)
        near(got[i], dx, slack(x.dtype, 2 * d) * dx_size)
        rows = x.shape[0] * x.shape[1] * x.shape[2]
        near(got[2 + i], dw, slack(x.dtype, d, rows) * dw_size)     # a sum of `rows` terms


def test_differences():
    case = ("f32", "f32", 1, 3, 2, 1, 16, 16, "halves")
    q, k, w, grads, at = made(case, 3, False)
    gq, gk, gwq, gwk = daf.rotary_norm_grad(q, k, *w, *grads, positions=at)

    def loss(q, k, w):
        return sum((forward(x, w[i], at, 16, "halves", 1e-6)[0] * grads[i].double()).sum() for i, x in enumerate((q, k)))
    h = 1e-6
    for name, t, got in (("q", q, gq), ("k", k, gk), ("wq", w[0], gwq), ("wk", w[1], gwk)):
        for j in range(0, t.numel(), 7):
            sides = []
            for sign in (1, -1):
                moved = t.double().clone()
                moved.view(-1)[j] += sign * h
                sides.append(loss(moved if name == "q" else q, moved if name == "k" else k, [moved if name == "wq" else w[0], moved if name == "wk" else w[1]]))
            slope = ((sides[0] - sides[1]) / (2 * h)).item()
            assert abs(got.reshape(-1)[j].item() - slope) <= 1e-4 * (1 + abs(slope)), (name, j)    # rounding of the loss / h is about 1e-8


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_far_positions(dtype):
    # the angle is exact modulo a turn: positions up to 2^40 need 64 bits and more, here by rational arithmetic
    from fractions import Fraction
    from decimal import Decimal, getcontext
    getcontext().prec = 60
    two_pi = Fraction(Decimal("6.283185307179586476925286766559005768394338798750211641949889"))
    f = [1.0, 0.1, 2.0 ** -20, 3.0]
    at = torch.tensor([0, -1, 1 << 20, (1 << 40) + 12345, -(1 << 35) - 1, 2 ** 31 - 1], device="cuda")
    q = torch.zeros((1, 6, 1, 8), dtype=TYPES[dtype], device="cuda")
    q[..., :4] = 1.0
    out, none = daf.rotary_norm(q, None, positions=at, frequencies=f, eps=0.0)
    assert none is None
    for s, p in enumerate(at.tolist()):
        for i, w in enumerate(f):
            turns = Fraction(w) * p / two_pi
            a = float((turns - math.floor(turns)) * two_pi)
            # n = sqrt(2); the frequency itself is held to 2^-65 turns: p 2^-65 turns off
            off = math.sqrt(2) * (slack(q.dtype, 8) + 2 * math.pi * abs(p) * 2.0 ** -64) + torch.finfo(q.dtype).eps
            assert abs(out[0, s, 0, i].item() - math.sqrt(2) * math.cos(a)) <= off and abs(out[0, s, 0, 4 + i].item() - math.sqrt(2) * math.sin(a)) <= off


def test_forms_of_positions():
    case = ("bf16", "f32", 3, 21, 4, 2, 64, 64, "halves")
    q, k, w, _, _ = made(case, 5, True)
    at = torch.arange(100, 121, device="cuda")
    want = daf.rotary_norm(q, k, *w, positions=at.expand(3, 21).contiguous())
    for same in (daf.rotary_norm(q, k, *w, positions=at), daf.rotary_norm(q, k, *w, positions=at.int()), daf.rotary_norm(q, k, *w, positions=100),
                 daf.rotary_norm(q, k, *w, positions=at.int().expand(3, 21))):
        assert torch.equal(same[0], want[0]) and torch.equal(same[1], want[1])
    zero = daf.rotary_norm(q, k, *w, positions=0)
    assert torch.equal(zero[0], daf.rotary_norm(q, k, *w)[0])
    # one token after another as a decoder takes them
    for i in (0, 20):
        one = daf.rotary_norm(q[:, i:i + 1], k[:, i:i + 1], *w, positions=100 + i)
        assert torch.equal(one[0], want[0][:, i:i + 1]) and torch.equal(one[1], want[1][:, i:i + 1])


def test_without_weights_and_without_keys():
    case = ("f16", "f32", 2, 5, 3, 3, 32, 32, "pairs")
    q, k, w, grads, at = made(case, 6, False)
    ones = torch.ones(32, device="cuda")
    bare, weighted = daf.rotary_norm(q, k, positions=at, style="pairs"), daf.rotary_norm(q, k, ones, ones, positions=at, style="pairs")
    assert torch.equal(bare[0], weighted[0]) and torch.equal(bare[1], weighted[1])
    g = daf.rotary_norm_grad(q, k, None, w[1], *grads, positions=at, style="pairs")
    assert g[2] is None and torch.equal(g[3], daf.rotary_norm_grad(q, k, w[0], w[1], *grads, positions=at, style="pairs")[3])
    alone = daf.rotary_norm_grad(q, None, w[0], w[1], grads[0], None, positions=at, style="pairs")
    both = daf.rotary_norm_grad(q, k, w[0], w[1], *grads, positions=at, style="pairs")
    assert torch.equal(alone[0], both[0]) and alone[1] is None and torch.equal(alone[2], both[2]) and not alone[3].any()


def test_in_place_outputs_and_guards():
    case = ("bf16", "f32", 2, 11, 4, 2, 40, 40, "halves")
    q, k, w, grads, at = made(case, 7, False)
    want, want_g = daf.rotary_norm(q, k, *w, positions=at), daf.rotary_norm_grad(q, k, *w, *grads, positions=at)
    room = torch.full((2, 11, 10, 40), 7.0, dtype=torch.bfloat16, device="cuda")     # a packed gradient: q, k, and v's place
    gq, gk, gv = room.split((4, 2, 4), 2)
    got = daf.rotary_norm_grad(q, k, *w, *grads, positions=at, grads=(gq, gk))
    assert torch.equal(gq, want_g[0]) and torch.equal(gk, want_g[1]) and (gv == 7).all() and torch.equal(got[2], want_g[2])
    daf.rotary_norm_grad(q, k, *w, *grads, positions=at, grads=tuple(grads))          # onto the incoming gradients
    assert torch.equal(grads[0], want_g[0]) and torch.equal(grads[1], want_g[1])
    a, b = daf.rotary_norm(q, k, *w, positions=at, out=(q, k))
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and a.data_ptr() == q.data_ptr()


def test_layouts_that_are_copied():
    case = ("bf16", "f32", 2, 6, 4, 2, 24, 24, "halves")
    q, k, w, grads, at = made(case, 8, False)
    want = daf.rotary_norm(q, k, *w, positions=at)
    apart = torch.empty((2, 6, 4, 48), dtype=q.dtype, device="cuda")[..., ::2]
    apart.copy_(q)
    off = torch.empty(k.numel() + 1, dtype=k.dtype, device="cuda")[1:].view(k.shape)
    off.copy_(k)
    got = daf.rotary_norm(apart, off, *w, positions=at)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    heads_first = q.transpose(1, 2).contiguous().transpose(1, 2)
    assert torch.equal(daf.rotary_norm(heads_first, k, *w, positions=at)[0], want[0])
    shared = daf.rotary_norm(q[:, :, :1].expand(2, 6, 4, 24), k, *w, positions=at)[0]    # broadcast heads
    assert torch.equal(shared, want[0][:, :, :1].expand(2, 6, 4, 24))
    g1 = daf.rotary_norm_grad(q, k, *w, grads[0][:, :, :1].expand(2, 6, 4, 24), grads[1], positions=at)
    g2 = daf.rotary_norm_grad(q, k, *w, grads[0][:, :, :1].expand(2, 6, 4, 24).contiguous(), grads[1], positions=at)
    assert all(torch.equal(a, b) for a, b in zip(g1, g2))


def test_rows_of_zeros_and_values_that_are_not_finite():
    q = torch.randn((1, 4, 2, 16), device="cuda")
    q[0, 0, 0] = 0.0
    q[0, 1, 1, 3] = math.nan
    q[0, 2, 0, 5] = math.inf
    out, _ = daf.rotary_norm(q, None)
    assert not out[0, 0, 0].any() and out[0, 1, 1].isnan().all()
    fine = torch.ones((4, 2), dtype=torch.bool, device="cuda")
    fine[1, 1] = fine[2, 0] = False
    assert out[0][fine].isfinite().all()
    g = daf.rotary_norm_grad(q, None, None, None, torch.ones_like(q), None)[0]
    assert g[0][fine].isfinite().all() and g[0, 1, 1].isnan().all()


def test_empty_calls():
    w = torch.ones(32, device="cuda")
    q, k = torch.empty((2, 0, 4, 32), device="cuda"), torch.empty((2, 0, 2, 32), device="cuda")
    assert daf.rotary_norm(q, k, w, w)[1].shape == k.shape
    g = daf.rotary_norm_grad(q, k, w, w, q, k)
    assert g[0].shape == q.shape and not g[2].any() and not g[3].any()


def test_other_streams_and_graphs():
    case = ("bf16", "f32", 2, 100, 4, 2, 64, 64, "halves")
    q, k, w, grads, at = made(case, 9, True)
    want = daf.rotary_norm_grad(q, k, *w, *grads, positions=at)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = daf.rotary_norm_grad(q, k, *w, *grads, positions=at, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got, out = daf.rotary_norm_grad(q, k, *w, *grads, positions=at), daf.rotary_norm(q, k, *w, positions=at)
    at.add_(1000)
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(got, daf.rotary_norm_grad(q, k, *w, *grads, positions=at)))
    assert torch.equal(out[0], daf.rotary_norm(q, k, *w, positions=at)[0])


def test_refusals():
    q, k, w = torch.randn((2, 3, 4, 32), device="cuda"), torch.randn((2, 3, 2, 32), device="cuda"), torch.ones(32, device="cuda")
    at = torch.zeros((2, 3), dtype=torch.int32, device="cuda")
    for bad in (lambda: daf.rotary_norm(q[0], k), lambda: daf.rotary_norm(q, k[:1]), lambda: daf.rotary_norm(q, k.half()), lambda: daf.rotary_norm(q.cpu(), k.cpu()),
                lambda: daf.rotary_norm(q, k.cpu()), lambda: daf.rotary_norm(q, k, w[:16]), lambda: daf.rotary_norm(q, k, w.half()),
                lambda: daf.rotary_norm(q.half(), k.half(), w, w.half()), lambda: daf.rotary_norm(q, k, positions=at.float()),
                lambda: daf.rotary_norm(q, k, positions=at[:, :2]), lambda: daf.rotary_norm(q, k, positions=at.cpu()), lambda: daf.rotary_norm(q, k, rotary_dim=40),
                lambda: daf.rotary_norm(q, k, style="thirds"), lambda: daf.rotary_norm(q, k, frequencies=[1.0]), lambda: daf.rotary_norm(q, k, out=(q, k[:1])),
                lambda: daf.rotary_norm(q.double(), k.double()), lambda: daf.rotary_norm_grad(q, k, w, w, q, None), lambda: daf.rotary_norm_grad(q, k, w, w, q[:1], k),
                lambda: daf.rotary_norm(q, None, out=(q, k))):
        with pytest.raises(ValueError):
            bad()
    for bad in (dict(rotary_dim=12), dict(base=0.0), dict(base=math.inf), dict(eps=-1.0), dict(eps=math.nan), dict(frequencies=[math.nan] * 16)):
        with pytest.raises(daf.DafError):
            daf.rotary_norm(q, k, **bad)
    with pytest.raises(daf.DafError):
        daf.rotary_norm(q[..., :12].contiguous(), k[..., :12].contiguous())
    with pytest.raises(daf.DafError):
        daf.rotary_norm(torch.zeros((1, 1, 1, 264), device="cuda"), None)
