"""Orthogonalised updates against the iteration in 64 bits."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
import paper_2507_07149_b200 as daf  # noqa: E402

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
A, B, C = 3.4445, -4.7750, 2.0315
HELD = 4096.0


def exact(g, steps=5, abc=(A, B, C), eps=1e-7):
    x = g.double().reshape(g.shape[0], -1)
    tall = x.shape[0] > x.shape[1]
    x = x.t() if tall else x
    x = x / (x.norm() + eps)
    a, b, c = (torch.tensor(v, dtype=torch.float32).double() for v in abc)
    for _ in range(steps):
        p = x @ x.t()
        x = a * x + (b * p + c * p @ p) @ x
    return (x.t() if tall else x).reshape(g.shape)


def cut(t, scale, planes):
    """What float16 parts (one, or two) of t * scale hold of t."""
    hi = (t * scale).half().double()
    return (hi + ((t * scale - hi).half().double() if planes == 2 else 0)) / scale


def model(g, planes, steps=5, eps=1e-7):
    """The iteration in 64 bits with the roundings that are documented and no others: the first x exact up to a power of two,
    Gram matrices, polynomials and x in float16 parts, a x from two parts behind the first two steps."""
    x = g.double().reshape(g.shape[0], -1)
    tall = x.shape[0] > x.shape[1]
    x = x.t() if tall else x
    norm = (x.norm() + eps).item()
    k = norm * 2.0 ** (12 - math.floor(math.log2(norm)))
    x = cut(x / norm, k, planes)
    for i in range(steps):
        op = cut(x, k, planes)
        p = cut(op @ op.t(), HELD, planes)
        y = A * x + cut(B * p + C * p @ p, HELD, planes) @ op
        x = y if i + 1 == steps else cut(y, k, 2 if planes == 2 or i < 2 else 1)
    return (x.t() if tall else x).reshape(g.shape)


def apart(got, want):
    return ((got.double() - want).norm() / want.norm()).item()


def gradient(shape, dtype, seed, kind="strong"):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r, c = shape[0], math.prod(shape[1:])
    x = torch.randn((r, c), generator=g, device="cuda")
    if kind == "strong":                                           # some directions far stronger than the others
        k = max(1, min(r, c) // 4)
        x = 0.1 * x + (torch.randn((r, k), generator=g, device="cuda") / (1 + torch.arange(k, device="cuda"))) @ torch.randn((k, c), generator=g, device="cuda")
    return (0.01 * x).reshape(shape).to(TYPES[dtype])


SHAPES = [(1, 1), (1, 300), (300, 1), (8, 64), (63, 65), (64, 64), (65, 63), (128, 256), (129, 127), (200, 1000), (1000, 200), (257, 257), (512, 130), (384, 1111),
          (1024, 768), (640, 2100)]


# One rounding to the result's type, the roundings of `model` (those of the kernel are others of the same sizes, hence twice), and the
# products' sums: the tensor cores cut each of n / 16 partial sums at 2^-23 or better of the sum, and a step multiplies relative errors
# by at most five in the part of the spectrum that ends near one (|p'(s)| s / p(s) for s up to 1.2), mostly by less: 100 n / 16 2^-23.
@pytest.mark.parametrize("kind", ["strong", "flat"])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_against_64_bits(shape, dtype, kind):
    g = gradient(shape, dtype, 3 + shape[0], kind)
    got, = daf.orthogonalize([g], check=True)
    assert got.dtype == g.dtype and got.shape == g.shape
    want = exact(g)
    of_model = apart(model(g, 1 if dtype == "bf16" else 2), want)
    bound = torch.finfo(g.dtype).eps / 2 + 2 * of_model + 100 * max(shape) / 16 * 2.0 ** -23
    assert apart(got, want) <= bound, (apart(got, want), of_model)


# held in binary64: one rounding, to the result's type, and what 5 steps of sums of 1030 products in binary64 are off, times a hundred
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("shape", [(1, 1), (1, 2), (2, 5), (3, 1), (4, 1031), (1031, 3), (5, 515), (32, 32), (32, 128), (127, 32), (29, 129), (17, 200), (9, 3, 5)],
                         ids=lambda s: "x".join(map(str, s)))
def test_smallest_matrices(shape, dtype):
    g = gradient(shape, dtype, 21)
    got, = daf.orthogonalize([g], check=True)
    want = exact(g)
    slack = 100 * 5 * 1031 * 2.0 ** -53 * want.norm()
    t = g.dtype
    assert ((got.double() - want).abs() <= torch.finfo(t).eps / 2 * want.abs() + slack + (2.0 ** -25 if t == torch.float16 else 0.0)).all()


# held in binary32: a sum of n products is at most n / 16 + 32 additions deep (parts of 16 columns or more, 64 parts at most, 16 or more of
# a long sum), each off by 2^-24, in three products a step; the largest of these shapes and the next ones, which are not held by one CTA
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(1, 1033), (4103, 1), (4, 4105), (5, 517), (32, 129), (32, 513), (513, 32), (512, 32), (32, 514), (33, 33), (1300, 12), (12, 1368)],
                         ids=lambda s: "x".join(map(str, s)))
def test_small_matrices(shape, dtype):
    g = gradient(shape, dtype, 22)
    got, = daf.orthogonalize([g], check=True)
    want = exact(g)
    of_model = apart(model(g, 1 if dtype == "bf16" and min(shape) > 32 else 2), want)
    assert apart(got, want) <= torch.finfo(g.dtype).eps / 2 + 2 * of_model + 100 * 3 * (max(shape) / 16 + 32) * 2.0 ** -24


def test_small_matrices_among_others():
    """Those of one CTA run beside the products of the others, more of them than go together, in place, in a graph."""
    shapes = [(2, 5), (300, 700), (32, 500)] * 3 + [(16, 40)] * 200 + [(30, 400)] * 195 + [(64, 9000), (0, 4), (4, 0)]
    gs = [gradient(s, ("bf16", "f32", "f16")[i % 3], 30 + i) if 0 not in s else torch.zeros(s, device="cuda") for i, s in enumerate(shapes)]
    want = [daf.orthogonalize([g], check=True)[0] for g in gs]
    assert all(torch.equal(a, b) for a, b in zip(daf.orthogonalize(gs, check=True), want))
    for order in (slice(None, None, -1), slice(None, None, 7)):
        assert all(torch.equal(a, b) for a, b in zip(daf.orthogonalize(gs[order], check=True), want[order]))
    held = [g.clone() for g in gs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        after = [2 * x for x in daf.orthogonalize(held, out=held)]
    for _ in range(3):
        for h, g in zip(held, gs):
            h.copy_(g)
        graph.replay()
        assert all(torch.equal(a, 2 * b) for a, b in zip(after, want)) and all(torch.equal(a, b) for a, b in zip(held, want))
    one = gradient((8, 20), "f32", 50)
    one[3, 4] = math.inf
    assert daf.orthogonalize([one])[0].isnan().all()
    assert not daf.orthogonalize([torch.zeros((8, 20), device="cuda")])[0].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(100, 333), (333, 100), (256, 256), (31, 2050)], ids=lambda s: "x".join(map(str, s)))
def test_one_step_element_by_element(shape, dtype):
    """y = a x + (b G + c G^2) x: every rounding is at most u of the magnitudes that enter it."""
    g = gradient(shape, dtype, 9)
    got, = daf.orthogonalize([g], steps=1, check=True)
    want = exact(g, 1)
    x = g.double().t() if shape[0] > shape[1] else g.double()
    x = (x / (x.norm() + 1e-7)).abs()
    gram = x @ x.t()
    once, twice = gram @ x, gram @ (gram @ x)
    u = 2.0 ** -11 if dtype == "bf16" else 2.0 ** -22              # float16 parts: half a step, doubled for what is below the normal range
    acc = max(shape) / 16 * 2.0 ** -22
    off = (abs(B) * once * 3 + C * twice * 4) * (u + acc) + x * 2.0 ** -20 + 2.0 ** -34
    off = off.t() if shape[0] > shape[1] else off
    bound = off + torch.finfo(g.dtype).eps / 2 * (want.abs() + off)
    assert ((got.double() - want).abs() <= bound).all()


@pytest.mark.parametrize("shape,dtype", [((1, 65536), "f32"), ((65536, 2), "bf16"), ((40000, 24), "f16"), ((24, 16000), "f32")], ids=lambda s: str(s))
def test_long_sides(shape, dtype):
    """As above; sums in segments keep binary32's loss per addition from adding up, float16 takes them above 8192."""
    g = gradient(shape, dtype, 7, "flat")
    got, = daf.orthogonalize([g], check=True)
    want = exact(g)
    segments = 100 * 2.0 ** -23 * (max(shape) / 16 if dtype == "bf16" else 8 + max(shape) ** 0.5 / 16)
    assert apart(got, want) <= torch.finfo(g.dtype).eps / 2 + 2 * apart(model(g, 1 if dtype == "bf16" else 2), want) + segments


def test_singular_values_end_near_one():
    for shape in ((768, 2304), (900, 500)):
        got, = daf.orthogonalize([gradient(shape, "bf16", 1, "flat")])
        s = torch.linalg.svdvals(got.double())
        # p maps [0.05, 1.2] into itself's upper part: five steps from 0.005 of the norm end in [0.65, 1.25]
        assert s.max() < 1.27 and s[:-5].min() > 0.6


def test_many_matrices_together():
    shapes = [(48, 80), (80, 48), (48, 80), (7, 5), (300, 200), (200, 300), (1, 9), (64, 3, 3, 3), (256, 256)]
    types = ["bf16", "f32", "bf16", "f16", "bf16", "bf16", "f32", "bf16", "f16"]
    gs = [gradient(s, t, 20 + i) for i, (s, t) in enumerate(zip(shapes, types))]
    got = daf.orthogonalize(gs, check=True)
    for g, o in zip(gs, got):
        # a matrix's tiles may have another width among others; its sums are the same
        assert torch.equal(o, daf.orthogonalize([g])[0])
    again = daf.orthogonalize(gs)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


def test_more_shapes_and_matrices_than_a_launch_holds():
    gs = [gradient((8 + i % 40, 8 + i % 30), "bf16", i) for i in range(230)]
    got = daf.orthogonalize(gs, check=True)
    for i in (0, 23, 24, 100, 191, 192, 229):
        assert torch.equal(got[i], daf.orthogonalize([gs[i]])[0])


def test_in_place_layouts_and_guards():
    for dtype in ("bf16", "f32", "f16"):
        g = gradient((33, 41), dtype, 2)
        want, = daf.orthogonalize([g])
        room = torch.full((33 * 41 + 65,), 7.0, dtype=TYPES[dtype], device="cuda")
        for off in (0, 1, 8):
            room.fill_(7.0)
            out = room[off:off + 33 * 41].view(33, 41)
            assert daf.orthogonalize([g], out=[out])[0] is out and torch.equal(out, want)
            assert (room[:off] == 7).all() and (room[off + 33 * 41:] == 7).all()
            out.copy_(g)                                            # an input off the boundaries, in place
            daf.orthogonalize([out], out=[out])
            assert torch.equal(out, want)
        across = g.t().contiguous().t()
        assert torch.equal(daf.orthogonalize([across])[0], want)
    g = gradient((32, 48), "bf16", 5)
    apart_ = torch.empty((32, 96), dtype=g.dtype, device="cuda")[:, ::2]
    apart_.copy_(g)
    assert torch.equal(daf.orthogonalize([apart_])[0], daf.orthogonalize([g])[0])


def test_sizes_of_values():
    g = gradient((96, 160), "f32", 4)
    want, = daf.orthogonalize([g * 2.0 ** 10])
    for up in (60, 100):                                            # squares that would leave binary32
        got, = daf.orthogonalize([g * 2.0 ** up])
        assert apart(got, exact(g * 2.0 ** up)) <= 1e-4
    small, = daf.orthogonalize([g * 2.0 ** -90], eps=1e-30)
    assert apart(small, exact(g * 2.0 ** -90, eps=1e-30)) <= 1e-4 and apart(want, exact(g * 2.0 ** 10)) <= 1e-4
    zero, = daf.orthogonalize([torch.zeros((20, 30), device="cuda")])
    assert not zero.any()
    for bad in (math.nan, math.inf):
        h = g.clone()
        h[3, 5] = bad
        broken, fine = daf.orthogonalize([h, g])
        assert broken.isnan().all() and torch.equal(fine, daf.orthogonalize([g])[0])


def test_other_coefficients_and_steps():
    g = gradient((120, 70), "f32", 8)
    for steps, abc in ((1, (1.5, -0.5, 0.0)), (12, (1.875, -1.25, 0.375)), (2, (A, B, C))):
        got, = daf.orthogonalize([g], steps=steps, coefficients=abc)
        assert apart(got, exact(g, steps, abc)) <= 1e-4


def test_empty_calls():
    assert daf.orthogonalize([]) == []
    a, b = daf.orthogonalize([torch.empty((0, 5), device="cuda"), torch.empty((4, 0), device="cuda")], check=True)
    assert a.shape == (0, 5) and b.shape == (4, 0)


def test_other_streams_and_graphs():
    gs = [gradient(s, "bf16", 30 + i) for i, s in enumerate([(64, 128), (256, 100)])]
    want = daf.orthogonalize(gs)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = daf.orthogonalize(gs, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = daf.orthogonalize(gs)
    gs[0].copy_(gs[0].flip(0))
    for _ in range(3):
        graph.replay()
    assert torch.equal(got[0], daf.orthogonalize(gs)[0]) and torch.equal(got[1], want[1])
    daf.check_device()


def test_two_calls_at_once():
    gs = [[gradient((300 + 50 * j, 700), "bf16", 40 + j + 10 * i) for j in range(3)] for i in range(2)]
    want = [daf.orthogonalize(g) for g in gs]
    torch.cuda.synchronize()
    sides = [torch.cuda.Stream() for _ in gs]
    for _ in range(3):
        got = [daf.orthogonalize(g, stream=s) for g, s in zip(gs, sides)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for w, o in zip(want, got) for a, b in zip(w, o))
    daf.check_device()


def test_refusals():
    g = torch.randn((8, 8), device="cuda")
    for bad in (lambda: daf.orthogonalize([g[0]]), lambda: daf.orthogonalize([g.cpu()]), lambda: daf.orthogonalize([g.double()]), lambda: daf.orthogonalize([g, g.cpu()]),
                lambda: daf.orthogonalize([g], steps=0), lambda: daf.orthogonalize([g], steps=65), lambda: daf.orthogonalize([g], coefficients=(1.0, 2.0)),
                lambda: daf.orthogonalize([g], out=[]), lambda: daf.orthogonalize([g], out=[g.half()]), lambda: daf.orthogonalize([g], out=[torch.empty((8, 16), device="cuda")[:, ::2]]),
                lambda: daf.orthogonalize([1.0])):
        with pytest.raises(ValueError):
            bad()
    for bad in (dict(eps=0.0), dict(eps=math.nan), dict(coefficients=(1.0, math.inf, 0.0))):
        with pytest.raises(daf.DafError):
            daf.orthogonalize([g], **bad)
    with pytest.raises(daf.DafError):
        daf.orthogonalize([torch.zeros((1, 65537), device="cuda")])
