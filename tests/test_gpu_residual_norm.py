"""The join between blocks (gate, residual scale, norms on both sides) and its backward pass against 64 bits.

Bounds: an output is a binary32 value within 2^-18 of the size of the terms it is made of (rows of up to 8192 terms are
summed by a tree, the steps before the sum lose a few 2^-24 each), rounded once to its type (u); column sums over R rows
add at most R terms one after another per CTA: sqrt(R) 2^-24 of the terms' absolute sum is generous for R <= 2^12."""
import pytest

import paper_2507_07149_b200 as daf

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
F32 = 2.0 ** -18
DTYPES = [torch.float32, torch.float16, torch.bfloat16]


def make(dtype, pdt, rows, C, gates, post, bias, offset=0.0, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def rnd(*shape, to=dtype, size=1.0, at=0.0):
        return (torch.randn(shape, generator=gen, device="cuda") * size + at).to(to)
    t = {"x": rnd(rows, C, at=offset), "y": rnd(rows, C, at=offset / 2), "weight": rnd(C, to=pdt, size=0.3, at=1.0),
         "bias": rnd(C, to=pdt) if bias else None,
         "gate": None if not gates else rnd(C, to=pdt) if gates == 1 else rnd(gates, C, to=pdt),
         "post_weight": rnd(C, to=pdt, size=0.3, at=0.5) if post else None,
         "post_bias": rnd(C, to=pdt) if post and bias else None, "gz": rnd(rows, C), "gh": rnd(rows, C)}
    return t


def norm64(t, layer, eps):
    m = t.mean(1, keepdim=True) if layer else torch.zeros_like(t[:, :1])
    r = (((t - m) ** 2).mean(1, keepdim=True) + eps).rsqrt()
    # the size of what the kernel's terms are made of: |t| + |mean| before the cancellation
    return (t - m) * r, r, (t.abs() + m.abs()) * r


def full_gate(t, rows):
    if t["gate"] is None:
        return torch.ones(1, 1, dtype=torch.float64, device="cuda")
    g = t["gate"].double()
    return g[None] if g.dim() == 1 else g.repeat_interleave(rows // g.shape[0], 0)


def close(got, want, size, u, what):
    off, bound = (got.double() - want).abs(), 1.01 * u * want.abs() + F32 * size + (2.0 ** -24 if u == 2.0 ** -11 else 0.0)
    assert torch.isfinite(got).all() and (off <= bound).all(), f"{what}: off by {float((off / bound).max()):.2f} bounds"


def run_case(dtype, pdt, rows, C, gates, post, bias, kind, a=0.75, eps=1e-6, offset=0.0, with_gz=True, seed=0):
    t = make(dtype, pdt, rows, C, gates, post, bias, offset, seed)
    layer, u, pu = kind == "layer", U[dtype], U[pdt]
    how = dict(gate=t["gate"], post_weight=t["post_weight"], post_bias=t["post_bias"], residual_scale=a, kind=kind, eps=eps)
    z, h = daf.residual_norm(t["x"], t["y"], t["weight"], t["bias"], **how)
    x, y, w = t["x"].double(), t["y"].double(), t["weight"].double()
    b = t["bias"].double() if bias else torch.zeros_like(w)
    g = full_gate(t, rows)
    yh, ry, ys = norm64(y, layer, eps) if post else (y, None, y.abs())
    w1 = t["post_weight"].double() if post else torch.ones_like(w)
    b1 = t["post_bias"].double() if t["post_bias"] is not None else torch.zeros_like(w)
    z64 = x + a * g * (yh * w1 + b1)
    zsize = x.abs() + abs(a) * g.abs() * (ys * w1.abs() + b1.abs())
    close(z, z64, zsize, u, "z")
    zh, rz, zs = norm64(z64, layer, eps)
    # h inherits the error of z, times r, and through the row's statistics that of every z of the row
    inherit = (zsize * rz + (zsize * rz).mean(1, keepdim=True) * (1 + zh.abs())) * w.abs()
    close(h, zh * w + b, zs * w.abs() + b.abs() + inherit, u, "h")

    gz = t["gz"] if with_gz else None
    got = daf.residual_norm_grad(z, t["y"], t["weight"], t["bias"], gz, t["gh"], **how)
    zh, rz, zs = norm64(z.double(), layer, eps)                     # the backward pass starts from the stored z
    gh = t["gh"].double()

    def back(hat, r, size, d):
        c = d.mean(1, keepdim=True) if layer else 0.0
        # size * mean(size) pieces: hat enters twice, with its own error
        return (r * (d - c - hat * (d * hat).mean(1, keepdim=True)),
                r * (d.abs() + d.abs().mean(1, keepdim=True) + (size + size.mean(1, keepdim=True)) * (d.abs() * (1 + size)).mean(1, keepdim=True)))
    dn, dn_size = back(zh, rz, zs, gh * w)
    gz64 = gz.double() if gz is not None else torch.zeros_like(gh)
    dx, dx_size = gz64 + dn, gz64.abs() + dn_size
    close(got["x"], dx, dx_size, u, "grad_x")
    close(got["weight"], (gh * zh).sum(0), (gh.abs() * zs).sum(0), pu, "grad_weight")
    if bias:
        close(got["bias"], gh.sum(0), gh.abs().sum(0), pu, "grad_bias")
    yh, ry, ys = norm64(y, layer, eps) if post else (y, None, y.abs())
    du, du_size = a * dx, abs(a) * dx_size
    if gates:
        each, size = du * (yh * w1 + b1), du_size * (ys * w1.abs() + b1.abs())
        close(got["gate"].view(gates, C), each.view(gates, -1, C).sum(1), size.view(gates, -1, C).sum(1), pu, "grad_gate")
    du, du_size = du * g, du_size * g.abs()
    if post:
        close(got["post_weight"], (du * yh).sum(0), (du_size * ys).sum(0), pu, "grad_post_weight")
        if t["post_bias"] is not None:
            close(got["post_bias"], du.sum(0), du_size.sum(0), pu, "grad_post_bias")
        du, _ = back(yh, ry, ys, du * w1)
        _, du_size = back(yh, ry, ys, du_size * w1.abs())
    close(got["y"], du, du_size, u, "grad_y")
    for n, wanted in (("bias", bias), ("gate", gates), ("post_weight", post), ("post_bias", t["post_bias"] is not None)):
        assert (got[n] is not None) == bool(wanted)
    return t, z, h, got, how


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("rows,C,gates,post,bias", [
    (1, 8, 0, False, False), (3, 64, 1, True, True), (7, 72, 0, True, False), (197, 768, 1, False, True), (64, 1000, 4, True, True),
    (12, 136, 12, False, True), (50, 4096, 1, True, True), (9, 4104, 3, True, True), (5, 8192, 0, False, False), (1000, 256, 1000, True, False)])
def test_both_directions(dtype, kind, rows, C, gates, post, bias):
    for pdt in {dtype, torch.float32}:
        run_case(dtype, pdt, rows, C, gates, post, bias, kind)


@pytest.mark.parametrize("dtype", DTYPES)
def test_more_rows_than_ctas_and_groups_that_span_them(dtype):
    run_case(dtype, torch.float32, 4096, 128, 8, True, True, "layer")
    run_case(dtype, torch.float32, 3001, 520, 1, False, True, "rms")
    run_case(dtype, torch.float32, 2000, 40, 500, False, False, "layer", with_gz=False)


def test_rows_far_from_zero_and_constant_rows():
    run_case(torch.float32, torch.float32, 40, 768, 1, True, True, "layer", offset=100.0)
    x = torch.full((4, 64), 3.0, device="cuda")
    w = torch.ones(64, device="cuda")
    z, h = daf.residual_norm(x, torch.zeros_like(x), w, eps=1e-6)
    assert torch.equal(z, x) and (h == 0).all()
    got = daf.residual_norm_grad(z, x, w, None, None, torch.ones_like(x), eps=1e-6)
    assert torch.isfinite(got["x"]).all() and (got["weight"] == 0).all()


def test_in_place_empty_and_repeated():
    t, z, h, got, how = run_case(torch.bfloat16, torch.float32, 300, 768, 4, True, True, "layer", seed=2)
    again = daf.residual_norm_grad(z, t["y"], t["weight"], t["bias"], t["gz"], t["gh"], **how)
    for n in got:                                                    # fixed order of the sums: the same bits
        assert torch.equal(got[n], again[n])
    x, y = t["x"].clone(), t["y"].clone()
    a, b = daf.residual_norm(x, y, t["weight"], t["bias"], out=(x, y), **how)
    assert a is x and b is y and torch.equal(x, z) and torch.equal(y, h)
    e = torch.empty((0, 768), device="cuda", dtype=torch.bfloat16)
    how["gate"] = t["gate"][:1].contiguous()[0]
    assert daf.residual_norm(e, e, t["weight"], t["bias"], **how)[0].numel() == 0
    got = daf.residual_norm_grad(e, e, t["weight"], t["bias"], None, e, **how)
    assert all((got[n] == 0).all() for n in ("weight", "bias", "gate", "post_weight", "post_bias"))


def test_gradient_against_differences():
    """Central differences of f = sum(z gz + h gh) at 1/64 in float32: truncation (1/64)^2 of a third derivative of the order
    of f, rounding 2^-23 * 64 |f|; 2% of the gradient's norm covers both."""
    t, z, h, got, how = run_case(torch.float32, torch.float32, 20, 128, 1, True, True, "layer", seed=4)
    torch.manual_seed(1)
    for name in ("x", "y", "weight", "bias", "gate", "post_weight", "post_bias"):
        d, f = torch.randn_like(t[name]), []
        for sign in (1, -1):
            s = dict(t)
            s[name] = t[name] + sign / 64 * d
            how2 = dict(how, gate=s["gate"], post_weight=s["post_weight"], post_bias=s["post_bias"])
            zz, hh = daf.residual_norm(s["x"], s["y"], s["weight"], s["bias"], **how2)
            f.append((zz.double() * t["gz"].double()).sum() + (hh.double() * t["gh"].double()).sum())
        slope, want = float(f[0] - f[1]) * 32, float((got[name].double() * d.double()).sum())
        assert abs(slope - want) <= 0.02 * float(got[name].double().norm()) + 0.02 * abs(want), (name, slope, want)
