"""Clipping by the global gradient norm against 64 bits.  Bounds: the norm's squares are summed in binary32 within a CTA
(at most a few thousand terms per accumulator, all positive: 2^-24 times their number's square root, far below 2^-16), so
the norm is within 2^-16; a scaled element is within that of its factor plus its type's rounding."""
import math

import pytest

import paper_2507_07149_b200 as daf

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
REL = 2.0 ** -16


def check(grads, out, norm, max_norm, eps=1e-6):
    want = math.sqrt(sum(float(g.double().square().sum()) for g in grads))
    assert abs(float(norm) - want) <= REL * want
    by = min(1.0, max_norm / (want + eps))
    for g, o in zip(grads, out):
        w = g.double() * by
        tiny = 2.0 ** -24 if g.dtype == torch.float16 else 0.0
        assert ((o.double() - w).abs() <= 1.01 * (U[g.dtype] + (REL if by < 1 else 0)) * w.abs() + tiny).all()
        if by == 1.0:
            assert torch.equal(o, g)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("max_norm", [0.0, 0.37, 1e9])
def test_odd_sizes_offsets_and_empty_tensors(dtype, max_norm):
    torch.manual_seed(0)
    flat = torch.randn(300000, device="cuda").to(dtype)
    sizes, at, grads = [1, 7, 0, 16, 31, 16384, 16385, 50001, 3, 129999], 1, []
    for n in sizes:
        grads.append(flat[at:at + n])
        at += n + 1
    outs = [torch.full((n + 9,), 5.0, dtype=dtype, device="cuda") for n in sizes]
    out = [o[i % 8: i % 8 + n] for i, (o, n) in enumerate(zip(outs, sizes))]
    norm = daf.clip_grad_norm(grads, max_norm, out=out)
    check(grads, out, norm, max_norm)
    for i, (o, n) in enumerate(zip(outs, sizes)):                    # nothing beside the outputs is touched
        assert (o[:i % 8] == 5).all() and (o[i % 8 + n:] == 5).all()
    keep = [g.clone() for g in grads]
    whole = flat.clone()
    norm2 = daf.clip_grad_norm(grads, max_norm)
    assert float(norm2) == float(norm) or max_norm == 0.0
    for k, g, o in zip(keep, grads, out):
        assert torch.equal(g, o)
    at = 0
    for n in sizes:                                                  # the gaps between the slices
        assert flat[at] == whole[at]
        at += n + 1


def test_mixed_types_and_more_tensors_than_a_launch_takes():
    torch.manual_seed(1)
    types = [torch.float32, torch.float16, torch.bfloat16]
    grads = [torch.randn(1 + 37 * (i % 29), device="cuda").to(types[i % 3]) for i in range(1300)]
    out = [torch.empty_like(g) for g in grads]
    norm = daf.clip_grad_norm(grads, 2.0, out=out)
    check(grads, out, norm, 2.0)
    assert torch.equal(daf.clip_grad_norm(grads, 2.0, out=out), norm)
    alone = torch.empty((), device="cuda")
    ws = torch.empty(daf.daf_clip_norm_workspace(1300), dtype=torch.uint8, device="cuda")
    daf.daf_clip_norm_batch(grads, None, 1.0, 0.0, alone, ws, ws.numel())
    assert torch.equal(alone, norm)


def test_large_set_and_norms_that_are_not_numbers():
    g = [torch.randn(40_000_003, device="cuda").bfloat16(), torch.randn(5_000_000, device="cuda")]
    out = [torch.empty_like(t) for t in g]
    check(g, out, daf.clip_grad_norm(g, 1.0, out=out), 1.0)
    g = [torch.ones(1000, device="cuda") for _ in range(3)]
    g[1][500] = float("inf")
    assert math.isinf(float(daf.clip_grad_norm(g, 1.0)))
    assert (g[0] == 0).all() and math.isnan(float(g[1][500]))
    g = [torch.full((1000,), float("nan"), device="cuda")]
    assert math.isnan(float(daf.clip_grad_norm(g, 1.0)))
    z = [torch.zeros(5, device="cuda")]
    assert float(daf.clip_grad_norm(z, 1.0)) == 0.0 and (z[0] == 0).all()
    assert float(daf.clip_grad_norm([torch.zeros(0, device="cuda")], 1.0)) == 0.0
    assert float(daf.clip_grad_norm([], 1.0)) == 0.0
