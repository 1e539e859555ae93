"""Host checks of the language operators' entry points: what they refuse, and with which status.  Nothing is launched."""
import ctypes
import math

import pytest

import paper_2507_07149_b200 as daf
from paper_2507_07149_b200 import build as daf_build

INV, SHAPE, UNS, CAP = daf.ERR_INVALID_ARG, daf.ERR_SHAPE, daf.ERR_UNSUPPORTED, daf.ERR_CAPACITY
A = 1 << 20                                      # an aligned address that is never used: every call below is refused


@pytest.fixture(scope="module", autouse=True)
def built():
    daf_build.build()


def changed(p, kw):
    for k, v in kw.items():
        if isinstance(v, tuple):
            getattr(p, k)[:] = v
        else:
            setattr(p, k, v)
    return p


def embedding_params(**kw):
    return changed(daf.daf_embedding_params(ctypes.sizeof(daf.daf_embedding_params), daf.BF16, daf.F32, 8, 10, 100, 64, 1.0, -1, 0), kw)


def rotary_params(**kw):
    p = daf.daf_rotary_params(ctypes.sizeof(daf.daf_rotary_params), daf.BF16, daf.F32, 0, 2, 5, 4, 2, 64, 64, 4, 0, 0, 10000.0, 1e-6)
    for n in ("q", "k", "q_out", "k_out", "grad_q", "grad_k"):
        h = 2 if n.endswith("k") or n.startswith("k") else 4
        getattr(p, n + "_stride")[:] = (5 * h * 64, h * 64, 64)
    return changed(p, kw)


def orthogonalize_params(**kw):
    return changed(daf.daf_orthogonalize_params(ctypes.sizeof(daf.daf_orthogonalize_params), 5, (3.4445, -4.7750, 2.0315), 1e-7), kw)


@pytest.mark.parametrize("change,status", [
    (dict(struct_size=8), INV), (dict(dtype=3), INV), (dict(table_dtype=3), INV), (dict(table_dtype=daf.F16), INV), (dict(token_bytes=2), INV),
    (dict(scale=math.inf), INV), (dict(scale=math.nan), INV), (dict(reserved=1), INV), (dict(vocabulary=0), SHAPE), (dict(width=0), SHAPE),
    (dict(vocabulary=2 ** 31 - 1), UNS), (dict(tokens=2 ** 31), UNS), (dict(width=2 ** 24 + 1), UNS), (dict(padding=100), INV)])
def test_embedding_parameters(change, status):
    p = ctypes.byref(embedding_params(**change))
    assert daf.lib().daf_embedding(p, A, A, A, None) == status
    assert daf.lib().daf_embedding_grad(p, A, A, A, A, 1 << 40, None) == status
    assert daf.lib().daf_embedding_grad_workspace(p) == 0


def test_embedding_pointers_and_workspace():
    p = embedding_params()
    need = daf.daf_embedding_grad_workspace(p)
    assert need >= 256 + 4 * 10 * 4
    ref = ctypes.byref(p)
    for bad in ((None, A, A), (A, None, A), (A, A, None), (A + 4, A, A), (A, A + 2, A), (A, A, A + 1)):
        assert daf.lib().daf_embedding(ref, *bad, None) == INV
    for bad in ((None, A, A, A), (A, None, A, A), (A, A, None, A), (A, A, A, None), (A + 4, A, A, A), (A, A + 1, A, A), (A, A, A + 2, A), (A, A, A, A + 16)):
        assert daf.lib().daf_embedding_grad(ref, *bad, need, None) == INV
    assert daf.lib().daf_embedding_grad(ref, A, A, A, A, need - 1, None) == CAP
    assert daf.lib().daf_embedding(None, A, A, A, None) == INV and daf.lib().daf_embedding_grad(None, A, A, A, A, need, None) == INV
    assert daf.lib().daf_embedding(ctypes.byref(embedding_params(tokens=0)), None, None, None, None) == daf.OK


def rotary(p, f=None, *, q=A, k=A, wq=A, wk=A, at=A, qo=A, ko=A):
    return daf.lib().daf_rotary_norm(ctypes.byref(p), f, q, k, wq, wk, at, qo, ko, None)


def rotary_grad(p, f=None, *, q=A, k=A, wq=A, wk=A, at=A, gqo=A, gko=A, gq=A, gk=A, gwq=A, gwk=A, ws=A, n=1 << 40):
    return daf.lib().daf_rotary_norm_grad(ctypes.byref(p), f, q, k, wq, wk, at, gqo, gko, gq, gk, gwq, gwk, ws, n, None)


@pytest.mark.parametrize("change,status", [
    (dict(struct_size=8), INV), (dict(dtype=3), INV), (dict(param_dtype=daf.F16), INV), (dict(style=2), INV), (dict(position_bytes=2), INV),
    (dict(shared_positions=2), INV), (dict(base=0.0), INV), (dict(base=math.inf), INV), (dict(eps=-1.0), INV), (dict(eps=math.nan), INV),
    (dict(reserved=(0, 0, 1)), INV), (dict(head_dim=60), SHAPE), (dict(head_dim=0), SHAPE), (dict(rotary_dim=20), SHAPE), (dict(rotary_dim=72), SHAPE),
    (dict(heads=0), SHAPE), (dict(head_dim=264, rotary_dim=64), UNS), (dict(tokens=2 ** 24 + 1), UNS), (dict(heads=65536), UNS),
    (dict(batch=2 ** 20, tokens=2 ** 10), UNS),
    (dict(batch=2 ** 31, tokens=2 ** 24, heads=512), UNS), (dict(batch=2 ** 31, tokens=2 ** 24, kv_heads=512), UNS)])
def test_rotary_parameters(change, status):
    p = rotary_params(**change)
    assert rotary(p) == status and rotary_grad(p) == status
    if "base" not in change:                     # the workspace does not depend on it
        assert daf.lib().daf_rotary_norm_grad_workspace(ctypes.byref(p)) == 0


@pytest.mark.parametrize("change", [dict(q_stride=(1280, 256, 60)), dict(k_stride=(640, 0, 64)), dict(q_out_stride=(1280, 252, 64)), dict(k_out_stride=(1 << 40, 128, 64))])
def test_rotary_strides(change):
    assert rotary(rotary_params(**change)) == INV and rotary_grad(rotary_params(**change)) == INV


def test_rotary_pointers_frequencies_and_workspace():
    p = rotary_params()
    need = daf.daf_rotary_norm_grad_workspace(p)
    assert need > 0
    for name in ("q", "k", "qo", "ko", "at"):
        assert rotary(p, **{name: None}) == INV
    for name in ("q", "k", "qo", "ko", "wq", "wk"):
        assert rotary(p, **{name: A + 8}) == INV
    assert rotary(p, at=A + 2) == INV
    for name in ("q", "k", "gqo", "gko", "gq", "gk", "ws", "at"):
        assert rotary_grad(p, **{name: None}) == INV
    for name in ("gq", "gk", "gwq", "gwk", "ws"):
        assert rotary_grad(p, **{name: A + 8}) == INV
    assert rotary_grad(p, wq=None) == INV and rotary_grad(p, wk=None) == INV        # a gradient of no weight
    assert rotary_grad(p, n=need - 1) == CAP
    bad = (ctypes.c_double * 32)(*[math.nan] * 32)
    assert rotary(p, bad) == INV and rotary_grad(p, bad) == INV
    assert rotary(rotary_params(batch=0), q=None, k=None, qo=None, ko=None) == daf.OK


def matrices(shapes, types=None):
    n = len(shapes)
    return ((ctypes.c_uint32 * n)(*(types or [daf.BF16] * n)), (ctypes.c_uint64 * n)(*[s[0] for s in shapes]), (ctypes.c_uint64 * n)(*[s[1] for s in shapes]))


def orthogonalize(p, m, src=None, dst=None, ws=A, n=1 << 50):
    count = len(m[0])
    a = (ctypes.c_void_p * count)(*(src or [A] * count))
    b = (ctypes.c_void_p * count)(*(dst or [A] * count))
    return daf.lib().daf_orthogonalize(ctypes.byref(p), count, m[0], a, b, m[1], m[2], ws, n, None)


@pytest.mark.parametrize("change,status", [
    (dict(struct_size=8), INV), (dict(steps=0), INV), (dict(steps=65), UNS), (dict(eps=0.0), INV), (dict(eps=math.inf), INV), (dict(eps=math.nan), INV),
    (dict(coefficients=(1.0, math.nan, 0.0)), INV), (dict(reserved=(0, 1)), INV)])
def test_orthogonalize_parameters(change, status):
    p, m = orthogonalize_params(**change), matrices([(4, 8)])
    assert orthogonalize(p, m) == status
    assert daf.lib().daf_orthogonalize_workspace(ctypes.byref(p), 1, *m) == 0


def test_orthogonalize_pointers_and_workspace():
    p = orthogonalize_params()
    m = matrices([(4, 8), (100, 3), (0, 7)], [daf.BF16, daf.F32, daf.F16])
    need = daf.lib().daf_orthogonalize_workspace(ctypes.byref(p), 3, *m)
    assert need > 256
    assert orthogonalize(p, m, n=need - 1) == CAP
    assert orthogonalize(p, m, src=[A, None, A]) == INV and orthogonalize(p, m, dst=[None, A, A]) == INV
    assert orthogonalize(p, m, src=[A + 1, A, A]) == INV and orthogonalize(p, m, dst=[A, A + 2, A]) == INV
    assert orthogonalize(p, m, ws=None) == INV and orthogonalize(p, m, ws=A + 128) == INV
    assert orthogonalize(p, matrices([(4, 8)], [3])) == INV and orthogonalize(p, matrices([(1, 65537)])) == UNS
    # a set of one shape needs as much however it is ordered, and the largest batch decides: at most 2^27 elements, or one matrix
    one = daf.lib().daf_orthogonalize_workspace(ctypes.byref(p), 1, *matrices([(2048, 8192)]))
    assert one >= 2 * 2 * 2 * 2048 * 8192
    many = daf.lib().daf_orthogonalize_workspace(ctypes.byref(p), 64, *matrices([(2048, 8192)] * 64))
    assert many <= 8 * one + 4096 * 64


def test_refusals_of_the_python_layer():
    torch = pytest.importorskip("torch")
    from paper_2507_07149_b200 import transformer as tr
    with pytest.raises(ValueError):
        daf.rotary_norm(torch.zeros(1, 1, 1, 8), None, style="thirds")
    with pytest.raises(ValueError):
        daf.rotary_norm_grad(torch.zeros(1, 1, 1, 8), None, None, None, torch.zeros(1, 1, 1, 8), None, style="thirds")
    for call in (lambda: daf.embedding(torch.zeros(3, dtype=torch.long), torch.zeros(4, 8)),         # tensors in host memory
                 lambda: daf.embedding_grad(torch.zeros(3, dtype=torch.long), torch.zeros(3, 8), 4), lambda: daf.rotary_norm(torch.zeros(1, 1, 1, 8), None),
                 lambda: daf.orthogonalize([torch.zeros(4, 8)])):
        with pytest.raises(ValueError):
            call()
    assert daf.orthogonalize([]) == []
    with pytest.raises(ValueError):
        tr.Muon([torch.nn.Parameter(torch.zeros(4))])
    with pytest.raises(ValueError):
        tr.Muon([torch.nn.Parameter(torch.zeros(4, 4))], momentum=1.0)
    with pytest.raises(ValueError):
        tr.embedding(torch.zeros(3, dtype=torch.long), torch.zeros(4, 8, requires_grad=True), padding=4)
