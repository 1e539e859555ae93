"""Host checks of the transformer operators' entry points: what they refuse, and with which status.  Nothing is launched."""
import ctypes

import pytest

import paper_2507_07149_b200 as daf
from paper_2507_07149_b200 import build as daf_build


@pytest.fixture(scope="module", autouse=True)
def built():
    daf_build.build()


def attention_params(**kw):
    p = daf.daf_attention_params(ctypes.sizeof(daf.daf_attention_params), daf.BF16, 2, 5, 7, 4, 2, 64, 0, 0.125)
    for n in ("q", "k", "v", "out", "grad_out", "grad_q", "grad_k", "grad_v"):
        h = 2 if n in ("k", "v", "grad_k", "grad_v") else 4
        getattr(p, n + "_stride")[:] = ((7 if h == 2 else 5) * h * 64, h * 64, 64)
    for k, v in kw.items():
        if isinstance(v, tuple):
            getattr(p, k)[:] = v
        else:
            setattr(p, k, v)
    return p


def norm_params(**kw):
    p = daf.daf_norm_params(ctypes.sizeof(daf.daf_norm_params), daf.BF16, daf.F32, daf.NORM_LAYER, 12, 64, 0, 1.0, 1e-6, 0)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


A = 1 << 20                                      # an aligned address that is never used: every call below is refused


@pytest.mark.parametrize("change,status", [
    (dict(struct_size=8), daf.ERR_INVALID_ARG), (dict(dtype=3), daf.ERR_INVALID_ARG), (dict(causal=2), daf.ERR_INVALID_ARG),
    (dict(scale=float("inf")), daf.ERR_INVALID_ARG), (dict(scale=float("nan")), daf.ERR_INVALID_ARG), (dict(reserved=(0, 1)), daf.ERR_INVALID_ARG),
    (dict(kv_heads=3), daf.ERR_SHAPE), (dict(heads=0), daf.ERR_SHAPE), (dict(kv_heads=0), daf.ERR_SHAPE), (dict(head_dim=60), daf.ERR_SHAPE),
    (dict(head_dim=0), daf.ERR_SHAPE), (dict(head_dim=136), daf.ERR_UNSUPPORTED), (dict(batch=1 << 15), daf.ERR_UNSUPPORTED),
    (dict(queries=(1 << 24) + 1), daf.ERR_UNSUPPORTED), (dict(keys=(1 << 24) + 1), daf.ERR_UNSUPPORTED),
    (dict(batch=16000, queries=1 << 24), daf.ERR_UNSUPPORTED),
    (dict(q_stride=(1280, 256, 60)), daf.ERR_INVALID_ARG), (dict(k_stride=(896, 0, 64)), daf.ERR_INVALID_ARG),
    (dict(v_stride=(896, 132, 64)), daf.ERR_INVALID_ARG), (dict(out_stride=(1 << 40, 256, 64)), daf.ERR_INVALID_ARG)])
def test_attention_parameters(change, status):
    p = ctypes.byref(attention_params(**change))
    assert daf.lib().daf_attention(p, A, A, A, None, A, A, A, 1 << 30, None) == status
    assert daf.lib().daf_attention_grad(p, A, A, A, None, A, A, A, A, A, A, A, 1 << 30, None) == status
    if not any(k.endswith("stride") for k in change):
        assert daf.lib().daf_attention_grad_workspace(p) == 0 and daf.lib().daf_attention_workspace(p) == 0


def test_attention_pointers_and_workspace():
    p = attention_params()
    ref = ctypes.byref(p)
    need = daf.daf_attention_grad_workspace(p)
    assert need >= 2 * 2 * 4 * 128 * 4
    ok = [A, A, A, None, A, A, A]
    for i, bad in ((0, None), (1, None), (2, A + 8), (3, A + 2), (4, None), (4, A + 4), (5, None), (5, A + 2), (6, None), (6, A + 8)):
        args = list(ok)
        args[i] = bad
        assert daf.lib().daf_attention(ref, *args, 1 << 20, None) == daf.ERR_INVALID_ARG, i
    assert daf.lib().daf_attention(ref, *ok, daf.daf_attention_workspace(p) - 1, None) == daf.ERR_CAPACITY
    ok = [A, A, A, None, A, A, A, A, A, A, A]
    for i, bad in ((0, A + 2), (4, None), (5, None), (6, None), (7, A + 8), (8, None), (9, None), (10, None), (10, A + 4)):
        args = list(ok)
        args[i] = bad
        assert daf.lib().daf_attention_grad(ref, *args, need, None) == daf.ERR_INVALID_ARG, i
    assert daf.lib().daf_attention_grad(ref, *ok, need - 1, None) == daf.ERR_CAPACITY
    for n in ("grad_out_stride", "grad_q_stride", "grad_k_stride", "grad_v_stride"):
        assert daf.lib().daf_attention_grad(ctypes.byref(attention_params(**{n: (896, 130, 64)})), *ok, need, None) == daf.ERR_INVALID_ARG
    # nothing to do is no error, whatever the pointers
    assert daf.lib().daf_attention(ctypes.byref(attention_params(batch=0)), None, None, None, None, None, None, None, 0, None) == daf.OK
    assert daf.lib().daf_attention(ctypes.byref(attention_params(queries=0)), None, None, None, None, None, None, None, 0, None) == daf.OK


@pytest.mark.parametrize("change,status", [
    (dict(struct_size=4), daf.ERR_INVALID_ARG), (dict(dtype=5), daf.ERR_INVALID_ARG), (dict(param_dtype=daf.F16), daf.ERR_INVALID_ARG),
    (dict(kind=2), daf.ERR_INVALID_ARG), (dict(eps=-1.0), daf.ERR_INVALID_ARG), (dict(reserved=1), daf.ERR_INVALID_ARG),
    (dict(width=0), daf.ERR_SHAPE), (dict(width=60), daf.ERR_SHAPE), (dict(width=8200), daf.ERR_UNSUPPORTED)])
def test_norm_parameters(change, status):
    p = ctypes.byref(norm_params(**change))
    assert daf.lib().daf_residual_norm(p, A, A, A, None, None, None, None, A, A, None) == status
    assert daf.lib().daf_residual_norm_grad(p, A, A, A, None, None, None, None, A, A, A, A, None, None, None, None, A, 1 << 30, None) == status
    assert daf.lib().daf_residual_norm_grad_workspace(p) == 0


def test_norm_pointers_and_workspace():
    p = norm_params()
    ref, need = ctypes.byref(p), daf.daf_residual_norm_grad_workspace(p)
    fwd = [A, A, A, None, None, None, None, A, A]
    for i, bad in ((0, None), (1, A + 8), (2, None), (2, A + 4), (3, A + 4), (4, A), (6, A), (7, None), (8, A + 2)):
        args = list(fwd)
        args[i] = bad
        assert daf.lib().daf_residual_norm(ref, *args, None) == daf.ERR_INVALID_ARG, i
    assert daf.lib().daf_residual_norm(ctypes.byref(norm_params(gates=1)), *fwd, None) == daf.ERR_INVALID_ARG          # gates without a gate
    assert daf.lib().daf_residual_norm(ctypes.byref(norm_params(gates=5)), A, A, A, None, A, None, None, A, A, None) == daf.ERR_SHAPE
    bwd = [A, A, A, None, None, None, A, A, A, A, A, None, None, None, None, A]
    for i, bad in ((0, None), (2, None), (6, A + 8), (7, None), (8, None), (9, A + 4), (12, A), (13, A), (15, None), (15, A + 8)):
        args = list(bwd)
        args[i] = bad
        assert daf.lib().daf_residual_norm_grad(ref, *args, need, None) == daf.ERR_INVALID_ARG, i
    assert daf.lib().daf_residual_norm_grad(ref, *bwd, need - 1, None) == daf.ERR_CAPACITY
    # binary32 rows take 32-byte accesses
    f = ctypes.byref(norm_params(dtype=daf.F32))
    assert daf.lib().daf_residual_norm(f, A + 16, A, A, None, None, None, None, A, A, None) == daf.ERR_INVALID_ARG
    assert daf.lib().daf_residual_norm(ctypes.byref(norm_params(rows=0)), None, None, A, None, None, None, None, None, None, None) == daf.OK


def test_clip_arguments():
    need = daf.daf_clip_norm_workspace(2)

    def call(dt=(0, 0), src=(A, A), dst=(A, A), numel=(5, 5), max_norm=1.0, eps=0.0, norm=A, ws=A, size=need):
        n = len(dt)
        arr = (ctypes.c_void_p * n)
        return daf.lib().daf_clip_norm_batch(n, (ctypes.c_uint32 * n)(*dt), arr(*src), None if dst is None else arr(*dst),
                                             (ctypes.c_uint64 * n)(*numel), max_norm, eps, norm, ws, size, None)
    for kw in (dict(dt=(0, 3)), dict(src=(A, None)), dict(src=(A, A + 2)), dict(dt=(2, 2), src=(A, A + 1)), dict(dst=(None, A)), dict(max_norm=-1.0),
               dict(max_norm=float("nan")), dict(eps=-1.0), dict(norm=None), dict(norm=A + 2), dict(ws=None), dict(ws=A + 8)):
        assert call(**kw) == daf.ERR_INVALID_ARG, kw
    assert call(size=need - 1) == daf.ERR_CAPACITY
    assert daf.lib().daf_clip_norm_batch(1, None, None, None, None, 1.0, 0.0, A, A, need, None) == daf.ERR_INVALID_ARG


def test_python_layer_refuses_what_it_cannot_marshal():
    torch = pytest.importorskip("torch")
    x = torch.zeros(2, 3, 4, 64)
    for fn in (lambda: daf.attention(x, x, x), lambda: daf.attention_grad(x, x, x, x, x, x), lambda: daf.residual_norm(x, x, x[0, 0, 0]),
               lambda: daf.clip_grad_norm([x], 1.0)):
        with pytest.raises(ValueError):                             # CPU tensors
            fn()
