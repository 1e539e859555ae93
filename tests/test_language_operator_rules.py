"""Rules of the language operators that hold without a GPU: how memory is read, what host code refuses and asks for."""
import ctypes
import os
import re

import pytest

import paper_2507_07149_b200 as daf
from paper_2507_07149_b200 import build as daf_build

CSRC = os.path.join(os.path.dirname(daf.__file__), "csrc")


def test_lists_that_another_launch_writes_are_not_read_as_constant():
    # embedding_sum_kernel and embedding_join_kernel start while the sort still writes its list: read-only loads are for the caller's tokens
    with open(os.path.join(CSRC, "embedding.cu")) as f:
        loads = re.findall(r"__ldg\(([^;]*?)\s*\+", f.read())
    assert loads and all("a.tokens" in what for what in loads), loads


@pytest.mark.parametrize("count", [0, 1, 31, 33])
def test_another_count_of_frequencies_is_refused_before_the_library_reads_them(count, monkeypatch):
    called = []
    monkeypatch.setattr(daf, "_call", lambda *a: called.append(a) or daf.OK)
    p, f = daf.daf_rotary_params(rotary_dim=64), [1.0] * count
    for call, more in ((daf.daf_rotary_norm, 7), (daf.daf_rotary_norm_grad, 14)):
        with pytest.raises(ValueError):
            call(p, f, *[None] * more)
        assert not called
        call(p, [1.0] * 32, *[None] * more)
        call(p, None, *[None] * more)
        assert len(called) == 2
        called.clear()


def test_as_many_outputs_as_matrices(monkeypatch):
    torch = pytest.importorskip("torch")
    called = []
    monkeypatch.setattr(daf, "_call", lambda *a: called.append(a) or daf.OK)
    two = [torch.zeros(4, 8), torch.zeros(3, 5)]
    for out in (two[:1], [], two + two):
        with pytest.raises(ValueError):
            daf.daf_orthogonalize(daf.daf_orthogonalize_params(), two, out, None, 0)
    assert not called
    daf.daf_orthogonalize(daf.daf_orthogonalize_params(), two, two, None, 0)
    assert len(called) == 1


def test_checked_embedding_refuses_what_the_plain_one_does_and_its_workspace():
    daf_build.build()
    a, lib = 1 << 20, daf.lib()                  # an address that is never used: every call below is refused
    p = daf.daf_embedding_params(ctypes.sizeof(daf.daf_embedding_params), daf.BF16, daf.F32, 8, 10, 100, 64, 1.0, -1, 0)
    need = daf.daf_embedding_workspace(p)
    ref = ctypes.byref(p)
    assert need > 0
    for bad in ((None, a, a, a), (a, None, a, a), (a, a, None, a), (a + 4, a, a, a), (a, a + 2, a, a), (a, a, a + 1, a), (a, a, a, None), (a, a, a, a + 16)):
        assert lib.daf_embedding_checked(ref, *bad, need, None) == daf.ERR_INVALID_ARG
    assert lib.daf_embedding_checked(ref, a, a, a, a, need - 1, None) == daf.ERR_CAPACITY
    assert lib.daf_embedding_checked(None, a, a, a, a, need, None) == daf.ERR_INVALID_ARG
    p.width = 0
    assert lib.daf_embedding_checked(ref, a, a, a, a, need, None) == daf.ERR_SHAPE and daf.daf_embedding_workspace(p) == 0


@pytest.mark.parametrize("shape,count", [((65536, 1), 192), ((65536, 65), 192), ((1, 65536), 192), ((40000, 33), 500), ((2048, 8192), 64)])
def test_a_batch_bounds_the_workspace_of_orthogonalised_updates(shape, count):
    """16 bytes for each of 2^27 elements, or for one matrix if that is larger, whatever the rows are padded to; 64 KiB for the rest."""
    daf_build.build()
    p = daf.daf_orthogonalize_params(ctypes.sizeof(daf.daf_orthogonalize_params), 5, (3.4445, -4.7750, 2.0315), 1e-7)
    for dtype in (daf.F32, daf.F16, daf.BF16):
        sizes = ((ctypes.c_uint32 * count)(*[dtype] * count), (ctypes.c_uint64 * count)(*[shape[0]] * count), (ctypes.c_uint64 * count)(*[shape[1]] * count))
        one = daf.lib().daf_orthogonalize_workspace(ctypes.byref(p), 1, *sizes)
        assert one <= daf.lib().daf_orthogonalize_workspace(ctypes.byref(p), count, *sizes) <= 16 * 2 ** 27 + (1 << 16) + 192 * 512 * 8
