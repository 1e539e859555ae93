"""How errors that only the device can see reach a caller who has let go of the workspace.  That a wait inside a kernel runs out
is not brought about here; the word that such a kernel writes is written by the test."""
import ctypes

import pytest

import paper_2507_07149_b200 as daf

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def write(value):
    """Puts a value into the device's word, through a tensor that stands on its address."""
    class Word:
        __cuda_array_interface__ = {"shape": (1,), "typestr": "<i4", "data": (daf.daf_device_status_word(), False), "version": 3}
    torch.as_tensor(Word(), device="cuda").fill_(value)


def qkv():
    return [torch.randn(1, 40, 2, 64, device="cuda").bfloat16().requires_grad_() for _ in range(3)]


def test_an_error_is_told_once():
    assert daf.daf_device_status() == daf.OK
    write(daf.ERR_TIMEOUT)
    with pytest.raises(daf.DafError) as e:
        daf.check_device()
    assert e.value.status == daf.ERR_TIMEOUT and daf.daf_device_status() == daf.OK
    assert daf.lib().daf_device_status_word(None) == daf.ERR_INVALID_ARG


def test_calls_without_errors_leave_an_earlier_one_there():
    """Unlike a workspace's status, which every call starts anew."""
    from paper_2507_07149_b200 import transformer as tr
    write(daf.ERR_TIMEOUT)
    q, k, v = qkv()
    out, lse = daf.attention(q.detach(), k.detach(), v.detach(), check=True)
    tr.attention(q, k, v).sum().backward()
    x = torch.randn(1, 40, 2, 64, device="cuda", requires_grad=True)
    tr.attention(x, x, x).sum().backward()
    assert daf.daf_device_status(stream=torch.cuda.Stream()) == daf.ERR_TIMEOUT


def test_the_compression_context_and_the_trainer_ask():
    from paper_2507_07149_b200 import transformer as tr
    from paper_2507_07149_b200.autograd import saved_activation_compression
    ctx = saved_activation_compression(group_size=256, bit_budget=4.0, min_numel=256)
    with ctx:
        out = tr.attention(*qkv())
    ctx.check_status()
    with ctx:
        out = tr.attention(*qkv())
    write(daf.ERR_TIMEOUT)
    with pytest.raises(daf.DafError):
        ctx.check_status()
    out.sum().backward()
    write(daf.ERR_TIMEOUT)
    with pytest.raises(daf.DafError):
        tr.train(1, compressed=False, batch=2, tokens=8)
