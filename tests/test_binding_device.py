"""The binding hands device addresses to the library: a tensor that lies in host memory is refused before the call."""
import contextlib

import pytest

import paper_2507_07149_b200 as daf

torch = pytest.importorskip("torch")


def test_a_host_tensor_never_reaches_the_library(monkeypatch):
    """What torch's own bookkeeping of streams and devices says to the device number of a host tensor (-1, "the current one")
    is stood in for here, so that the check alone decides."""
    called = []
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch.cuda, "device", lambda index: contextlib.nullcontext())

    class Stream:
        cuda_stream = 0
    for stream in (None, Stream()):
        with pytest.raises(ValueError):
            daf._call(lambda *a: called.append(a) or 0, torch.zeros(8), stream, 1, 2)
    x = torch.zeros(64)
    for fn in (lambda: daf.daf_residual_norm(daf.daf_norm_params(), x, x, x, None, None, None, None, x, x),
               lambda: daf.daf_attention(daf.daf_attention_params(), x, x, x, None, x, x, x, 0),
               lambda: daf.daf_clip_norm_batch([x], [x], 1.0, 0.0, x, x, 0)):
        with pytest.raises(ValueError):
            fn()
    assert not called
