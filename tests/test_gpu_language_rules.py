"""The language operators where calls meet: workspaces used again, errors of others, large offsets; and their results within bounds of
their own arithmetic."""
import ctypes

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
import paper_2507_07149_b200 as daf  # noqa: E402


@pytest.mark.parametrize("width", [32, 33])
def test_a_workspace_that_one_call_after_another_uses(width):
    """The list of one call lies where the next one's does: thirty calls without a break, each of its own tokens."""
    g = torch.Generator(device="cuda").manual_seed(1)
    n, vocabulary = 6000, 900
    p = daf.daf_embedding_params(ctypes.sizeof(daf.daf_embedding_params), daf.F32, daf.F32, 8, n, vocabulary, width, 1.0, -1, 0)
    size = daf.daf_embedding_grad_workspace(p)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    grad = torch.randint(-8, 9, (n, width), generator=g, device="cuda").float()        # whole numbers: sums are exact
    calls = [(torch.rand(n, generator=g, device="cuda") ** (1 + i % 5) * vocabulary).long().clamp_(max=vocabulary - 1) for i in range(30)]
    made = torch.full((30, vocabulary, width), 7.0, device="cuda")
    for t, out in zip(calls, made):
        daf.daf_embedding_grad(p, t, grad, out, ws, size)
    for t, out in zip(calls, made):
        assert torch.equal(out, torch.zeros((vocabulary, width), device="cuda").index_add_(0, t, grad))
    assert daf.daf_poll_status(ws) == daf.OK


def test_a_checked_embedding_asks_for_its_own_tokens():
    """The device's word holds what others have recorded: it neither fails a call of known tokens nor is it cleared by one."""
    w = torch.randn((10, 24), device="cuda")
    good, bad = torch.tensor([3, 9], device="cuda"), torch.tensor([3, 10], device="cuda")
    daf.daf_device_status()
    for t in (good, good[:0]):
        daf.embedding(bad, w)                                       # somebody else's error, not asked for yet
        assert torch.equal(daf.embedding(t, w, check=True), w[t])
        with pytest.raises(daf.DafError):
            daf.check_device()
    for out in (None, torch.empty((2, 24), device="cuda")):
        with pytest.raises(daf.DafError) as e:
            daf.embedding(bad, w, out=out, check=True)
        assert e.value.status == daf.ERR_INVALID_ARG
    assert torch.equal(out, torch.stack((w[3], torch.zeros_like(w[3]))))
    daf.check_device()                                              # who asked was told
    p = daf.daf_embedding_params(ctypes.sizeof(daf.daf_embedding_params), daf.F32, daf.F32, 8, 2, 10, 24, 1.0, -1, 0)
    size = daf.daf_embedding_workspace(p)
    ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
    for t, status in ((good, daf.OK), (bad, daf.ERR_INVALID_ARG), (good, daf.OK)):
        daf.daf_embedding_checked(p, t, w, out, ws, size)
        assert daf.daf_poll_status(ws) == status
    daf.check_device()


def test_thin_matrices_of_several_batches_are_those_of_one():
    g = torch.Generator(device="cuda").manual_seed(2)
    gs = [torch.randn((60000, 1 + i % 3), generator=g, device="cuda").to((torch.float32, torch.bfloat16)[i % 2]) for i in range(90)]
    made = daf.orthogonalize(gs, check=True)
    for i in (0, 1, 33, 34, 35, 70, 89):
        assert torch.equal(made[i], daf.orthogonalize([gs[i]])[0])
