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
