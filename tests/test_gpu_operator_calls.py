"""How the operators' Python functions take what they are given: truth values, layouts, types, errors, version counters."""
import pytest

import paper_2507_07149_b200 as daf

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def qkv():
    return [torch.randn(1, 40, 2, 64, device="cuda").bfloat16() for _ in range(3)]


@pytest.mark.parametrize("check,waits", [(1, True), ([0], True), (True, True), (0, False), (False, False), ([], False)])
def test_check_takes_any_truth_value(check, waits):
    q, k, v = qkv()
    out, lse = daf.attention(q, k, v)
    for fn in (lambda: daf.attention(q, k, v, check=check), lambda: daf.attention_grad(q, k, v, out, lse, out, check=check)):
        torch.cuda.synchronize()
        torch.cuda._sleep(200_000_000)
        done = torch.cuda.Event()
        done.record()
        fn()
        assert done.query() == waits
    with pytest.raises(ValueError):
        daf.attention(q, k, v, check=torch.zeros(2))
    with pytest.raises(ValueError):
        daf.attention(q, k, v, causal=torch.zeros(2))
