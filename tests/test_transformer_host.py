"""The differentiable layer of the operators without a GPU: elementary torch operations stand in for the kernels, what is tested is
what the layer does around them."""
import pytest

torch = pytest.importorskip("torch")

from paper_2507_07149_b200 import transformer as tr  # noqa: E402


def plain_attention(q, k, v, *, causal=False, scale=None, key_lengths=None):
    s = torch.einsum("bqhd,bkhd->bhqk", q, k) * (q.shape[-1] ** -0.5 if scale is None else scale)
    if key_lengths is not None:
        s = s.masked_fill(torch.arange(k.shape[1]) >= key_lengths[:, None, None, None], float("-inf"))
    p = torch.softmax(s, -1).nan_to_num()
    return torch.einsum("bhqk,bkhd->bqhd", p, v), torch.logsumexp(s, -1)


def plain_attention_grad(q, k, v, out, lse, grad_out, **how):
    x = [t.detach().requires_grad_() for t in (q, k, v)]
    with torch.enable_grad():
        return torch.autograd.grad(plain_attention(*x, **how)[0], x, grad_out)


def plain_join(x, y, weight, bias, *, gate=None, post_weight=None, post_bias=None, residual_scale=1.0, kind="layer", eps=1e-6):
    assert x.dtype == y.dtype
    z = x + residual_scale * (1 if gate is None else gate) * y
    return z, torch.nn.functional.layer_norm(z.float(), z.shape[-1:], weight, bias, eps).to(z.dtype)


def plain_join_grad(z, y, weight, bias, grad_z, grad_h, *, gate=None, **how):
    g = (0 if grad_z is None else grad_z) + grad_h
    return {"x": g, "y": g if gate is None else g * gate, "weight": weight * 0, "bias": None if bias is None else bias * 0,
            "gate": None if gate is None else gate * 0, "post_weight": None, "post_bias": None}


@pytest.fixture(autouse=True)
def kernels(monkeypatch):
    monkeypatch.setattr(tr, "_attention", plain_attention)
    monkeypatch.setattr(tr, "attention_grad", plain_attention_grad)
    monkeypatch.setattr(tr, "_residual_norm", plain_join)
    monkeypatch.setattr(tr, "residual_norm_grad", plain_join_grad)


@pytest.mark.parametrize("operator", ["attention", "join"])
def test_a_second_derivative_is_an_error(operator):
    """The kernels' gradients carry no graph: a penalty on gradients would lose these layers' part without a word."""
    q, k, v = (torch.randn(1, 5, 2, 8, requires_grad=True) for _ in range(3))
    if operator == "attention":
        f = tr.attention(q, k, v).square().sum()
    else:
        f = sum(t.square().sum() for t in tr.residual_norm(q, k, torch.ones(8)))
    g, = torch.autograd.grad(f, q, create_graph=True)
    with pytest.raises(RuntimeError, match="differentia"):
        g.square().sum().backward()


def test_lengths_that_change_between_the_passes_are_an_error():
    q, k, v = (torch.randn(2, 5, 2, 8, requires_grad=True) for _ in range(3))
    lengths = torch.tensor([5, 3], dtype=torch.int32)
    out = tr.attention(q, k, v, key_lengths=lengths)
    out.sum().backward()
    out = tr.attention(q, k, v, key_lengths=lengths)
    lengths[1] = 4                                                  # a buffer that the next batch is read into
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.sum().backward()


@pytest.mark.parametrize("stream,block,wide", [(torch.float32, torch.bfloat16, torch.float32), (torch.bfloat16, torch.float32, torch.float32),
                                               (torch.bfloat16, torch.bfloat16, torch.bfloat16)])
def test_a_block_in_another_type_than_the_stream(stream, block, wide):
    """As under autocast: the sum has the wider type, as torch's own has, and each gradient its tensor's."""
    x, y = torch.randn(3, 8, dtype=stream, requires_grad=True), torch.randn(3, 8, dtype=block, requires_grad=True)
    z, h = tr.residual_norm(x, y, torch.ones(8))
    assert z.dtype == h.dtype == wide and torch.equal(z, x + y)
    (z.sum() + h.sum()).backward()
    assert x.grad.dtype == stream and y.grad.dtype == block


def test_the_classifier_averages_over_the_tokens_that_exist():
    """What lies in the padding changes neither the scores nor any gradient; a sequence of no tokens averages to zero."""
    torch.manual_seed(0)
    net = tr.Classifier(6, 3, 5, width=16, heads=2, blocks=2, hidden=16)
    inputs, lengths = torch.randn(3, 5, 6), torch.tensor([5, 2, 0], dtype=torch.int32)
    other = inputs.clone()
    other[1, 2:], other[2] = 7.0, -3.0
    a, b = net(inputs, lengths), net(other, lengths)
    assert torch.equal(a, b) and torch.equal(a[2], net.head.bias)
    assert torch.allclose(a[0], net(inputs)[0], atol=1e-6)
    short = tr.Classifier(6, 3, 2, width=16, heads=2, blocks=2, hidden=16)
    state = net.state_dict()
    state["place"] = state["place"][:, :2]
    short.load_state_dict(state)
    assert torch.allclose(a[1], short(inputs[1:2, :2])[0], atol=1e-6)
