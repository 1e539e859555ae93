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


def test_what_is_written_into_counts_as_modified():
    """autograd tells by the version counter that a tensor it keeps has changed."""
    q, k, v = qkv()
    out, lse = daf.attention(q, k, v)
    made = [torch.empty_like(t) for t in (out, q, k, v)] + [torch.empty_like(lse)]
    versions = [t._version for t in made]
    daf.attention(q, k, v, out=made[0], lse=made[4])
    daf.attention_grad(q, k, v, out, lse, out, grads=made[1:4])
    x, y, w = torch.randn(8, 64, device="cuda"), torch.randn(8, 64, device="cuda"), torch.ones(64, device="cuda")
    z = torch.empty_like(x)
    made, versions = made + [z, y], versions + [z._version, y._version]
    daf.residual_norm(x, y, w, out=(z, y))
    g = [torch.randn(100, device="cuda"), torch.randn(7, device="cuda")]
    made, versions = made + g, versions + [t._version for t in g]
    daf.clip_grad_norm(g, 1.0)
    assert all(t._version > before for t, before in zip(made, versions))
    into, read = [torch.empty_like(t) for t in g], [t._version for t in (x, q, k, v, lse, *g)]
    versions = [t._version for t in into]
    daf.clip_grad_norm(g, 1.0, out=into)
    assert all(t._version > before for t, before in zip(into, versions))
    assert read == [t._version for t in (x, q, k, v, lse, *g)]       # what is only read stays as it was
    a = torch.randn(100, device="cuda", requires_grad=True)
    f = (a * g[0]).sum()
    daf.clip_grad_norm(g, 0.5)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        f.backward()
    with torch.inference_mode():
        h = [torch.randn(100, device="cuda")]
        daf.clip_grad_norm(h, 1.0)
    daf.clip_grad_norm(h, 1.0)                                      # tensors without a counter


def test_running_out_of_memory_is_told_apart():
    """A copy of half a terabyte (a broadcast tensor, which the kernels cannot address) is refused by torch's allocator, by the
    process's own limit."""
    q, k, v = qkv()
    torch.cuda.set_per_process_memory_fraction(0.05)
    try:
        with pytest.raises(torch.cuda.OutOfMemoryError):
            daf.attention(q[:, :1, :1].expand(1, 1 << 23, 512, 64), k[:, :, :1], v[:, :, :1])
    finally:
        torch.cuda.set_per_process_memory_fraction(1.0)
    assert daf.attention(q, k, v)[0].isfinite().all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_join_reads_tensors_off_their_boundary(dtype):
    """Like attention: what the kernels cannot address is copied first, what they write has to be addressable."""
    def off(*shape):
        n = 1
        for s in shape:
            n *= s
        return torch.randn(n + 1, device="cuda").to(dtype)[1:].view(shape)
    x, y, gz, gh = (off(6, 64) for _ in range(4))
    w, b, g, pw, pb = (off(64) for _ in range(5))
    how = dict(gate=g, post_weight=pw, post_bias=pb)
    fit = {n: t.clone() for n, t in how.items()}
    for a, c in zip(daf.residual_norm(x, y, w, b, **how), daf.residual_norm(x.clone(), y.clone(), w.clone(), b.clone(), **fit)):
        assert torch.equal(a, c)
    got = daf.residual_norm_grad(x, y, w, b, gz, gh, **how)
    want = daf.residual_norm_grad(x.clone(), y.clone(), w.clone(), b.clone(), gz.clone(), gh.clone(), **fit)
    assert all(torch.equal(got[n], want[n]) for n in want)
    with pytest.raises(ValueError):
        daf.residual_norm(x, y, w, b, out=(off(6, 64), torch.empty_like(x)))
    half = torch.randn(6 * 64 + 8, device="cuda")[4:-4].view(6, 64)  # on 16 bytes, not on 32
    assert half.data_ptr() % 32 == 16
    for a, c in zip(daf.residual_norm(half, half, torch.ones(64, device="cuda")), daf.residual_norm(half.clone(), half.clone(), torch.ones(64, device="cuda"))):
        assert torch.equal(a, c)


def test_gradients_in_other_orders_are_clipped_in_place():
    """Channels-last and transposed gradients fill their memory without gaps: order does not matter to a norm."""
    from paper_2507_07149_b200 import transformer as tr
    torch.manual_seed(0)
    ps = [torch.nn.Parameter(torch.randn(8, 6, 3, 3, device="cuda").to(memory_format=torch.channels_last)), torch.nn.Parameter(torch.randn(40, 30, device="cuda"))]
    ps[0].grad = torch.randn(8, 6, 3, 3, device="cuda").to(memory_format=torch.channels_last)
    ps[1].grad = torch.randn(30, 40, device="cuda").t()
    keep = [(p.grad, p.grad.data_ptr(), p.grad.stride(), p.grad.clone()) for p in ps]
    norm = tr.clip_grad_norm_(ps, 0.5)
    want = torch.cat([k[3].reshape(-1) for k in keep]).double().norm()
    assert abs(float(norm) - float(want)) <= 2.0 ** -16 * float(want)
    for p, (grad, at, strides, before) in zip(ps, keep):
        assert p.grad is grad and grad.data_ptr() == at and grad.stride() == strides
        assert (grad.double() - before.double() * 0.5 / (want + 1e-6)).abs().max() <= 2.0 ** -16
    out = [torch.empty_like(p.grad) for p in ps]
    daf.clip_grad_norm([k[3] for k in keep], 0.5, out=out)
    assert all(torch.equal(o, p.grad) for o, p in zip(out, ps))
    with pytest.raises(ValueError):                                 # another order
        daf.clip_grad_norm([keep[1][3]], 0.5, out=[torch.empty(40, 30, device="cuda")])
    for gaps in (torch.randn(10, 10, device="cuda")[:, :5], torch.randn(10, 1, device="cuda").expand(10, 4)):
        with pytest.raises(ValueError):
            daf.clip_grad_norm([gaps], 0.5)
    ps[1].grad = None
    ps[1].grad = torch.randn(40, 60, device="cuda")[:, ::2]          # this one has to be copied
    before = ps[1].grad.clone()
    tr.clip_grad_norm_(ps[1:], 0.5)
    assert (ps[1].grad.double() - before.double() * 0.5 / (before.double().norm() + 1e-6)).abs().max() <= 2.0 ** -16


def test_no_gradients_have_a_norm_on_their_device():
    from paper_2507_07149_b200 import transformer as tr
    norm = daf.clip_grad_norm([], 1.0)
    assert norm.is_cuda and norm.dtype == torch.float32 and float(norm) == 0.0
    norm = tr.clip_grad_norm_([torch.nn.Parameter(torch.randn(3, device="cuda"))], 1.0)
    assert norm.is_cuda and float(norm) == 0.0


def test_a_block_under_autocast():
    """The stream stays in float32, the products run in bfloat16: within a few 2^-8 of the block in float32."""
    from paper_2507_07149_b200 import transformer as tr
    torch.manual_seed(0)
    block = tr.Block(128, 2, 256, gate_init=0.5).cuda()
    x, h = torch.randn(2, 30, 128, device="cuda"), torch.randn(2, 30, 128, device="cuda")
    want = block(x, h)
    with torch.autocast("cuda", torch.bfloat16):
        got = block(x, h)
    for a, b in zip(got, want):
        assert a.dtype == torch.float32 and (a - b).norm() <= 2.0 ** -6 * b.norm()
    sum(t.square().sum() for t in got).backward()
    assert all(p.grad is not None and p.grad.isfinite().all() for p in block.parameters())
