"""The language operators where calls meet: workspaces used again, errors of others, large offsets; and their results within bounds of
their own arithmetic."""
import ctypes
import math
from fractions import Fraction

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


# Frequencies whose fraction of a turn lies above a half, the largest of what is held in 64 bits: they are held within 2^-64 turns, which
# position 2^56 makes 2^-8 turns, far above what binary32 does to the angle.
@pytest.mark.parametrize("sign", [1, -1])
def test_frequencies_are_held_within_2_to_the_minus_64_turns(sign):
    two_pi = Fraction("6.283185307179586476925286766559005768394338798750211641949889")
    f = [6.220240124624253, 6.1985164879813235, 6.1188054798018, 6.262672126026183, 4.0, 3.25, 6.0, 1.0]
    q = torch.zeros((1, 1, 1, 16), device="cuda")
    q[..., :8] = 1.0
    for frequencies in (f, [w - float(two_pi) for w in f]):          # and negative ones, up to a turn
        out, _ = daf.rotary_norm(q, None, positions=sign << 56, frequencies=frequencies, eps=0.0)
        for i, w in enumerate(frequencies):
            turns = Fraction(w) * (sign << 56) / two_pi
            a = float((turns - math.floor(turns)) * two_pi)
            # n = sqrt(2); 2^-64 turns a position, the angle in 24 bits, its cut at 2^-32 turns, the accurate functions and four roundings
            off = math.sqrt(2) * (2 * math.pi * 2.0 ** -8 + math.pi * 2.0 ** -24 + 2.0 ** -28 + 2.0 ** -22 + 4 * 2.0 ** -24)
            assert abs(out[0, 0, 0, i].item() - math.sqrt(2) * math.cos(a)) <= off and abs(out[0, 0, 0, 8 + i].item() - math.sqrt(2) * math.sin(a)) <= off


def test_a_vocabulary_beyond_the_limits_is_refused_as_such():
    t, grad = torch.tensor([1, 2], device="cuda"), torch.ones((2, 8), device="cuda")
    for vocabulary in (2 ** 31 - 1, 1 << 40, (1 << 63) - 1):         # not as a lack of memory for its table
        with pytest.raises(daf.DafError) as e:
            daf.embedding_grad(t, grad, vocabulary)
        assert e.value.status == daf.ERR_UNSUPPORTED
    with pytest.raises(daf.DafError) as e:
        daf.embedding_grad(t, grad[:, :0], 10)
    assert e.value.status == daf.ERR_SHAPE


@pytest.mark.parametrize("width", [8192, 8191])
def test_a_sorted_gradient_of_a_table_beyond_32_bits(width):
    """Rows of a table of more than 2^32 bytes and 2^31 elements, from the sums, the joined runs and both ways of clearing."""
    g = torch.Generator(device="cuda").manual_seed(3)
    vocabulary, n = 300000, 3000                                    # 4.9e9 bytes; more tokens than are looked through
    t = torch.randint(vocabulary, (n,), generator=g, device="cuda")
    t[::6] = vocabulary - 7                                         # runs across chunks, one beyond every border
    t[1::12] = 3
    t[2:2 + 9 * 13:9] = torch.tensor([0, vocabulary - 1, 262143, 262144, 262145, 131071, 131072, 2170, 2171, 2172, 2173, 2174, 290000], device="cuda")
    grad = torch.randint(-1, 2, (n, width), generator=g, device="cuda").bfloat16()      # sums are exact, and rounded once
    words, at = torch.unique(t, return_inverse=True)
    want = torch.zeros((words.numel(), width), device="cuda").index_add_(0, at, grad.float()).bfloat16()
    out = torch.full((vocabulary, width), 7.0, dtype=torch.bfloat16, device="cuda")
    daf.embedding_grad(t, grad, vocabulary, out=out, check=True)
    assert torch.equal(out[words], want)
    out[words] = 0
    for lo in range(0, vocabulary, 50000):
        assert not out[lo:lo + 50000].any()


# A weight's gradient is a sum over all rows in pieces: a group of lanes' own rows (of 296 CTAs of eight groups or more, eight heads at a time),
# the groups of a CTA (256 at most), the CTAs (32 at a time), each piece in order.  Every addition of a chain of that length loses 2^-24 of
# the magnitudes, and a term its own roundings.  The terms have one sign, so that a CTA's part that is lost is missed.
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("b,s,h,kv,d", [(64, 40, 12, 12, 64), (1, 2000, 24, 8, 32), (4, 1024, 16, 4, 128), (3, 700, 5, 3, 40)])
def test_weight_gradients_are_sums_of_all_rows(dtype, b, s, h, kv, d):
    g = torch.Generator(device="cuda").manual_seed(4)
    q, k = (torch.randn((b, s, n, d), generator=g, device="cuda").to(dtype) for n in (h, kv))
    gq, gk = ((x.sign() * torch.rand(x.shape, generator=g, device="cuda")).to(dtype) for x in (q, k))
    w = torch.ones(d, device="cuda")
    got = daf.rotary_norm_grad(q, k, w, w, gq, gk, rotary_dim=0)
    for x, gx, made in ((q, gq, got[2]), (k, gk, got[3])):
        x = x.double()
        terms = gx.double() * x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)
        want, rows = terms.sum((0, 1, 2)), b * s * x.shape[2]
        chain = rows / (296 * 8) + 8 + min(256, rows) + 10 + 32
        assert ((made.double() - want).abs() <= (chain + d / 2 + 12) * 2.0 ** -24 * terms.abs().sum((0, 1, 2))).all()
        lost = terms.flatten(0, 2)[:max(1, rows // 296)].sum(0)       # what one CTA of them all adds
        assert (lost > 4 * (chain + d / 2 + 12) * 2.0 ** -24 * want).all()
