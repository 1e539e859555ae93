"""Token embedding and its gradient against their definitions in 64 bits."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
import paper_2507_07149_b200 as daf  # noqa: E402

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SMALLEST = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -133}


def tokens_of(kind, n, vocabulary, g, dtype=torch.int64):
    if kind == "even":
        t = torch.randint(vocabulary, (n,), generator=g, device="cuda")
    elif kind == "one":                                            # a single word
        t = torch.full((n,), vocabulary - 1, device="cuda")
    elif kind == "few":                                            # runs of all lengths
        t = (torch.rand(n, generator=g, device="cuda") ** 6 * vocabulary).long().clamp_(max=vocabulary - 1)
    else:                                                          # every second place the same word, the others distinct ones
        t = torch.where(torch.arange(n, device="cuda") % 2 == 0, 0, torch.arange(n, device="cuda") % vocabulary)
    return t.to(dtype)


def near(got, want, slack):
    """One rounding to got's type (half a step relative, half the smallest step absolute) of a value that is `slack` off."""
    half = torch.finfo(got.dtype).eps / 2
    bound = slack + half * (want.abs() + slack) + SMALLEST[got.dtype] / 2
    off = (got.double() - want).abs()
    assert (off <= bound).all(), f"off by {off.max().item()}, {(off / bound).max().item()} of the bound"


@pytest.mark.parametrize("table,act", [("f32", "f32"), ("f16", "f16"), ("bf16", "bf16"), ("f32", "bf16"), ("f32", "f16")])
@pytest.mark.parametrize("shape,vocabulary,width", [((1,), 1, 1), ((61,), 100, 8), ((3, 41), 513, 264), ((2, 5, 7), 50, 1031), ((1000,), 3, 2048), ((4099,), 70000, 33)])
def test_forward(table, act, shape, vocabulary, width):
    g = torch.Generator(device="cuda").manual_seed(1)
    t = torch.randint(vocabulary, shape, generator=g, device="cuda", dtype=torch.int64 if len(shape) != 2 else torch.int32)
    w = torch.randn((vocabulary, width), generator=g, device="cuda").to(TYPES[table])
    for scale in (1.0, math.sqrt(width)):
        out = daf.embedding(t, w, scale=scale, dtype=TYPES[act])
        assert out.shape == (*shape, width) and out.dtype == TYPES[act]
        want = w[t.long()].double() * torch.tensor(scale, dtype=torch.float32).double()
        near(out, want, want.abs() * 2.0 ** -24)
        if table == act and scale == 1.0:
            assert torch.equal(out, w[t.long()])
    daf.check_device()


# the sum of n values in binary32 is off by at most n 2^-24 times the sum of their magnitudes, its product with scale by another 2^-24
def check_grad(t, grad, vocabulary, got, scale, padding):
    flat, rows = t.reshape(-1).long(), grad.reshape(-1, grad.shape[-1]).double()
    scale = torch.tensor(scale, dtype=torch.float32).double().item()
    want = torch.zeros((vocabulary, rows.shape[1]), dtype=torch.float64, device="cuda").index_add_(0, flat, rows) * scale
    size = torch.zeros_like(want).index_add_(0, flat, rows.abs()) * abs(scale)
    count = torch.bincount(flat, minlength=vocabulary)[:, None]
    if padding is not None:
        want[padding], size[padding] = 0, 0
    near(got, want, (count + 2) * 2.0 ** -24 * size)
    nobody = (count[:, 0] == 0).nonzero()[:, 0]
    assert not got[nobody].any()


@pytest.mark.parametrize("table,act", [("f32", "f32"), ("f16", "f16"), ("bf16", "bf16"), ("f32", "bf16"), ("f32", "f16")])
@pytest.mark.parametrize("n,vocabulary,width,kind", [
    (1, 1, 1, "even"), (1, 5, 8, "even"), (15, 7, 16, "few"), (16, 2, 24, "one"), (17, 300, 40, "other"), (128, 129, 72, "few"), (1000, 512, 256, "even"),
    (1031, 511, 264, "few"), (4096, 513, 320, "one"), (5003, 40, 1031, "few"), (8193, 9, 33, "other"), (33001, 70001, 64, "few"), (100003, 300000, 8, "even"),
    (70001, 5, 7, "one"), (20000, 262145, 9, "few")])
def test_gradient(table, act, n, vocabulary, width, kind):
    g = torch.Generator(device="cuda").manual_seed(n + width)
    t = tokens_of(kind, n, vocabulary, g, torch.int32 if n % 2 else torch.int64)
    grad = torch.randn((n, width), generator=g, device="cuda").to(TYPES[act])
    padding = None if n % 3 == 0 else int(t[0])
    scale = 1.0 if n % 5 else 0.3
    got = daf.embedding_grad(t, grad, vocabulary, scale=scale, padding=padding, dtype=TYPES[table], check=True)
    assert got.shape == (vocabulary, width) and got.dtype == TYPES[table]
    check_grad(t, grad, vocabulary, got, scale, padding)
    again = daf.embedding_grad(t, grad, vocabulary, scale=scale, padding=padding, dtype=TYPES[table])
    assert torch.equal(got, again)                                 # the same bits


# on both sides of where tokens are looked through (1024 of them, 2048 of no smaller a vocabulary, 2048 pairs of slabs of 256 columns) and sorted
@pytest.mark.parametrize("table,act", [("f32", "f32"), ("bf16", "bf16"), ("f32", "f16")])
@pytest.mark.parametrize("n,vocabulary,width,kind", [
    (2, 70001, 3, "one"), (255, 31, 8, "few"), (256, 400, 264, "other"), (257, 9, 16, "one"), (1023, 2000, 135, "few"), (1024, 5, 256, "even"), (1024, 5000, 520, "few"),
    (1025, 5000, 512, "few"), (1024, 300, 513, "one"), (409, 300, 2056, "few"), (410, 300, 2056, "few"), (600, 3, 1031, "even"),
    (2048, 2048, 33, "few"), (2048, 2047, 40, "one"), (2047, 3000, 500, "one"), (2049, 5000, 24, "other")])
def test_gradient_of_few_tokens(table, act, n, vocabulary, width, kind):
    test_gradient(table, act, n, vocabulary, width, kind)


def test_sorted_tokens_in_their_places():
    # the calls of the tests below with a few tokens, among enough others for them to be sorted
    g = torch.Generator(device="cuda").manual_seed(9)
    grad = torch.full((1500, 8), 2.0 ** -24, device="cuda")
    grad[0] = 1.0
    t = torch.cat((torch.zeros(4, dtype=torch.int64), torch.randint(1, 50, (1496,)))).cuda()
    assert (daf.embedding_grad(t, grad, 50)[0] == 1.0).all()
    order = torch.tensor([3, 2, 1, 0, *range(4, 1500)], device="cuda")
    assert (daf.embedding_grad(t, grad[order], 50)[0] == 1.0 + 2.0 ** -22).all()
    for bad in (-1, 50, 1 << 40):
        where = torch.arange(1500, device="cuda") % 7 == 3
        got = daf.embedding_grad(t.where(~where, bad), grad, 50)
        check_grad(t, grad.where(~where[:, None], 0), 50, got, 1.0, None)
        with pytest.raises(daf.DafError) as e:
            daf.check_device()
        assert e.value.status == daf.ERR_INVALID_ARG
        with pytest.raises(daf.DafError):
            daf.embedding_grad(t.where(~where, bad), grad, 50, check=True)
        daf.daf_device_status()
    for width in (24, 29):
        for dt in (torch.float32, torch.bfloat16):
            for off in (0, 1, 4):
                grad = torch.randn((1500, width), generator=g, device="cuda").to(dt)
                room = torch.full((off + 50 * width + 64,), 7.0, dtype=dt, device="cuda")
                gw = room[off:off + 50 * width].view(50, width)
                daf.embedding_grad(t, grad, 50, out=gw)
                check_grad(t, grad, 50, gw, 1.0, None)
                assert (room[:off] == 7).all() and (room[off + 50 * width:] == 7).all()
        grad = torch.ones((1500, width), device="cuda")
        grad[0, 0], grad[1400, 1] = math.nan, -math.inf
        got, want = daf.embedding_grad(t, grad, 50), torch.bincount(t, minlength=50)[:, None].float().repeat(1, width)
        want[0, 0], want[t[1400], 1] = math.nan, -math.inf
        assert torch.equal(got.nan_to_num(nan=77.0), want.nan_to_num(nan=77.0))
        assert daf.embedding_grad(t, grad, 50, padding=0)[0].eq(0).all()


def test_gradient_of_every_chunk_length_and_border():
    # runs that begin and end everywhere relative to the chunks' borders
    g = torch.Generator(device="cuda").manual_seed(4)
    for n in (40000, 1 << 18):
        t = torch.repeat_interleave(torch.arange(n, device="cuda"), torch.randint(1, 300, (n,), generator=g, device="cuda"))[:n]
        t = t[torch.randperm(n, generator=g, device="cuda")]
        vocabulary = int(t.max()) + 3
        grad = torch.randn((n, 16), generator=g, device="cuda")
        check_grad(t, grad, vocabulary, daf.embedding_grad(t, grad, vocabulary, check=True), 1.0, None)


def test_order_of_the_sum_is_that_of_the_tokens():
    # 1, then 2^-24 three times: each is half a step of 1 and lost (ties go to the even 1).  The other way round their sum, one and a
    # half steps, is exact, and 1 + 1.5 steps ties between one step and two: the even one is two, 2^-22.
    grad = torch.full((4, 8), 2.0 ** -24, device="cuda")
    grad[0] = 1.0
    t = torch.tensor([2, 2, 2, 2], device="cuda")
    assert (daf.embedding_grad(t, grad, 3)[2] == 1.0).all()
    assert (daf.embedding_grad(t, grad.flip(0), 3)[2] == 1.0 + 2.0 ** -22).all()


def test_unknown_tokens_are_zeros_and_reported():
    g = torch.Generator(device="cuda").manual_seed(5)
    w = torch.randn((10, 24), generator=g, device="cuda")
    for bad in (-1, 10, 1 << 40):
        t = torch.tensor([3, bad, 9], device="cuda")
        assert torch.equal(daf.embedding(t, w), torch.stack((w[3], torch.zeros_like(w[3]), w[9])))
        with pytest.raises(daf.DafError) as e:
            daf.check_device()
        assert e.value.status == daf.ERR_INVALID_ARG
        daf.check_device()                                          # asked once
        grad = torch.randn((3, 24), generator=g, device="cuda")
        got = daf.embedding_grad(t, grad, 10)
        want = torch.zeros((10, 24), device="cuda")
        want[3], want[9] = grad[0], grad[2]
        assert torch.equal(got, want)
        with pytest.raises(daf.DafError):
            daf.check_device()
        with pytest.raises(daf.DafError):
            daf.embedding_grad(t, grad, 10, check=True)
        daf.daf_device_status()
        with pytest.raises(daf.DafError):
            daf.embedding(t, w, check=True)


def test_empty_calls():
    w = torch.randn((10, 24), device="cuda")
    none = torch.empty((3, 0), dtype=torch.int64, device="cuda")
    assert daf.embedding(none, w).shape == (3, 0, 24)
    assert not daf.embedding_grad(none, torch.empty((3, 0, 24), device="cuda"), 10, check=True).any()


@pytest.mark.parametrize("width", [24, 29])
def test_layouts_outputs_and_guards(width):
    g = torch.Generator(device="cuda").manual_seed(6)
    for dt in (torch.float32, torch.bfloat16):
        for off in (0, 1, 4):                                       # starts off the boundaries of wide accesses
            base = torch.full((off + 10 * width + 64,), 7.0, dtype=dt, device="cuda")
            w = torch.randn((10, width), generator=g, device="cuda").to(dt)
            base[off:off + 10 * width] = w.reshape(-1)
            t = torch.randint(10, (33,), generator=g, device="cuda")
            table = base[off:off + 10 * width].view(10, width)
            room = torch.full((off + 33 * width + 64,), 7.0, dtype=dt, device="cuda")
            out = room[off:off + 33 * width].view(33, width)
            assert daf.embedding(t, table, out=out) is out and torch.equal(out, w[t])
            assert (room[:off] == 7).all() and (room[off + 33 * width:] == 7).all()
            grad = torch.randn((33, width), generator=g, device="cuda").to(dt)
            room = torch.full((off + 10 * width + 64,), 7.0, dtype=dt, device="cuda")
            gw = room[off:off + 10 * width].view(10, width)
            assert daf.embedding_grad(t, grad, 10, out=gw) is gw
            check_grad(t, grad, 10, gw, 1.0, None)
            assert (room[:off] == 7).all() and (room[off + 10 * width:] == 7).all()
        wide = torch.randn((10, 2 * width), generator=g, device="cuda").to(dt)[:, ::2]              # copied first
        assert torch.equal(daf.embedding(t, wide), wide[t])
        across = torch.randn((width, 33), generator=g, device="cuda").to(dt).t()
        check_grad(t, across, 10, daf.embedding_grad(t, across, 10), 1.0, None)
        one = torch.randn((1, width), generator=g, device="cuda").to(dt).expand(33, width)          # a broadcast gradient
        check_grad(t, one, 10, daf.embedding_grad(t, one, 10), 1.0, None)


def test_values_that_are_not_finite_stay_in_their_rows():
    w = torch.randn((6, 16), device="cuda")
    w[2, 3], w[4, 5] = math.nan, math.inf
    t = torch.tensor([0, 2, 4, 5], device="cuda")
    assert torch.equal(daf.embedding(t, w).nan_to_num(nan=77.0), w[t].nan_to_num(nan=77.0))
    grad = torch.ones((4, 16), device="cuda")
    grad[1, 0], grad[2, 1] = math.nan, -math.inf
    got = daf.embedding_grad(t, grad, 6)
    assert got[2, 0].isnan() and got[4, 1] == -math.inf and got.nan_to_num(nan=0.0, neginf=0.0).sum() == 4 * 16 - 2
    assert daf.embedding_grad(t, grad, 6, padding=2)[2].eq(0).all()  # what the padding's places hold is not looked at


def test_long_table_offsets_pass_32_bits():
    vocabulary, width = 300000, 8192                                # 2.4e9 elements of two bytes
    w = torch.zeros((vocabulary, width), dtype=torch.bfloat16, device="cuda")
    t = torch.tensor([0, vocabulary - 1, 262145], device="cuda")
    w[t] = torch.arange(1, 4, device="cuda", dtype=torch.bfloat16)[:, None]
    assert (daf.embedding(t, w)[:, ::511] == torch.arange(1, 4, device="cuda")[:, None]).all()
    got = daf.embedding_grad(t, w[t].clone(), vocabulary, out=w, check=True)
    assert (got[t] == torch.arange(1, 4, device="cuda")[:, None]).all() and int(got.any(1).sum()) == 3


def test_other_streams_and_graphs():
    g = torch.Generator(device="cuda").manual_seed(7)
    t = torch.randint(1000, (3000,), generator=g, device="cuda")
    grad, w = torch.randn((3000, 64), generator=g, device="cuda"), torch.randn((1000, 64), generator=g, device="cuda")
    want, rows = daf.embedding_grad(t, grad, 1000), daf.embedding(t, w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a, b = daf.embedding_grad(t, grad, 1000, stream=side), daf.embedding(t, w, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(a, want) and torch.equal(b, rows)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a, b = daf.embedding_grad(t, grad, 1000), daf.embedding(t, w)
    t.copy_(t.flip(0))
    graph.replay()
    assert torch.equal(a, daf.embedding_grad(t, grad, 1000)) and torch.equal(b, rows.flip(0))


def test_refusals():
    w, t = torch.randn((10, 24), device="cuda"), torch.tensor([1, 2], device="cuda")
    grad = torch.randn((2, 24), device="cuda")
    for bad in (lambda: daf.embedding(t.float(), w), lambda: daf.embedding(t, w[0]), lambda: daf.embedding(t.cpu(), w), lambda: daf.embedding(t, w.cpu()),
                lambda: daf.embedding(t, w.double()), lambda: daf.embedding(t, w.half(), dtype=torch.float32), lambda: daf.embedding(t, w, dtype=torch.int32),
                lambda: daf.embedding(t, w, out=torch.empty((2, 23), device="cuda")), lambda: daf.embedding_grad(t, grad[:1], 10),
                lambda: daf.embedding_grad(t, grad, 0), lambda: daf.embedding_grad(t, grad, 10, padding=10), lambda: daf.embedding_grad(t, grad, 10, padding=-1),
                lambda: daf.embedding_grad(t, grad, 10, out=torch.empty((9, 24), device="cuda")), lambda: daf.embedding_grad(t, grad, 10, dtype=torch.bfloat16)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(daf.DafError):
        daf.embedding(t, w, scale=math.inf)
