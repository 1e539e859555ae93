"""Orthogonalised updates in 64 bits with the kernels' documented roundings and no others, for bounds on their errors: two float16 parts of
every operand (small times small left out), sums in tensor memory that lose what `added` says and, for segments, added up in binary32;
a matrix of one CTA with binary32 products and sums and its polynomial in 64 bits.  Tensors of any device."""
import torch

A, B, C = (torch.tensor(v, dtype=torch.float32).double().item() for v in (3.4445, -4.7750, 2.0315))
HELD = 4096.0


def exact(g, steps=5, eps=1e-7):
    x = g.double()
    tall = x.shape[0] > x.shape[1]
    x = x.t() if tall else x
    x = x / (x.norm() + eps)
    for _ in range(steps):
        p = x @ x.t()
        x = A * x + (B * p + C * p @ p) @ x
    return x.t() if tall else x


def apart(got, want):
    return ((got.double() - want).norm() / want.norm()).item()


def bias(got, want):
    """The part of the error along the result, in which roundings to nearest cancel and sums that are cut downwards add up."""
    return (((got.double() - want) * want).sum() / want.square().sum()).item()


def binary32(t):
    return t.float().double()


def added(total, a, b):
    """total + a b for 16 products of each sum, as the tensor cores add: all 17 are cut towards zero two bits below the last of the
    largest one's 24, their sum at its 24th.  Seventeen halves of a quarter of a unit are the two units that an addition loses."""
    terms = torch.cat((total[:, None], a[:, :, None] * b[None]), 1)
    unit = torch.exp2((torch.frexp(terms.abs().amax(1))[1] - 26).double())
    total = ((terms / unit[:, None]).trunc_() * unit[:, None]).sum(1)
    m, e = torch.frexp(total)
    return torch.ldexp(torch.trunc(m * 2.0 ** 24), e - 24)


def parts(t, count):
    hi = (t * HELD).half().double()
    lo = (t * HELD - hi).half().double() if count == 2 else torch.zeros_like(hi)
    return hi / HELD, lo / HELD


def product(a, b, segment):
    total = large = torch.zeros((a[0].shape[0], b[0].shape[1]), dtype=torch.float64, device=a[0].device)
    small = a[0] @ b[1] + a[1] @ b[0]                               # 2^-11 of the others: so is what their sum loses
    for k in range(0, a[0].shape[1], 16):
        large = added(large, a[0][:, k:k + 16], b[0][k:k + 16])
        if segment and (k + 16) % segment == 0:
            total, large = binary32(total + large), torch.zeros_like(large)
    return binary32(total + large + small)


def on_tensor_cores(g, *, segment, count=2, steps=5, eps=1e-7):
    """segment: products of a sum that is added up outside of tensor memory, None: all of them.  count: parts of an operand."""
    x = g.double()
    tall = x.shape[0] > x.shape[1]
    x = x.t() if tall else x
    op = parts(x / (x.norm() + eps), count)
    for i in range(steps):
        gram = parts(product(op, [p.t() for p in op], segment), count)
        poly = parts(binary32(B * (gram[0] + gram[1]) + C * product(gram, [p.t() for p in gram], segment)), count)
        x = binary32(A * (op[0] + op[1]) + product(poly, op, segment))
        op = parts(x, count)
    return x.t() if tall else x


def by_one_cta(g, *, exact_poly=True, steps=5, eps=1e-7):
    """Binary32 throughout but for the polynomial and what adds up the Gram matrix's sixteen pieces (the fewest there are of a long side),
    and for the update of up to eight rows."""
    x = g.double()
    tall = x.shape[0] > x.shape[1]
    x = x.t() if tall else x
    x = binary32(x / (x.norm() + eps))
    rows, n = x.shape
    for _ in range(steps):
        pieces = torch.nn.functional.pad(x, (0, -n % 16)).view(rows, -1, 16)
        sums = torch.zeros((16, rows, rows), dtype=torch.float64, device=g.device)
        for k in range(pieces.shape[1]):
            column = pieces[:, k].t()
            sums = binary32(sums + column[:, :, None] * column[:, None, :])
        gram = sums.sum(0)
        poly = B * gram + C * gram @ gram
        if not exact_poly:
            gram = binary32(gram)
            poly = binary32(B * gram + binary32(C * binary32(gram @ gram)))
        if rows > 8 or not exact_poly:
            poly, y = binary32(poly), binary32(A * x)
            for k in range(rows):
                y = binary32(y + poly[:, k:k + 1] * x[k])
            x = y
        else:
            x = binary32(A * x + poly @ x)
    return x.t() if tall else x


def update(shape, seed, kind, device="cpu"):
    """A matrix as updates are: some directions far stronger than the others, or all alike."""
    g = torch.Generator(device=device).manual_seed(seed)
    r, c = shape
    x = torch.randn((r, c), generator=g, device=device)
    if kind == "strong":
        k = max(1, min(r, c) // 4)
        x = 0.1 * x + (torch.randn((r, k), generator=g, device=device) / (1 + torch.arange(k, device=device))) @ torch.randn((k, c), generator=g, device=device)
    return 0.01 * x
