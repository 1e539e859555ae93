"""Orthogonalised updates within what their documented roundings leave (orthogonalize_model.py), close enough that sums without segments,
operands in one part or a polynomial in 32 bits do not pass."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
import paper_2507_07149_b200 as daf  # noqa: E402
from orthogonalize_model import apart, bias, by_one_cta, exact, on_tensor_cores, update  # noqa: E402

SIZE = pytest.mark.parametrize("kind", ["strong", "flat"])


def name(shape):
    return "x".join(map(str, shape))


# The kernel's roundings are others of the same sizes as the model's: twice its error, and the result's own half step.
@SIZE
@pytest.mark.parametrize("shape", [(33, 33), (63, 65), (77, 77), (128, 256), (129, 127), (200, 1000), (333, 1285), (384, 1111), (512, 130), (640, 2100), (1000, 512),
                                   (64, 8192), (8192, 64), (33, 20000), (4, 4105)], ids=name)
def test_binary32(shape, kind):
    g = update(shape, 3, kind, "cuda")
    got, = daf.orthogonalize([g], check=True)
    want = exact(g)
    assert apart(got, want) <= 2 * apart(on_tensor_cores(g, segment=128), want) + 2.0 ** -24


# Few rows: one sequence of roundings may be lucky, so the largest error of eight orders of the columns.
@SIZE
@pytest.mark.parametrize("shape", [(1, 4096), (1, 1033), (4103, 1), (4, 4103), (5, 517), (12, 1300), (1300, 12), (512, 16), (32, 129), (32, 510), (513, 32)], ids=name)
def test_binary32_by_one_cta(shape, kind):
    g = update(shape, 4, kind, "cuda")
    got, = daf.orthogonalize([g], check=True)
    want, wide = exact(g), g if shape[0] <= shape[1] else g.t()
    turned = want if shape[0] <= shape[1] else want.t()
    errors = []
    for seed in range(8):
        order = torch.randperm(wide.shape[1], generator=torch.Generator().manual_seed(seed)).cuda()
        errors.append(apart(by_one_cta(wide[:, order]), turned[:, order]))
    assert apart(got, want) <= 2 * max(errors) + 2.0 ** -24


# float16 on both sides of where it takes segments.  Its results' rounding, 2^-12 or so of the result's size, is all that is to be seen of the
# error; along the result roundings cancel (deviation 2^-11 over the root of the elements at most), and what is cut off sums does not.
@SIZE
@pytest.mark.parametrize("shape,segment", [((64, 8192), None), ((64, 8200), 128), ((8192, 48), None), ((8193, 48), 128), ((40, 40000), 128)], ids=str)
def test_half_precision(shape, segment, kind):
    g = update(shape, 5, kind, "cuda").half()
    got, = daf.orthogonalize([g], check=True)
    want = exact(g)
    model = on_tensor_cores(g, segment=segment)
    assert apart(got, want) <= 1.05 * apart(want.half(), want) + 2 * apart(model, want)
    assert abs(bias(got, want)) <= 2 * apart(model, want) + 6 * 2.0 ** -11 / want.numel() ** 0.5


# bfloat16 of few columns takes two parts; its long sums have no segments, and lose less than the result's rounding
@pytest.mark.parametrize("shape", [(65536, 2), (20, 30000)], ids=name)
def test_long_bfloat16(shape):
    g = update(shape, 6, "flat", "cuda").bfloat16()
    got, = daf.orthogonalize([g], check=True)
    want = exact(g)
    assert apart(got, want) <= 1.05 * apart(want.bfloat16(), want) + 2 * apart(on_tensor_cores(g, segment=None), want)
