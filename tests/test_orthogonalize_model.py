"""The roundings that bound the kernels' errors (orthogonalize_model.py): what the bounds must not let pass lies above them."""
import pytest

torch = pytest.importorskip("torch")
from orthogonalize_model import apart, bias, by_one_cta, exact, on_tensor_cores, update  # noqa: E402


@pytest.mark.parametrize("kind", ["strong", "flat"])
@pytest.mark.parametrize("shape", [(60, 4000), (4000, 48)])
def test_losing_segments_or_a_part_shows(shape, kind):
    g = update(shape, 1, kind)
    want = exact(g)
    bound = 2 * apart(on_tensor_cores(g, segment=128), want) + 2.0 ** -24
    assert apart(on_tensor_cores(g, segment=None), want) > 1.1 * bound
    assert apart(on_tensor_cores(g, segment=128, count=1), want) > 100 * bound


def test_sums_that_are_cut_downwards_show_along_the_result():
    # float16 results: their own rounding hides the loss in the size of the error, but not in its part along the result
    g = update((24, 12000), 2, "flat")
    want = exact(g)
    rounding = 6 * 2.0 ** -11 / want.numel() ** 0.5                 # six deviations of what roundings of all elements leave
    assert abs(bias(want.half(), want)) < rounding
    assert abs(bias(on_tensor_cores(g, segment=128), want)) < rounding
    assert abs(bias(on_tensor_cores(g, segment=None), want)) > 2 * rounding


@pytest.mark.parametrize("shape", [(1, 4096), (4, 4103), (1031, 5)])
def test_a_polynomial_in_32_bits_shows_for_few_rows(shape):
    # one such rounding sequence may be lucky: the mean of eight orders of the columns
    g = update(shape, 3, "flat")
    g = g.t() if shape[0] > shape[1] else g
    want, errors = exact(g), [0.0, 0.0]
    for seed in range(8):
        order = torch.randperm(g.shape[1], generator=torch.Generator().manual_seed(seed))
        for i in (0, 1):
            errors[i] += apart(by_one_cta(g[:, order], exact_poly=i == 0), want[:, order])
    assert errors[1] > 2 * errors[0]
