"""Pins of the oracle of dropout and log probabilities: the generator against its published vectors and by its
statistics, gradients against differences, the definitions on rows that can be written down."""
import numpy as np
import pytest

from oracle import training as ref


@pytest.mark.parametrize("counter,key,words", [
    ((0, 0, 0, 0), (0, 0), (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
    ((0xffffffff,) * 4, (0xffffffff,) * 2, (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
    ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0),
     (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1)),
])
def test_generator_gives_the_known_words(counter, key, words):
    assert tuple(int(w) for w in ref.philox4x32_10(counter, key)) == words


@pytest.mark.parametrize("shape", [(40, 50, 169), (300, 1000, 1)])
@pytest.mark.parametrize("p", [0.1, 0.5, 0.9])
def test_masks_have_their_rate_and_differ_by_step_and_seed(shape, p):
    keep, scale = ref.dropout_keep(*shape, p, 77, 5)
    n = keep.size
    sigma = np.sqrt(p * (1 - p) / n)
    assert abs(keep.mean() - (1 - p)) < 5 * sigma + 2.0 ** -17
    assert abs(scale * (1 - np.rint(p * 65536) / 65536) - 1) < 1e-15
    for seed, step in ((78, 5), (77, 6), (77, 5 + 2**32), (77 + 2**32, 5)):
        other, _ = ref.dropout_keep(*shape, p, seed, step)
        assert abs((keep == other).mean() - (p * p + (1 - p) ** 2)) < 5 * np.sqrt(0.25 / n)
    # neighbouring columns and rows are independent
    k = keep.reshape(-1, keep.shape[2] if shape[2] > 1 else keep.shape[1]).astype(float) - (1 - p)
    for product in (k[:, 1:] * k[:, :-1], k[1:] * k[:-1]):
        assert abs(product.mean()) < 5 * p * (1 - p) / np.sqrt(product.size)


def test_maps_and_features_number_their_rows_apart():
    maps, _ = ref.dropout_keep(3, 4, 10, 0.5, 9, 0)
    rows, _ = ref.dropout_keep(12, 10, 1, 0.5, 9, 0)
    np.testing.assert_array_equal(maps.reshape(12, 10), rows.reshape(12, 10))


@pytest.mark.parametrize("relu", [0, 1])
def test_dropout_gradient_by_differences(relu):
    rng = np.random.default_rng(3)
    x, b, w = rng.standard_normal((3, 4, 6)), rng.standard_normal(4), rng.standard_normal((3, 4, 6))
    loss = lambda x, b: (w * ref.dropout_forward(x, b, relu, 0.3, 11, 2)).sum()
    dx, db = ref.dropout_backward(w, x, b, relu, 0.3, 11, 2)
    eps = 1e-6
    for _ in range(20):
        i = tuple(rng.integers(0, n) for n in x.shape)
        e = np.zeros_like(x)
        e[i] = eps
        assert abs((loss(x + e, b) - loss(x - e, b)) / (2 * eps) - dx[i]) < 1e-8
    for k in range(4):
        e = np.zeros_like(b)
        e[k] = eps
        assert abs((loss(x, b + e) - loss(x, b - e)) / (2 * eps) - db[k]) < 1e-8


def test_logprobs_gradient_by_differences():
    rng = np.random.default_rng(4)
    x = rng.standard_normal((3, 9)) * 2
    x[1, 4] = -np.inf
    labels, g, h = np.array([2, 0, -1]), rng.standard_normal(3), rng.standard_normal(3)

    def loss(x):
        lp, H, _, _, _ = ref.logprobs_forward(x, labels, 0)
        return (g * lp).sum() + (h * H).sum()

    dx = ref.logprobs_backward(x, labels, g, h)
    assert dx[1, 4] == 0
    np.testing.assert_allclose(dx.sum(1), 0, atol=1e-12)  # a constant added to a row changes nothing
    for i in range(3):
        for j in range(9):
            if x[i, j] > -np.inf:
                e = np.zeros_like(x)
                e[i, j] = 1e-5
                assert abs((loss(x + e) - loss(x - e)) / 2e-5 - dx[i, j]) < 1e-8


def test_logprobs_of_rows_that_can_be_written_down():
    inf, nan = np.inf, np.nan
    x = np.array([[0, 0, 0, 0], [-inf, 5, -inf, 5], [-inf] * 4, [0, nan, 0, 0], [inf, 0, 0, 0], [0.0, -0.0, -1e30, -inf]])
    labels = np.array([3, 0, 1, 2, 1, 7])
    lp, H, stats, tc, tl = ref.logprobs_forward(x, labels, 3)
    ln2 = np.log(2)
    np.testing.assert_allclose(lp, [-2 * ln2, -inf, -inf, nan, nan, nan])
    np.testing.assert_allclose(H, [2 * ln2, ln2, 0, nan, nan, ln2])
    np.testing.assert_allclose(stats, [[0, 2 * ln2], [5, ln2], [-inf, 0], [nan, nan], [nan, nan], [0, ln2]])
    np.testing.assert_array_equal(tc, [[0, 1, 2], [1, 3, -1], [-1] * 3, [-1] * 3, [-1] * 3, [0, 1, 2]])
    np.testing.assert_allclose(tl[1], [-ln2, -ln2, -inf])
