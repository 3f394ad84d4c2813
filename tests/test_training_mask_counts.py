"""How layers and passes number their masks: by offset + step, so a network of L dropout layers counts its step up by L."""
import itertools

import numpy as np

from oracle import training as ref

SEED, P = 77, 0.5


def mask(shape, count):
    return ref.dropout_keep(*shape, P, SEED, count)[0]


def test_no_mask_comes_back_when_the_step_counts_all_layers():
    layers, passes, shape = 3, 4, (8, 16, 49)
    counts = [i * layers + layer for i in range(passes) for layer in range(layers)]
    masks = [mask(shape, c) for c in counts]
    n = masks[0].size
    for a, b in itertools.combinations(masks, 2):
        assert abs((a == b).mean() - 0.5) < 5 * np.sqrt(0.25 / n)


def test_equal_sums_agree_on_what_they_have_in_common():
    """A step counted up by 1 gives layer 2 of the next pass the mask of layer 3 of this one, of other sizes too."""
    step = 9
    np.testing.assert_array_equal(mask((8, 16, 49), step + 3), mask((8, 16, 49), (step + 1) + 2))
    large, small = mask((4, 8, 49), 12).reshape(32, 49), mask((3, 8, 25), 12).reshape(24, 25)
    np.testing.assert_array_equal(large[:24, :25], small)
    np.testing.assert_array_equal(mask((40, 100, 1), 12)[:24, :25, 0], small)
