"""Rows without a label: log probability 0 and no gradient through it, whatever the scores hold; a row that holds NaN or +inf
shows by its statistics, entropy and best classes."""
import numpy as np
import pytest

from test_gpu_logprobs import check, scores
from training_ops import TYPES

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", list(TYPES))
@pytest.mark.parametrize("classes,top", [(40, 5), (9000, 64), (70001, 20)])
def test_poisoned_rows_without_a_label(name, classes, top):
    x, labels, _ = scores(5, classes, classes + 2)
    x[0, classes - 1] = np.nan
    x[1, classes // 2] = np.inf
    x[2, :] = np.nan
    x[3, :] = -np.inf
    labels[:] = [-1, -7, -2**31, -1, -1]
    got = check(name, x, labels, top)
    assert (got["logprob"] == 0).all()
    for key in ("stats", "entropy", "top_logprob"):
        assert np.isnan(got[key][:3]).all() and not np.isnan(got[key][3:]).any()
    assert (got["top_class"][:4] == -1).all()
