"""The sums of swconv_logprobs_forward in long rows: bounds that do not grow with the row, and rows whose scores are all rounded
the same way.

U is half a step of fp32.  A term exp(x - m) is off by 2 U |x - m| (the exponent's rounding, and that of log2 e) and 2 U (the
instruction) of itself.  All terms are of one sign, so an addition is off by U of the sum at most: 7 in a group of 16 bytes, 3 to
join a tile's groups, 2 in the running sum however many tiles there are, 6 between lanes, 4 between waves, 18 between parts: 40.
The scale of a row and its return from the reference: 4.  Where the largest score changes, in a wave or a join, the sums are scaled:
6 U for each change, and U |x - m| for all of them together."""
import numpy as np
import pytest
import torch

from training_ops import TYPES, U, Rows, logprobs_forward

pytestmark = pytest.mark.gpu


def rows_of(x):
    xs = Rows.__new__(Rows)
    xs.rows, xs.span, xs.stride, xs.view, xs.ptr = x.shape[0], x.shape[1], x.shape[1], x, x.data_ptr()
    return xs


def sum_bounds(ls, mean_d, reach, changes):
    """mean_d: mean distance below the largest score, weighted by the terms; reach: how far down terms that count lie.
    -> bounds of ls and of the entropy."""
    rel = U * (2 * mean_d + 2 + 40 + 4 + 6 * changes + reach)
    ls_bound = rel + 4 * U * (abs(ls) + 1)
    return ls_bound, ls_bound + mean_d * (2 * rel + 2 * U * reach + 8 * U) + 2 * U * (abs(ls) + mean_d)


# one wave, four and sixteen waves to a row, and rows in parts
SHAPES = [("bf16", 2048, 65536, 1), ("f16", 8192, 262144, 1), ("f32", 4096, 65536, 3), ("bf16", 300, 262144, 5), ("f16", 200, 262144, 0),
          ("f32", 3, 1000003, 5), ("bf16", 64, 150001, 20), ("bf16", 1, 32768, 5)]


@pytest.mark.parametrize("name,rows,classes,top", SHAPES)
def test_one_score_above_many_equal_ones(name, rows, classes, top):
    deltas = [1.5, 5.0, 7.0, 9.0, 0.3125, 12.0]
    delta = np.array([deltas[i % len(deltas)] for i in range(rows)])
    x = torch.zeros((rows, classes), dtype=TYPES[name][1], device="cuda")
    x[:, 0] = torch.from_numpy(delta).cuda().to(x.dtype)
    labels = (torch.arange(rows, device="cuda") % 2).int()
    got = logprobs_forward(name, rows_of(x), labels, top)
    s = (classes - 1) * np.exp(-delta)
    ls, mean_d = np.log1p(s), s * delta / (1 + s)
    ls_bound, H_bound = sum_bounds(ls, mean_d, 0.0, 1)  # the one score is met in the first tile; a join may be behind it
    worst = np.abs(got["stats"][:, 1] - ls) / ls_bound, np.abs(got["entropy"] - (ls + mean_d)) / H_bound
    print(name, rows, classes, top, "share of the bounds", worst[0].max(), worst[1].max(), flush=True)
    assert worst[0].max() <= 1 and worst[1].max() <= 1
    lp = np.where(np.arange(rows) % 2, -delta, 0.0) - ls
    assert (np.abs(got["logprob"] - lp) <= ls_bound + 2 * U * (np.abs(lp) + ls)).all()
    if top:
        np.testing.assert_array_equal(got["top_class"], np.tile(np.arange(top), (rows, 1)))
        assert (np.abs(got["top_logprob"][:, 0] + ls) <= ls_bound + 4 * U * ls).all()


@pytest.mark.parametrize("name,rows,classes,top", [("f32", 4096, 65536, 1), ("f32", 300, 262144, 5), ("f32", 5, 1000003, 5)])
def test_scores_that_rise_all_along_a_row(name, rows, classes, top):
    """Every tile of a wave changes its largest score."""
    step = 2.0 ** -13
    x = (torch.arange(classes, device="cuda", dtype=torch.float64) * step).float().expand(rows, classes).contiguous()
    got = logprobs_forward(name, rows_of(x), torch.zeros(rows, dtype=torch.int32, device="cuda"), top)
    d = np.arange(classes) * step
    e = np.exp(-d)
    ls, mean_d = np.log(e.sum()), (e * d).sum() / e.sum()
    # the sums of tiles d further down have shrunk by exp(-d): changes count by what is left of the sums, 1 / (1 - exp(-tile))
    changes = 1 / (1 - np.exp(-1024 * step)) + 22
    ls_bound, H_bound = sum_bounds(ls, mean_d, mean_d, changes)
    assert (np.abs(got["stats"][:, 1] - ls) <= ls_bound).all()
    assert (np.abs(got["entropy"] - (ls + mean_d)) <= H_bound).all()


def test_more_equal_scores_than_fp32_counts():
    """More than 2^24 equal scores in one wave, an odd number of them in every tile."""
    rows, classes = 257, 5 << 24
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 43 GB")
    x = torch.zeros((rows, classes), dtype=torch.float16, device="cuda")
    x[:, ::2048] = -1.0
    got = logprobs_forward("f16", rows_of(x), None, 0)
    others = classes // 2048
    n, s = classes - others, others * np.exp(-1.0)
    ls, mean_d = np.log(n + s), s / (n + s)
    ls_bound, H_bound = sum_bounds(ls, mean_d, 0.0, 1)
    assert (np.abs(got["stats"][:, 1] - ls) <= ls_bound).all()
    assert (np.abs(got["entropy"] - (ls + mean_d)) <= H_bound).all()
    del x
    torch.cuda.empty_cache()
