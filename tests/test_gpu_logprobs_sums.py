"""The sums of swconv_logprobs_forward in long rows: bounds that do not grow with the row, rows whose scores are all rounded the
same way, and rows of which every part, wave and tail has to be there.

U is half a step of fp32.  A term exp(x - m) is off by 2 U |x - m| (the exponent's rounding, and that of log2 e) and 2 U (the
instruction) of itself.  All terms are of one sign, so an addition is off by U of the sum at most: 7 in a group of 16 bytes, 3 to
join a tile's groups, 2 in the running sum however many tiles there are, 6 between lanes, 4 between waves, 18 between parts: 40.
The scale of a row and its return from the reference: 4.  Where the largest score changes, in a wave or a join, the sums are scaled:
6 U for each change, and U |x - m| for all of them together."""
import numpy as np
import pytest
import torch

from training_ops import TYPES, U, Rows, half_step, logprobs_backward, logprobs_forward

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
          ("f32", 3, 1000003, 5), ("bf16", 64, 150001, 20), ("bf16", 1, 32768, 5), ("bf16", 2048, 65537, 1), ("f16", 8192, 262143, 1),
          ("f32", 2000, 24571, 3)]


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


@pytest.mark.parametrize("name", list(TYPES))
@pytest.mark.parametrize("rows,classes,top", [(64, 150001, 20), (64, 300007, 0), (40, 1000003, 5), (200, 262147, 3), (300, 262147, 3),
                                              (2048, 65537, 1), (2048, 65537, 0), (64, 40001, 5)])
def test_every_stretch_of_a_row_counts(name, rows, classes, top):
    """Row i holds equal scores in the i-th stretch of its classes alone, the others are masked or far below: ls is the logarithm of
    their number, to the last digits; the last rows have theirs at the very end."""
    x = torch.full((rows, classes), float("-inf"), dtype=TYPES[name][1], device="cuda")
    x[::2] = -1000.0
    ends = [(i * classes // rows, max((i + 1) * classes // rows, i * classes // rows + 1)) for i in range(rows)]
    ends[-3:] = [(classes - 1, classes), (classes - 2, classes), (classes - 9, classes)]
    for i, (a, b) in enumerate(ends):
        x[i, a:b] = 0.5
    got = logprobs_forward(name, rows_of(x), torch.tensor([a for a, _ in ends], device="cuda").int(), top)
    n = np.array([b - a for a, b in ends])
    # counted, not added: the logarithm and nothing else
    for value, want in ((got["stats"][:, 1], np.log(n)), (got["entropy"], np.log(n)), (got["logprob"], -np.log(n))):
        assert (np.abs(value - want) <= 4 * U * np.log(n)).all()
    assert (got["stats"][:, 0] == 0.5).all()
    for i in range(rows):
        left = min(top, n[i])
        np.testing.assert_array_equal(got["top_class"][i, :left], ends[i][0] + np.arange(left))


@pytest.mark.parametrize("name,rows,classes,top", [
    ("f16", 1100, 34001, 8), ("bf16", 2100, 65537, 0), ("bf16", 300, 300007, 20), ("f32", 140, 600001, 64), ("bf16", 100, 2000003, 30),
    ("f16", 3, 9000001, 64), ("f32", 5000, 4000, 33),
])
def test_values_and_gradients_of_large_rows(name, rows, classes, top):
    gen = torch.Generator(device="cuda").manual_seed(classes)
    x = torch.randn((rows, classes), generator=gen, device="cuda").mul_(2).to(TYPES[name][1])
    x[-1, classes // 2:] = float("-inf")
    labels = torch.randint(0, classes // 2, (rows,), generator=gen, device="cuda").int()
    g, h = torch.randn(rows, generator=gen, device="cuda"), torch.randn(rows, generator=gen, device="cuda")
    xs = rows_of(x)
    got = logprobs_forward(name, xs, labels, top)
    dx = torch.full_like(x, 77.0)
    logprobs_backward(name, xs, labels, got, g, h, rows_of(dx))
    rel, tiny = half_step(name)
    step = max(1, (1 << 25) // classes)
    for r in range(0, rows, step):
        at = slice(r, min(rows, r + step))
        z = x[at].double()
        d = z - z.amax(1, keepdim=True)
        ls = torch.logsumexp(d, 1)
        lp = d - ls[:, None]
        p = lp.exp()
        lp0 = torch.where(p > 0, lp, torch.zeros_like(lp))
        mean_d = -(p * torch.where(p > 0, d, torch.zeros_like(d))).sum(1)
        H = ls + mean_d
        # scores drawn independently: the k-th tile changes the largest one with chance 1 / k, so 24 changes and 22 joins
        # are more than there are; the terms that count lie within 30
        ls_bound, H_bound = sum_bounds(ls, mean_d, 30.0, 46)
        e = lambda a: torch.from_numpy(a[at]).cuda().double()
        assert ((e(got["stats"])[:, 1] - ls).abs() <= ls_bound).all()
        assert ((e(got["entropy"]) - H).abs() <= H_bound).all()
        own = lp.gather(1, labels[at].long()[:, None])
        assert ((e(got["logprob"]) - own[:, 0]).abs() <= ls_bound + 2 * U * (2 * own[:, 0].abs() + ls)).all()
        g64, h64 = g[at].double()[:, None], h[at].double()[:, None]
        want = -p * (g64 + h64 * (lp0 + H[:, None]))
        want.scatter_add_(1, labels[at].long()[:, None], g64)
        elp = ls_bound[:, None] + 4 * U * (lp0.abs() + ls[:, None])
        factor = g64.abs() + h64.abs() * (lp0.abs() + H[:, None])
        err = p * factor * (elp + 3 * U * lp0.abs() + 8 * U) + p * h64.abs() * (elp + H_bound[:, None]) + 2 * U * g64.abs()
        assert ((dx[at].double() - want).abs() <= err * 1.01 + want.abs() * rel + 1e-37 + tiny).all()


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
