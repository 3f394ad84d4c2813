"""swconv_logprobs_forward / _backward against the definition in 64 bits: classes exactly, values by their roundings."""
import numpy as np
import pytest
import torch

from oracle import training as ref
from paper_1702_08597_amd import binding as sw
from training_ops import (TYPES, U, Rows, grad_bound, logprob_bound, logprobs_backward, logprobs_forward, ptr, row_bounds, stream)

pytestmark = pytest.mark.gpu


def scores(rows, classes, seed, scale=2.0):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, classes)).astype(np.float32) * np.float32(scale)
    x[np.arange(rows), rng.integers(0, classes, rows)] += rng.uniform(0, 12, rows).astype(np.float32)
    labels = rng.integers(-1, classes, rows).astype(np.int32)
    return x, labels, rng


def same_or_close(got, want, bound):
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    special = ~np.isfinite(want)
    np.testing.assert_array_equal(got[special], want[special])
    assert (np.abs(got[~special] - want[~special]) <= np.broadcast_to(bound, want.shape)[~special]).all()


def check(name, x, labels, top, stride=0, shift=0, backward=True, seed=0):
    rows, classes = x.shape
    print("logprobs", name, rows, classes, top, stride, shift, flush=True)
    xs = Rows(name, rows, classes, stride, shift, x)
    lab = torch.from_numpy(labels).cuda()
    got = logprobs_forward(name, xs, lab, top)
    x64 = xs.f64()
    lp, H, stats, tc, tl = ref.logprobs_forward(x64, labels, top)
    with np.errstate(invalid="ignore"):
        m, ls_bound, H_bound = row_bounds(x64)
    np.testing.assert_array_equal(got["stats"][:, 0], stats[:, 0].astype(np.float32))
    same_or_close(got["stats"][:, 1], stats[:, 1], ls_bound)
    same_or_close(got["logprob"], lp, logprob_bound(x64, lp))
    same_or_close(got["entropy"], H, H_bound)
    np.testing.assert_array_equal(got["top_class"], tc)
    same_or_close(got["top_logprob"], tl, logprob_bound(x64, tl) if top else 0.0)
    assert xs.guards_hold()
    if backward:
        rng = np.random.default_rng(seed)
        g, h = rng.standard_normal(rows).astype(np.float32), rng.standard_normal(rows).astype(np.float32)
        gd, hd = torch.from_numpy(g).cuda(), torch.from_numpy(h).cuda()
        for use_g, use_h in ((True, True), (True, False), (False, True)):
            dx = Rows(name, rows, classes, stride, shift)
            logprobs_backward(name, xs, lab, got, gd if use_g else None, hd if use_h else None, dx)
            want = ref.logprobs_backward(x64, labels, g if use_g else None, h if use_h else None)
            with np.errstate(invalid="ignore"):
                bound = grad_bound(name, x64, g * use_g, h * use_h, np.nan_to_num(H), np.nan_to_num(stats, neginf=0), want)
            limit = {"f32": 3e38, "f16": 65504, "bf16": 3e38}[name]
            assert (np.abs(want[np.isfinite(want)]) < limit).all()
            same_or_close(dx.view.double().cpu().numpy(), want, bound)
            assert dx.guards_hold()
    return got


@pytest.mark.parametrize("name", list(TYPES))
@pytest.mark.parametrize("rows,classes,top", [
    (1, 1, 1), (1, 2, 0), (3, 1, 64), (5, 7, 3), (4, 8, 8), (2, 63, 64), (2, 64, 64), (3, 65, 64), (7, 511, 5), (6, 512, 2), (4, 513, 33),
    (9, 1000, 5), (2, 2047, 20), (3, 2048, 1), (3, 2049, 7), (2, 4097, 64), (5, 10007, 5), (1, 32768, 5), (2, 50021, 20),
    (1, 150001, 64), (300, 10, 5), (1030, 129, 2), (1100, 2500, 3),
])
def test_sizes(name, rows, classes, top):
    x, labels, _ = scores(rows, classes, rows + classes)
    check(name, x, labels, top)


@pytest.mark.parametrize("name", list(TYPES))
@pytest.mark.parametrize("classes", [10, 1000, 3001])
@pytest.mark.parametrize("pad,shift", [(1, 1), (7, 3), (8, 0), (43, 6)])
def test_strides_and_alignment(name, classes, pad, shift):
    x, labels, _ = scores(5, classes, classes + pad)
    check(name, x, labels, 4, classes + pad, shift)


SHAPES = [(40, 5), (1000, 20), (9000, 64), (70001, 20)]


@pytest.mark.parametrize("name", list(TYPES))
@pytest.mark.parametrize("classes,top", SHAPES)
def test_masked_classes(name, classes, top):
    x, labels, rng = scores(8, classes, classes)
    inf = np.inf
    x[0, :] = -inf                                        # nothing left
    x[1, :] = -inf
    x[1, classes // 2] = -3.0                             # one class left
    labels[1] = classes // 2
    x[2, rng.random(classes) < 0.7] = -inf
    x[3, 3:] = -inf                                       # fewer left than are asked for
    labels[3] = 2
    x[4, :-2] = -inf
    labels[4] = 0                                         # a masked label
    lowest = float(torch.finfo(TYPES[name][1]).min)
    x[5, :] = lowest                                      # the type's lowest value is a score
    x[6, 4:] = lowest
    labels[6] = classes - 1
    x[7, :classes - 1] = lowest
    check(name, x, labels, top)


@pytest.mark.parametrize("name", list(TYPES))
@pytest.mark.parametrize("classes,top", SHAPES)
def test_rows_that_are_not_finite(name, classes, top):
    x, labels, _ = scores(6, classes, classes + 1)
    x[0, 0] = np.nan
    x[1, classes - 1] = np.inf
    x[2, classes // 3] = -np.nan
    x[2, classes // 3 + 1] = np.inf
    x[3, :] = np.nan
    x[4, :] = -np.inf
    x[4, classes // 2] = np.nan
    labels[:5] = 1
    check(name, x, labels, top)


@pytest.mark.parametrize("classes,top", SHAPES)
def test_ties_and_orders(classes, top):
    x = np.zeros((7, classes), np.float32)
    x[1] = np.arange(classes) * 1e-3                      # every score beats those before it
    x[2] = -np.arange(classes) * 1e-3
    x[3, ::2] = -0.0
    x[4] = np.arange(classes) // 7 % 5                    # many of each value
    x[5] = np.where(np.arange(classes) % 3 == 0, -1e30, 1e30)
    x[6, -1] = 1.0
    for name in TYPES:
        y = np.clip(x, -6e4, 6e4) if name == "f16" else x
        got = check(name, y, np.arange(7, dtype=np.int32), top, backward=name == "f32")
        # equal scores: every exponential is 1, sums of whole numbers are exact, the logarithm is off by two steps at most
        assert abs(got["stats"][0, 1] - np.log(classes)) <= 4 * U * np.log(classes)


def test_labels_outside_the_classes():
    x, labels, _ = scores(4, 500, 5)
    labels[:] = [500, 2**31 - 1, -1, -2**31]
    check("f32", x, labels, 3)


@pytest.mark.parametrize("shift", [0.0, 1000.0, -3000.0])
def test_scores_far_from_zero(shift):
    x, labels, _ = scores(3, 777, 6, scale=5.0)
    check("f32", x + np.float32(shift), labels, 5)


@pytest.mark.parametrize("classes", [100, 5000, 40000])
def test_outputs_one_by_one(classes):
    x, labels, _ = scores(3, classes, 7)
    xs, lab = Rows("bf16", 3, classes, values=x), torch.from_numpy(labels).cuda()
    full = logprobs_forward("bf16", xs, lab, 9)
    only = logprobs_forward("bf16", xs, None, 0, entropy=False)
    np.testing.assert_array_equal(only["stats"], full["stats"])
    only = logprobs_forward("bf16", xs, None, 9, entropy=False, stats=False)
    np.testing.assert_array_equal(only["top_class"], full["top_class"])
    np.testing.assert_array_equal(only["top_logprob"], full["top_logprob"])
    only = logprobs_forward("bf16", xs, None, 0, stats=False)
    np.testing.assert_array_equal(only["entropy"], full["entropy"])
    only = logprobs_forward("bf16", xs, lab, 0, entropy=False, stats=False)
    np.testing.assert_array_equal(only["logprob"], full["logprob"])


def test_gradient_in_place_and_no_rows():
    x, labels, _ = scores(5, 3001, 8)
    xs, lab = Rows("f16", 5, 3001, 3010, 1, x), torch.from_numpy(labels).cuda()
    fwd = logprobs_forward("f16", xs, lab, 0)
    g = torch.full((5,), -0.2, device="cuda")
    dx = Rows("f16", 5, 3001, 3010, 1)
    logprobs_backward("f16", xs, lab, fwd, g, None, dx)
    logprobs_backward("f16", xs, lab, fwd, g, None, xs)
    assert torch.equal(xs.view, dx.view) and xs.guards_hold()
    sw.swconv_logprobs_forward(sw.SWCONV_F16, 0, 10, 0, 0, 0, 5, 0, 0, stream(), 0, 0, 0, 0, 0)
    sw.swconv_logprobs_backward(sw.SWCONV_F16, 0, 10, 0, 0, 0, 0, 0, 0, 0, stream(), 0, 0)


def test_equal_calls_give_equal_bits():
    x, labels, _ = scores(3, 90001, 9)
    xs, lab = Rows("bf16", 3, 90001, values=x), torch.from_numpy(labels).cuda()
    a = [logprobs_forward("bf16", xs, lab, 20) for _ in range(3)]
    for b in a[1:]:
        for key in ("logprob", "entropy", "stats", "top_class", "top_logprob"):
            np.testing.assert_array_equal(a[0][key], b[key])


def test_offsets_beyond_32_bits():
    # rows 2^31 + 8 elements apart: the last one begins behind 2^33 bytes
    rows, classes, stride = 3, 5001, (1 << 31) + 8
    x, labels, _ = scores(rows, classes, 10)
    buffer = torch.zeros(2 * stride + classes, dtype=torch.bfloat16, device="cuda")
    view = buffer.as_strided((rows, classes), (stride, 1))
    view.copy_(torch.from_numpy(x))
    xs = Rows.__new__(Rows)
    xs.rows, xs.span, xs.stride, xs.view, xs.ptr = rows, classes, stride, view, buffer.data_ptr()
    lab = torch.from_numpy(labels).cuda()
    got = logprobs_forward("bf16", xs, lab, 5)
    small = Rows("bf16", rows, classes, values=x)
    want = logprobs_forward("bf16", small, lab, 5)
    for key in ("logprob", "entropy", "stats", "top_class", "top_logprob"):
        np.testing.assert_array_equal(got[key], want[key])
    g = torch.full((rows,), -0.5, device="cuda")
    dx = Rows("bf16", rows, classes)
    logprobs_backward("bf16", small, lab, want, g, None, dx)
    logprobs_backward("bf16", xs, lab, got, g, None, xs)
    assert torch.equal(view, dx.view)


def test_more_rows_than_one_launch_has_workgroups_for():
    rows = (1 << 22) + 1030  # four rows a workgroup, 2^20 workgroups
    x = torch.zeros((rows, 2), dtype=torch.float16, device="cuda")
    x[:, 1] = (torch.arange(rows, device="cuda") % 8).half()
    xs = Rows.__new__(Rows)
    xs.rows, xs.span, xs.stride, xs.view, xs.ptr = rows, 2, 2, x, x.data_ptr()
    labels = (torch.arange(rows, device="cuda") % 2).int()
    got = logprobs_forward("f16", xs, labels, 1)
    d = np.arange(rows) % 8
    ls = np.log1p(np.exp(-d.astype(np.float64)))
    assert np.abs(got["stats"][:, 1] - ls).max() <= 64 * U
    np.testing.assert_array_equal(got["top_class"][:, 0], (d > 0).astype(np.int32))
    g = torch.ones(rows, device="cuda")
    dx = torch.empty_like(x)
    out = Rows.__new__(Rows)
    out.rows, out.span, out.stride, out.view, out.ptr = rows, 2, 2, dx, dx.data_ptr()
    logprobs_backward("f16", xs, labels, got, g, None, out)
    p1 = 1 / (1 + np.exp(-d.astype(np.float64)))
    want = np.where(np.arange(rows) % 2 == 1, 1 - p1, -p1)
    assert np.abs(dx[:, 1].double().cpu().numpy() - want).max() <= 2.0 ** -11 + 64 * U


# (rows, classes, top): a wave, four and sixteen waves a row and rows in parts, with several tiles to a segment of the second
# look; rows whose best classes overflow the common list (all scores equal in places)
@pytest.mark.parametrize("name,rows,classes,top", [
    ("f16", 1100, 34001, 8), ("bf16", 1100, 34001, 0), ("bf16", 300, 300007, 20), ("f32", 140, 600001, 64), ("bf16", 100, 2000003, 30),
    ("f16", 3, 9000001, 64), ("bf16", 40000, 300, 64), ("f32", 5000, 4000, 33),
])
def test_large_rows_and_many(name, rows, classes, top):
    dtype = TYPES[name][1]
    gen = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn((rows, classes), generator=gen, device="cuda").mul_(3).to(dtype)
    x[rows // 2, ::2] = 11.0
    x[-1, classes // 2:] = float("-inf")
    labels = torch.randint(0, classes, (rows,), generator=gen, device="cuda").int()
    xs = Rows.__new__(Rows)
    xs.rows, xs.span, xs.stride, xs.view, xs.ptr = rows, classes, classes, x, x.data_ptr()
    got = logprobs_forward(name, xs, labels, top)
    step = max(1, (1 << 27) // classes)
    for r in range(0, rows, step):
        at = slice(r, min(rows, r + step))
        z = x[at].double()
        lp = torch.log_softmax(z, 1)
        e = lambda a: torch.from_numpy(a[at]).cuda().double()
        ls = torch.logsumexp(z - z.amax(1, keepdim=True), 1)
        # additions one behind the other: classes / 64 + 32 at most; the scores lie within 40 of each other, or are masked
        bound = U * (3 * 40 + 4 * (classes / 64 + 32) + 6 + 6 * np.log(classes)) + 2 * U * 60
        assert ((e(got["stats"])[:, 1] - ls).abs() <= bound).all()
        want = lp.gather(1, labels[at].long()[:, None])[:, 0]
        seen = want > -np.inf
        assert torch.equal(e(got["logprob"])[~seen], want[~seen])
        assert ((e(got["logprob"]) - want)[seen].abs() <= bound).all()
        if top:
            value, index = torch.sort(z, dim=1, descending=True, stable=True)
            value, index = value[:, :top], index[:, :top].int()
            index[value == -np.inf] = -1
            assert torch.equal(torch.from_numpy(got["top_class"][at]).cuda(), index)
            wanted = lp.gather(1, index.long().clamp(min=0))
            ok = index >= 0
            assert ((e(got["top_logprob"]) - wanted)[ok].abs() <= bound).all()
        del z, lp
