"""Dropout and log probabilities at drawn shapes, types, strides, alignments and options, against the definition in 64 bits;
and calls that the fixed sizes of the other tests do not make."""
import numpy as np
import pytest
import torch

from oracle import training as ref
from paper_1702_08597_amd import binding as sw
from test_gpu_dropout import check as check_dropout
from test_gpu_logprobs import check as check_logprobs
from test_gpu_logprobs import scores
from training_ops import (TYPES, Rows, dbias_bound, dropout_backward, dropout_bound, dropout_forward, guarded, logprobs_backward,
                          logprobs_forward, ptr, rng_state, stream)

pytestmark = pytest.mark.gpu


def log_int(rng, lo, hi):
    return int(round(np.exp(rng.uniform(np.log(lo), np.log(hi)))))


@pytest.mark.parametrize("seed", range(40))
def test_dropout_drawn(seed):
    rng = np.random.default_rng(seed)
    S = 1 if rng.random() < 0.4 else log_int(rng, 2, 3000)
    K = log_int(rng, 1, 3000 if S == 1 else 60)
    N = log_int(rng, 1, max(1, 200000 // (K * S)))
    gap = int(rng.choice([0, 0, 1, 5, 8, 64]))
    check_dropout(str(rng.choice(list(TYPES))), N, K, S, float(rng.choice([0.0, 0.1, 0.5, 0.93])), int(rng.integers(2)),
                  bool(rng.integers(2)), K * S + gap, int(rng.choice([0, 0, 1, 2, 3, 7, 8])), seed=int(rng.integers(1 << 62)),
                  step=int(rng.integers(1 << 62)), offset=int(rng.integers(100)), with_dbias=bool(rng.integers(2)))


@pytest.mark.parametrize("seed", range(40))
def test_logprobs_drawn(seed):
    rng = np.random.default_rng(seed)
    classes = log_int(rng, 1, 60000)
    rows = log_int(rng, 1, max(1, 200000 // classes))
    x, labels, _ = scores(rows, classes, seed, scale=float(rng.choice([0.1, 2.0, 8.0])))
    if rng.random() < 0.4:
        x[rng.random(x.shape) < rng.choice([0.01, 0.5, 0.99])] = -np.inf
    x = x + np.float32(rng.choice([0.0, -40.0, 100.0]))
    pad, shift = int(rng.choice([0, 0, 1, 3, 8])), int(rng.choice([0, 0, 1, 5]))
    check_logprobs(str(rng.choice(list(TYPES))), x, labels, int(rng.choice([0, 1, 5, 9, 20, 64])), classes + pad, shift, seed=seed)


@pytest.mark.parametrize("name", list(TYPES))
@pytest.mark.parametrize("rows,classes,top", [(2, 131075, 20), (7, 100003, 5), (33, 70001, 64)])
def test_rows_in_parts_at_any_alignment(name, rows, classes, top):
    assert sw.swconv_logprobs_workspace_bytes(TYPES[name][0], rows, classes, top) > 0
    x, labels, rng = scores(rows, classes, classes)
    x[0, rng.random(classes) < 0.5] = -np.inf
    x[rows - 1, :] = np.float32(1.5)                      # every class of a part is as good as another
    check_logprobs(name, x, labels, top, classes + 5, 3)


def test_parts_in_a_captured_graph():
    rows, classes, top = 12, 100003, 20
    nbytes = sw.swconv_logprobs_workspace_bytes(sw.SWCONV_BF16, rows, classes, top)
    assert nbytes > 0
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((rows, classes), generator=gen, device="cuda").to(torch.bfloat16)
    lab = torch.randint(0, classes, (rows,), generator=gen, device="cuda").int()

    def buffers():
        return [torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda"), torch.zeros((rows, 2), device="cuda"),
                torch.zeros((rows, top), dtype=torch.int32, device="cuda"), torch.zeros((rows, top), device="cuda"),
                torch.zeros(nbytes, dtype=torch.uint8, device="cuda")]

    def call(b):
        sw.swconv_logprobs_forward(sw.SWCONV_BF16, rows, classes, ptr(x), 0, ptr(lab), top, ptr(b[5]), nbytes, stream(), ptr(b[0]),
                                   ptr(b[1]), ptr(b[2]), ptr(b[3]), ptr(b[4]))

    g, e = buffers(), buffers()
    call(g)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(g)
        call(g)                                           # twice over one workspace, one behind the other
    for _ in range(3):
        x.copy_(torch.randn((rows, classes), generator=gen, device="cuda"))
        for t in g:
            t.fill_(9)
        graph.replay()
        call(e)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(g[:5], e[:5]))


def test_gradient_of_more_rows_than_one_launch_has_in_a_column():
    rows, classes = 70001, 1101
    x = torch.zeros((rows, classes), dtype=torch.bfloat16, device="cuda")
    x[:, 3] = (torch.arange(rows, device="cuda") % 5).to(torch.bfloat16)
    xs = Rows.__new__(Rows)
    xs.rows, xs.span, xs.stride, xs.view, xs.ptr = rows, classes, classes, x, x.data_ptr()
    labels = (torch.arange(rows, device="cuda") % 3 - 1).int()
    fwd = logprobs_forward("bf16", xs, labels, 0)
    g = torch.ones(rows, device="cuda")
    dx = torch.empty_like(x)
    out = Rows.__new__(Rows)
    out.rows, out.span, out.stride, out.view, out.ptr = rows, classes, classes, dx, dx.data_ptr()
    logprobs_backward("bf16", xs, labels, fwd, g, None, out)
    d = np.arange(rows) % 5
    total = 1100 + np.exp(d.astype(np.float64))
    label = np.arange(rows) % 3 - 1
    has = (label >= 0).astype(np.float64)
    want = {0: (label == 0) - has / total, 1: (label == 1) - has / total, 3: -has * np.exp(d) / total, 1100: -has / total}
    for j, w in want.items():
        got = dx[:, j].double().cpu().numpy()
        # p is off by less than 1e-5 of itself, then one rounding
        assert (np.abs(got - w) <= np.abs(w) * (2.0 ** -8 + 1e-5) + 1e-40).all()


@pytest.mark.parametrize("S", [1, 50])
def test_bias_gradient_alone_without_relu(S):
    N, K, p = 9, 33, 0.4
    rng = np.random.default_rng(2)
    dy = Rows("f32", N, K * S, values=rng.standard_normal((N, K * S)).astype(np.float32))
    state = rng_state(7, 7)
    db = guarded(K)
    dropout_backward("f32", dy, None, N, K, S, None, 0, p, state, 0, None, db)
    _, want = ref.dropout_backward(dy.f64().reshape(N, K, S), None, None, 0, p, 7, 7)
    terms = np.abs(ref.dropout_backward(dy.f64().reshape(N, K, S), None, None, 0, p, 7, 7)[0]).sum((0, 2))
    assert (np.abs(db[:K].double().cpu().numpy() - want) <= (N * S + 2) * 2.0 ** -24 * terms * 1.001).all()


def test_small_values_are_kept():
    x = Rows("f32", 1, 4, values=np.array([[2.0 ** -149, -2.0 ** -140, 2.0 ** -127, 0.0]], np.float32))
    y = Rows("f32", 1, 4)
    dropout_forward("f32", x, 1, 4, 1, None, 0, 0.0, None, 0, y)
    assert torch.equal(y.view, x.view)


@pytest.mark.parametrize("name", list(TYPES))
@pytest.mark.parametrize("K", [7, 9, 10, 11, 12, 13, 14, 15, 257, 260, 263])
def test_bias_of_ragged_rows(name, K):
    """The bias lies between NaN and off 16 bytes; every count of columns behind the last whole chunk."""
    N, p, relu = 37, 0.2, 1
    rng = np.random.default_rng(K)
    around = torch.full((K + 18,), float("nan"), device="cuda")
    b = around[9:9 + K]
    b.copy_(torch.from_numpy(rng.standard_normal(K).astype(np.float32)))
    b64 = b.double().cpu().numpy()
    x = Rows(name, N, K, values=rng.standard_normal((N, K)).astype(np.float32))
    dy = Rows(name, N, K, values=rng.standard_normal((N, K)).astype(np.float32))
    y, dx, dx2, db = Rows(name, N, K), Rows(name, N, K), Rows(name, N, K), guarded(K)
    state = rng_state(11, 2)
    dropout_forward(name, x, N, K, 1, b, relu, p, state, 4, y)
    dropout_backward(name, dy, x, N, K, 1, b, relu, p, state, 4, dx, db)
    dropout_backward(name, dy, x, N, K, 1, b, relu, p, state, 4, dx2, None)
    x64, dy64 = x.f64().reshape(N, K, 1), dy.f64().reshape(N, K, 1)
    want = ref.dropout_forward(x64, b64, relu, p, 11, 6)
    assert (np.abs(y.f64().reshape(N, K, 1) - want) <= dropout_bound(name, want, 3)).all()
    wdx, wdb = ref.dropout_backward(dy64, x64, b64, relu, p, 11, 6)
    for got in (dx, dx2):
        assert (np.abs(got.f64().reshape(N, K, 1) - wdx) <= dropout_bound(name, wdx, 2)).all()
        assert got.guards_hold()
    assert (np.abs(db[:K].double().cpu().numpy() - wdb) <= dbias_bound(wdx)).all()
    assert y.guards_hold()
