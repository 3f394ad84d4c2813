"""swconv_dropout_forward / _backward against the definition in 64 bits: masks exactly, values by their roundings."""
import numpy as np
import pytest
import torch

from oracle import training as ref
from paper_1702_08597_amd import binding as sw
from training_ops import (GUARD, TYPES, Rows, dbias_bound, dropout_backward, dropout_bound, dropout_forward, guarded, ptr,
                          rng_state, stream)

pytestmark = pytest.mark.gpu


def inputs(name, N, K, S, seed, stride=0, shift=0):
    rng = np.random.default_rng(seed)
    x = Rows(name, N, K * S, stride, shift, rng.standard_normal((N, K * S)).astype(np.float32))
    dy = Rows(name, N, K * S, stride, shift, (rng.standard_normal((N, K * S)) * 0.1).astype(np.float32))
    bias = torch.from_numpy((rng.standard_normal(K) * 0.3).astype(np.float32)).cuda()
    return x, dy, bias


def check(name, N, K, S, p, relu, with_bias, stride=0, shift=0, seed=1, step=5, offset=3, with_dbias=True):
    print("dropout", name, N, K, S, p, relu, with_bias, stride, shift, flush=True)
    x, dy, bias = inputs(name, N, K, S, 100 * N + K + S, stride, shift)
    b = bias if with_bias else None
    b64 = bias.double().cpu().numpy() if with_bias else None
    rng = rng_state(seed, step)
    y = Rows(name, N, K * S, stride, shift)
    dropout_forward(name, x, N, K, S, b, relu, p, rng, offset, y)
    x64, dy64 = x.f64().reshape(N, K, S), dy.f64().reshape(N, K, S)
    want = ref.dropout_forward(x64, b64, relu, p, seed, step + offset)
    got = y.f64().reshape(N, K, S)
    keep, _ = ref.dropout_keep(N, K, S, p, seed, step + offset)
    assert (got[~keep] == 0).all()
    assert (np.abs(got - want) <= dropout_bound(name, want, 3)).all()   # bias, scale, product
    assert y.guards_hold()
    dx = Rows(name, N, K * S, stride, shift)
    dbias = guarded(K) if with_dbias else None
    dropout_backward(name, dy, x if relu else None, N, K, S, b if relu else None, relu, p, rng, offset, dx, dbias)
    wdx, wdb = ref.dropout_backward(dy64, x64, b64, relu, p, seed, step + offset)
    gdx = dx.f64().reshape(N, K, S)
    assert (np.abs(gdx - wdx) <= dropout_bound(name, wdx, 2)).all()
    assert dx.guards_hold() and x.guards_hold() and dy.guards_hold()
    if with_dbias:
        assert (np.abs(dbias[:K].double().cpu().numpy() - wdb) <= dbias_bound(wdx)).all()
        assert (dbias[K:] == 77).all()
    return got


@pytest.mark.parametrize("name", list(TYPES))
@pytest.mark.parametrize("relu,with_bias", [(0, False), (1, True), (0, True), (1, False)])
@pytest.mark.parametrize("N,K,S", [(2, 3, 169), (5, 16, 1)])
def test_forms(name, relu, with_bias, N, K, S):
    check(name, N, K, S, 0.25, relu, with_bias)
    check(name, N, K, S, 0.25, relu, with_bias, with_dbias=False)


@pytest.mark.parametrize("name", list(TYPES))
@pytest.mark.parametrize("N,K,S", [
    (1, 1, 1), (1, 1, 2), (1, 7, 1), (3, 1, 7), (2, 5, 8), (2, 5, 9), (300, 3, 3), (65, 70, 4), (4, 33, 49), (2, 9, 512),
    (3, 5, 729), (2, 3, 4095), (1, 2, 4096), (2, 2, 4097), (1, 3, 12345), (1, 1, 100003), (17, 24, 64),
    (4, 2048, 1), (9, 2049, 1), (1000, 10, 1), (513, 63, 1), (33, 4096, 1), (3, 5000, 1), (2500, 72, 1), (1, 20011, 1),
])
def test_sizes(name, N, K, S):
    check(name, N, K, S, 0.4, 1, True)


@pytest.mark.parametrize("name", list(TYPES))
@pytest.mark.parametrize("N,K,S,gap,shift", [(3, 4, 25, 100, 0), (3, 4, 25, 1, 1), (5, 33, 1, 7, 3), (4, 40, 1, 8, 5), (2, 3, 64, 5, 7),
                                             (2, 8, 49, 392, 392)])
def test_strides_and_alignment(name, N, K, S, gap, shift):
    for with_dbias in (True, False):
        check(name, N, K, S, 0.3, 1, True, K * S + gap, shift, with_dbias=with_dbias)


@pytest.mark.parametrize("S", [1, 30])
@pytest.mark.parametrize("p", [0.0, 2.0 ** -18, 2.0 ** -16, 0.5, 1 - 2.0 ** -16, 1.0])
def test_rates(S, p):
    check("f32", 4, 50, S, p, 1, True)


def test_the_mask_is_one_of_sizes_and_numbers_alone():
    N, K, S = 3, 10, 37
    got = {}
    for name in TYPES:
        for stride, shift in ((0, 0), (K * S + 3, 5)):
            got[name, stride] = check(name, N, K, S, 0.5, 0, True, stride, shift, seed=2**63 + 9, step=2**64 - 2, offset=7) != 0
    first = got["f32", 0]
    assert all((m == first).all() for m in got.values())
    other = check("f32", N, K, S, 0.5, 0, True, seed=2**63 + 9, step=2**64 - 2, offset=8) != 0
    assert (other != first).any()


def test_rate_zero_reads_no_generator():
    x, _, bias = inputs("f32", 2, 6, 5, 3)
    y = Rows("f32", 2, 30)
    sw.swconv_dropout_forward(sw.SWCONV_F32, 2, 6, 5, x.ptr, 0, ptr(bias), 1, 0.0, 0, 0, stream(), y.ptr, 0)
    z = x.view.view(2, 6, 5) + bias[None, :, None]
    assert torch.equal(y.view.view(2, 6, 5), torch.where(z < 0, torch.zeros_like(z), z))


@pytest.mark.parametrize("S", [1, 12])
def test_dropped_and_kept_values_that_are_not_finite(S):
    N, K, p = 6, 40, 0.5
    x = Rows("f32", N, K * S, values=np.full((N, K * S), np.nan, np.float32))
    dy = Rows("f32", N, K * S, values=np.full((N, K * S), np.inf, np.float32))
    rng = rng_state(4, 0)
    keep, _ = ref.dropout_keep(N, K, S, p, 4, 0)
    keep = keep.reshape(N, K * S)
    y, dx = Rows("f32", N, K * S), Rows("f32", N, K * S)
    dropout_forward("f32", x, N, K, S, None, 1, p, rng, 0, y)
    assert np.isnan(y.f64()[keep]).all() and (y.f64()[~keep] == 0).all()
    dropout_backward("f32", dy, x, N, K, S, None, 1, p, rng, 0, dx, None)  # a NaN is not below zero
    assert np.isposinf(dx.f64()[keep]).all() and (dx.f64()[~keep] == 0).all()


def test_half_precision_overflows_to_infinity_and_rounds_once():
    x = Rows("f16", 1, 4, values=np.array([[60000.0, -60000.0, 1.0, 2.0 ** -24]], np.float32))
    y = Rows("f16", 1, 4)
    dropout_forward("f16", x, 1, 4, 1, torch.tensor([10000.0, -10000.0, 2.0 ** -12, 0.0], device="cuda"), 0, 0.0, None, 0, y)
    assert y.f64().tolist() == [[np.inf, -np.inf, 1.0, 2.0 ** -24]]


@pytest.mark.parametrize("S", [1, 21])
def test_in_place(S):
    N, K = 5, 30
    x, dy, bias = inputs("bf16", N, K, S, 8)
    rng = rng_state(1, 1)
    y, dx = Rows("bf16", N, K * S), Rows("bf16", N, K * S)
    dropout_forward("bf16", x, N, K, S, bias, 1, 0.3, rng, 0, y)
    dbias, again = guarded(K), guarded(K)
    dropout_backward("bf16", dy, x, N, K, S, bias, 1, 0.3, rng, 0, dx, dbias)
    dropout_backward("bf16", dy, x, N, K, S, bias, 1, 0.3, rng, 0, dy, again)      # dx in dy's place
    assert torch.equal(dy.view, dx.view) and torch.equal(dbias, again)
    dropout_forward("bf16", x, N, K, S, bias, 1, 0.3, rng, 0, x)
    assert torch.equal(x.view, y.view)


@pytest.mark.parametrize("S", [1, 49])
def test_groups_of_one_tensor_side_by_side(S):
    # two channel groups of one tensor, the output of the first in the place of the second
    N, K = 4, 16
    x, _, bias = inputs("f32", N, 2 * K, S, 9)
    before = x.view.clone()
    sw.swconv_dropout_forward(sw.SWCONV_F32, N, K, S, x.ptr, 2 * K * S, ptr(bias), 0, 0.0, 0, 0, stream(), x.ptr + 4 * K * S,
                              2 * K * S)
    assert torch.equal(x.view[:, :K * S], before[:, :K * S])
    want = before[:, :K * S].reshape(N, K, S) + bias[:K][None, :, None]
    assert torch.equal(x.view[:, K * S:].reshape(N, K, S), want)


def test_bias_gradient_alone_and_of_no_images():
    N, K, S = 7, 20, 40
    x, dy, bias = inputs("f16", N, K, S, 10)
    rng = rng_state(3, 3)
    a, b = guarded(K), guarded(K)
    dx = Rows("f16", N, K * S)
    dropout_backward("f16", dy, x, N, K, S, bias, 1, 0.3, rng, 0, dx, a)
    dropout_backward("f16", dy, x, N, K, S, bias, 1, 0.3, rng, 0, None, b)
    assert torch.equal(a, b)
    for S in (1, 40):
        b.fill_(77)
        sw.swconv_dropout_backward(sw.SWCONV_F16, 0, K, S, 0, 0, 0, 0, 0, 1, 0.3, 0, 0, 0, 0, stream(), 0, 0, ptr(b))
        assert (b[:K] == 0).all() and (b[K:] == 77).all()
    sw.swconv_dropout_forward(sw.SWCONV_F16, 0, K, S, 0, 0, 0, 1, 0.3, 0, 0, stream(), 0, 0)


def test_equal_calls_give_equal_bits():
    for N, K, S in ((64, 48, 169), (3000, 200, 1)):
        x, dy, bias = inputs("f32", N, K, S, 11)
        rng = rng_state(5, 5)
        out = []
        for _ in range(3):
            dx, db = Rows("f32", N, K * S), guarded(K)
            dropout_backward("f32", dy, x, N, K, S, bias, 1, 0.2, rng, 0, dx, db)
            out.append((dx.view.clone(), db))
        assert all(torch.equal(out[0][0], o[0]) and torch.equal(out[0][1], o[1]) for o in out)


def test_more_rows_and_images_than_one_launch_has_workgroups_for():
    # 2^20 workgroups of 512 groups; the last rows against the definition
    N, K = (1 << 29) + 70, 3
    x = torch.full((N, K), 1.0, dtype=torch.bfloat16, device="cuda")
    y = torch.empty_like(x)
    rng = rng_state(6, 6)
    sw.swconv_dropout_forward(sw.SWCONV_BF16, N, K, 1, x.data_ptr(), 0, 0, 0, 0.5, ptr(rng), 0, stream(), y.data_ptr(), 0)
    rows = np.concatenate([np.arange(50), np.arange(N - 50, N)])
    words = ref.philox4x32_10((np.zeros(100, int), rows, np.full(100, 6), np.zeros(100, int)), (6, 0))
    fields = np.stack([words[0] & np.uint64(0xFFFF), words[0] >> np.uint64(16), words[1] & np.uint64(0xFFFF)], 1)
    got = y[torch.from_numpy(rows).cuda()].float().cpu().numpy()
    np.testing.assert_array_equal(got, np.where(fields >= 32768, 2.0, 0.0))
