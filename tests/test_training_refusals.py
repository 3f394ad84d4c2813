"""What swconv_dropout_* and swconv_logprobs_* refuse, before anything is launched: no GPU needed."""
import pytest

from paper_1702_08597_amd import binding as sw

P = 1 << 40  # an address that is never read: every call here is refused
EINVAL, EUNSUPPORTED = sw.SWCONV_EINVAL, sw.SWCONV_EUNSUPPORTED


def status(fn, args):
    with pytest.raises(sw.SwconvError) as e:
        fn(*args)
    return e.value.status


def forward(**change):
    a = dict(dtype=0, N=2, K=3, S=4, x=P, xs=0, bias=P, relu=1, p=0.5, rng=P, offset=0, stream=0, y=P + 4096, ys=0)
    a.update(change)
    return list(a.values())


def backward(**change):
    a = dict(dtype=0, N=2, K=3, S=4, dy=P, dys=0, x=P + 4096, xs=0, bias=P, relu=1, p=0.5, rng=P, offset=0, ws=P, nbytes=1 << 20,
             stream=0, dx=P + 8192, dxs=0, dbias=P)
    a.update(change)
    return list(a.values())


SIZES = [
    (dict(dtype=3), EINVAL), (dict(dtype=-1), EINVAL), (dict(N=-1), EINVAL), (dict(K=0), EINVAL), (dict(S=0), EINVAL),
    (dict(N=2**31), EUNSUPPORTED), (dict(K=2**31), EUNSUPPORTED), (dict(S=2**31), EUNSUPPORTED),
    (dict(N=2**20, K=2**12), EUNSUPPORTED), (dict(K=2**30, S=2**30), EUNSUPPORTED),
    (dict(xs=11), EINVAL), (dict(xs=-12), EINVAL), (dict(xs=2**41), EUNSUPPORTED), (dict(N=2**20, xs=2**21), EUNSUPPORTED),
    (dict(p=-0.01), EINVAL), (dict(p=1.01), EINVAL), (dict(p=float("nan")), EINVAL), (dict(rng=0), EINVAL), (dict(rng=P + 4), EINVAL),
    (dict(x=0), EINVAL), (dict(x=P + 2), EINVAL), (dict(bias=P + 2), EINVAL),
]


@pytest.mark.parametrize("change,want", SIZES + [
    (dict(ys=11), EINVAL), (dict(y=0), EINVAL), (dict(y=P + 1), EINVAL),
    (dict(y=P + 4), EINVAL), (dict(y=P + 4 * 23), EINVAL), (dict(y=P - 4), EINVAL),      # overlaps in another way
    (dict(y=P, ys=13), EINVAL), (dict(y=P + 4 * 12, xs=20, ys=20), EINVAL),
    (dict(dtype=1, y=P + 1), EINVAL),
])
def test_dropout_forward(change, want):
    assert status(sw.swconv_dropout_forward, forward(**change)) == want


@pytest.mark.parametrize("change,want", SIZES + [
    (dict(dys=11), EINVAL), (dict(dxs=11), EINVAL), (dict(dy=0), EINVAL), (dict(dx=0, dbias=0), EINVAL), (dict(dx=P + 4), EINVAL),
    (dict(dx=P + 4096 + 8), EINVAL), (dict(dbias=P + 2), EINVAL), (dict(ws=P + 2), EINVAL), (dict(ws=0), EINVAL),
    (dict(nbytes=2 * 3 * 4 - 1), EINVAL), (dict(N=9000, K=8, S=1, nbytes=3), EINVAL),
])
def test_dropout_backward(change, want):
    assert status(sw.swconv_dropout_backward, backward(**change)) == want


def test_dropout_workspace():
    assert sw.swconv_dropout_workspace_bytes(1, 10, 100) == 0          # one partial sum a channel: none is kept
    assert sw.swconv_dropout_workspace_bytes(6, 10, 100) == 6 * 10 * 4
    assert sw.swconv_dropout_workspace_bytes(0, 10, 100) == 0
    for sizes, want in (((-1, 1, 1), EINVAL), ((1, 0, 1), EINVAL), ((1, 1, 0), EINVAL), ((2**31, 1, 1), EUNSUPPORTED)):
        assert status(sw.swconv_dropout_workspace_bytes, sizes) == want
    assert sw.lib().swconv_dropout_workspace_bytes(1, 1, 1, None) == EINVAL


def logp_forward(**change):
    a = dict(dtype=0, rows=2, classes=10, x=P, stride=0, labels=P, top=3, ws=P, nbytes=1 << 30, stream=0, logprob=P, entropy=P, stats=P,
             tc=P, tl=P)
    a.update(change)
    return list(a.values())


def logp_backward(**change):
    a = dict(dtype=0, rows=2, classes=10, x=P, stride=0, labels=P, stats=P, entropy=P, g=P, h=P, stream=0, dx=P + 4096, dxs=0)
    a.update(change)
    return list(a.values())


SCORES = [
    (dict(dtype=7), EINVAL), (dict(rows=-1), EINVAL), (dict(classes=0), EINVAL), (dict(classes=2**31), EUNSUPPORTED),
    (dict(stride=9), EINVAL), (dict(stride=-10), EINVAL), (dict(stride=2**41), EUNSUPPORTED), (dict(rows=2**30, stride=2**20), EUNSUPPORTED),
    (dict(x=0), EINVAL), (dict(x=P + 2), EINVAL), (dict(dtype=2, x=P + 1), EINVAL), (dict(labels=0), EINVAL), (dict(labels=P + 2), EINVAL),
    (dict(stats=P + 1), EINVAL), (dict(entropy=P + 2), EINVAL),
]


@pytest.mark.parametrize("change,want", SCORES + [
    (dict(top=-1), EINVAL), (dict(top=65), EUNSUPPORTED), (dict(tc=0), EINVAL), (dict(tl=0), EINVAL), (dict(top=0), EINVAL),
    (dict(logprob=0, entropy=0, stats=0, top=0, tc=0, tl=0), EINVAL), (dict(logprob=P + 2), EINVAL), (dict(tc=P + 1), EINVAL),
    (dict(classes=1 << 20, ws=0), EINVAL), (dict(classes=1 << 20, ws=P + 8), EINVAL), (dict(classes=1 << 20, nbytes=100), EINVAL),
])
def test_logprobs_forward(change, want):
    assert status(sw.swconv_logprobs_forward, logp_forward(**change)) == want


@pytest.mark.parametrize("change,want", SCORES + [
    (dict(dxs=9), EINVAL), (dict(dx=0), EINVAL), (dict(stats=0), EINVAL), (dict(entropy=0), EINVAL), (dict(g=0, h=0), EINVAL),
    (dict(g=P + 2), EINVAL), (dict(h=P + 2), EINVAL), (dict(dx=P + 4), EINVAL), (dict(dx=P, dxs=12), EINVAL),
])
def test_logprobs_backward(change, want):
    assert status(sw.swconv_logprobs_backward, logp_backward(**change)) == want


def test_logprobs_workspace():
    assert sw.swconv_logprobs_workspace_bytes(0, 100, 1000, 5) == 0
    assert sw.swconv_logprobs_workspace_bytes(2, 1, 1 << 20, 5) > 0
    assert sw.swconv_logprobs_workspace_bytes(2, 0, 1 << 20, 5) == 0
    for args, want in (((9, 1, 1, 0), EINVAL), ((0, -1, 1, 0), EINVAL), ((0, 1, 0, 0), EINVAL), ((0, 1, 1, -1), EINVAL),
                       ((0, 1, 1, 65), EUNSUPPORTED), ((0, 1, 2**31, 0), EUNSUPPORTED)):
        assert status(sw.swconv_logprobs_workspace_bytes, args) == want
    assert sw.lib().swconv_logprobs_workspace_bytes(0, 1, 1, 0, None) == EINVAL
