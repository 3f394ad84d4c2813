"""Gradients of log probabilities for incoming gradients near the end of fp32: finite where the formula is, 0 at masked classes."""
import numpy as np
import pytest
import torch

from oracle import training as ref
from test_gpu_logprobs import same_or_close, scores
from training_ops import Rows, grad_bound, logprobs_backward, logprobs_forward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("classes", [50, 3001])
def test_entropy_gradients_near_the_end_of_fp32(classes):
    rows = 4
    x, labels, _ = scores(rows, classes, classes)
    x[:, 5] = -np.inf
    x[:, 7] = -300.0                                      # so far down that the exponential is 0
    x[:, 9] -= 100.0
    labels[:] = [5, 3, -1, 0]
    xs, lab = Rows("f32", rows, classes, values=x), torch.from_numpy(labels).cuda()
    fwd = logprobs_forward("f32", xs, lab, 0)
    g = np.array([1e30, -1e30, 1.0, 0.0], np.float32)
    h = np.array([3e36, -3e36, 1e37, 2e36], np.float32)
    dx = Rows("f32", rows, classes)
    logprobs_backward("f32", xs, lab, fwd, torch.from_numpy(g).cuda(), torch.from_numpy(h).cuda(), dx)
    x64 = xs.f64()
    _, H, stats, _, _ = ref.logprobs_forward(x64, labels, 0)
    want = ref.logprobs_backward(x64, labels, g, h)
    assert np.abs(want).max() < 3e38 and (want[:, 5] == 0).all()
    got = dx.f64()
    assert np.isfinite(got).all() and (got[:, 5] == 0).all()
    # a product with the last exponential that is not 0 may be lost: 2^-126 of h times its distance
    same_or_close(got, want, grad_bound("f32", x64, g, h, H, stats, want) + 2.0 ** -126 * 256 * np.abs(h)[:, None])
