"""What the tests of dropout and log probabilities share: tensors at any alignment inside guarded buffers, the calls, and
the bounds of their rounding errors."""
import numpy as np
import torch

from oracle import training as ref
from paper_1702_08597_amd import binding as sw

TYPES = {"f32": (sw.SWCONV_F32, torch.float32), "f16": (sw.SWCONV_F16, torch.float16), "bf16": (sw.SWCONV_BF16, torch.bfloat16)}
U = 2.0 ** -24  # half a step of fp32
GUARD = 77.0


def half_step(name):
    """Half a step of the type and the largest error among its subnormals; fp32 results are counted as operations."""
    return {"f32": (0.0, 2.0 ** -149), "f16": (2.0 ** -11, 2.0 ** -25), "bf16": (2.0 ** -8, 2.0 ** -134)}[name]


def stream():
    return torch.cuda.current_stream().cuda_stream


def ptr(t):
    return 0 if t is None else t.data_ptr()


class Rows:
    """rows x span values of a type, `stride` apart, `shift` elements behind an aligned address, guards everywhere else."""

    def __init__(self, name, rows, span, stride=0, shift=0, values=None):
        self.dtype = TYPES[name][1]
        self.rows, self.span, self.stride = rows, span, stride or span
        self.buffer = torch.full((shift + rows * self.stride + 64,), GUARD, dtype=self.dtype, device="cuda")
        self.view = self.buffer[shift:].as_strided((rows, span), (self.stride, 1))
        self.ptr = self.buffer.data_ptr() + shift * self.buffer.element_size()
        if values is not None:
            self.view.copy_(torch.as_tensor(values).reshape(rows, span))

    def f64(self):
        return self.view.double().cpu().numpy()

    def guards_hold(self):
        """What lies around and between the rows was left as it was."""
        rest = self.buffer.clone()
        rest.as_strided((self.rows, self.span), (self.stride, 1), self.view.storage_offset()).fill_(GUARD)
        return bool((rest == GUARD).all())


def guarded(n, dtype=torch.float32):
    b = torch.full((n + 16,), 77, dtype=dtype, device="cuda")
    return b


def workspace(nbytes):
    """Of the size asked for, with a guard behind it and NaN in it."""
    return torch.full((nbytes // 4 + 16,), float("nan"), device="cuda")


def rng_state(seed, step):
    two = np.array([seed % 2**64, step % 2**64], dtype=np.uint64).view(np.int64)
    return torch.from_numpy(two).cuda()


def dropout_forward(name, x, N, K, S, bias, relu, p, rng, offset, y):
    sw.swconv_dropout_forward(TYPES[name][0], N, K, S, x.ptr, x.stride, ptr(bias), relu, p, ptr(rng), offset, stream(), y.ptr,
                              y.stride)


def dropout_backward(name, dy, x, N, K, S, bias, relu, p, rng, offset, dx, dbias):
    nbytes = sw.swconv_dropout_workspace_bytes(N, K, S)
    ws = workspace(nbytes)
    sw.swconv_dropout_backward(TYPES[name][0], N, K, S, dy.ptr, dy.stride, x.ptr if x else 0, x.stride if x else 0, ptr(bias),
                               relu, p, ptr(rng), offset, ws.data_ptr(), nbytes, stream(), dx.ptr if dx else 0,
                               dx.stride if dx else 0, ptr(dbias))
    assert torch.isnan(ws[nbytes // 4:]).all()


def logprobs_forward(name, x, labels, top, entropy=True, stats=True):
    """-> dict of numpy arrays and the device tensors under "dev"."""
    rows, classes = x.rows, x.span
    nbytes = sw.swconv_logprobs_workspace_bytes(TYPES[name][0], rows, classes, top)
    ws = workspace(nbytes)
    lp, H, st = guarded(rows), guarded(rows), guarded(2 * rows)
    tc, tl = guarded(rows * top, torch.int32), guarded(rows * top)
    sw.swconv_logprobs_forward(TYPES[name][0], rows, classes, x.ptr, x.stride, ptr(labels), top, ws.data_ptr(), nbytes,
                               stream(), ptr(lp) if labels is not None else 0, ptr(H) if entropy else 0,
                               ptr(st) if stats else 0, ptr(tc) if top else 0, ptr(tl) if top else 0)
    for t, n in ((lp, rows), (H, rows), (st, 2 * rows), (tc, rows * top), (tl, rows * top)):
        assert (t[n:] == 77).all()
    assert torch.isnan(ws[nbytes // 4:]).all()
    n = lambda t, shape: t[:int(np.prod(shape))].cpu().numpy().reshape(shape)
    return dict(logprob=n(lp, (rows,)), entropy=n(H, (rows,)), stats=n(st, (rows, 2)), top_class=n(tc, (rows, top)),
                top_logprob=n(tl, (rows, top)), dev=dict(stats=st, entropy=H))


def logprobs_backward(name, x, labels, fwd, g, h, dx):
    sw.swconv_logprobs_backward(TYPES[name][0], x.rows, x.span, x.ptr, x.stride, ptr(labels), ptr(fwd["dev"]["stats"]),
                                ptr(fwd["dev"]["entropy"]) if h is not None else 0, ptr(g), ptr(h), stream(), dx.ptr, dx.stride)


# ---- bounds -----------------------------------------------------------------------------------------------------
def dropout_bound(name, want, operations):
    """`operations` roundings of fp32 (the scale's own among them) and the one to the type."""
    rel, tiny = half_step(name)
    return np.abs(want) * (operations * U + rel) * 1.001 + tiny


def dbias_bound(dz):
    """Each dz two roundings (scale, product); its way through the sums at most min(count, 1024) additions."""
    terms = dz.shape[0] * dz.shape[2]
    return (min(terms, 1024) + 2) * U * np.abs(dz).sum((0, 2)) * 1.001 + 1e-45


def row_bounds(x):
    """For every row the bounds of ls and of the entropy.  An exponential of d = x - m takes the subtraction, the product
    with log2 e and that constant's own rounding (3 U |d| in the exponent) and the instruction's error of one step (2 U);
    a running sum is scaled whenever the largest score changes, by factors of the same kind whose exponents add up to at
    most the range of the row, and by exactly 1 otherwise.  Weighted by p, the |d| add up to m - sum p x = ls - H.  Sums:
    at most classes / 64 + 32 additions one behind the other, and for every lane as many changes of the largest score as
    it has loads, three roundings each.  The logarithm and the outer sum: two steps."""
    x = np.asarray(x, np.float64)
    seen = np.isfinite(x)
    m = np.where(seen, x, -np.inf).max(1, initial=-np.inf)
    m = np.where(np.isfinite(m), m, 0.0)
    reach = np.minimum(m - np.where(seen, x, np.inf).min(1, initial=np.inf), 110.0)  # further down e is 0
    reach = np.where(np.isfinite(reach), reach, 0.0)
    with np.errstate(divide="ignore", invalid="ignore"):
        e = np.where(seen, np.exp(np.where(seen, x, 0) - m[:, None]), 0.0)
        s = np.maximum(e.sum(1), 1e-300)
        mean_d = -(e * np.where(e > 0, np.where(seen, x, 0) - m[:, None], 0.0)).sum(1) / s
    depth = x.shape[1] / 64 + 32
    rel = U * (3 * mean_d + 3 * reach + 4 * depth + 2)            # of s
    ls = rel + 4 * U * (np.abs(np.log(s)) + 1)
    rel_t = rel + U * (3 * reach + 4)                              # of t = sum d e: one more product, and d's own rounding
    H = ls + mean_d * (rel_t + rel + 2 * U) + 2 * U * (np.abs(np.log(s)) + mean_d)
    return m, ls, H


def logprob_bound(x, lp):
    """(x - m) - ls: the difference's rounding, ls's error, the outer difference's rounding."""
    m, ls, _ = row_bounds(x)
    lp = np.abs(np.where(np.isfinite(lp), lp, 0.0))
    extra = np.abs(np.log(x.shape[1])) + lp
    per_row = ls if lp.ndim == 1 else ls[:, None]
    return per_row + 2 * U * (lp + extra)


def grad_bound(name, x, g, h, entropy, stats, want):
    """p: its exponent has the error of log p and three roundings of its size; d = -p (g + h (lp + H)) [+ g]."""
    _, ls, H = row_bounds(x)
    with np.errstate(invalid="ignore", over="ignore"):
        lp = np.where(np.isfinite(x), (x - stats[:, :1]) - stats[:, 1:], -200.0)
        p = np.exp(np.maximum(lp, -200.0))
    elp = ls[:, None] + 4 * U * (np.abs(lp) + np.abs(stats[:, 1:]))
    g, h = np.abs(g)[:, None], np.abs(h)[:, None]
    factor = g + h * (np.abs(lp) + np.abs(entropy)[:, None])
    err = p * factor * (elp + 3 * U * np.abs(lp) + 8 * U) + p * h * (elp + H[:, None]) + 2 * U * g
    rel, tiny = half_step(name)
    return err * 1.01 + np.abs(want) * rel + 1e-37 + tiny  # below 2^-126 the exponential gives 0
