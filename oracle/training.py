"""Dropout between layers and log probabilities at a network's end, from their definitions in 64 bits (numpy): the
oracle of swconv_dropout_* and swconv_logprobs_*."""
from __future__ import annotations

import numpy as np

_LOW = 0xFFFFFFFF


def philox4x32_10(counter, key):
    """Salmon et al. 2011.  counter: four arrays (or numbers) of 32-bit words, key: two numbers -> four uint64 arrays."""
    c = [np.asarray(w, dtype=np.uint64) for w in counter]
    mask = np.uint64(_LOW)
    for r in range(10):
        k0, k1 = np.uint64((key[0] + r * 0x9E3779B9) & _LOW), np.uint64((key[1] + r * 0xBB67AE85) & _LOW)
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ k0, p1 & mask, (p0 >> np.uint64(32)) ^ c[3] ^ k1, p0 & mask]
    return c


def dropout_keep(N, K, S, p, seed, step):
    """-> (bool [N][K][S], scale)."""
    rows, cols = (N, K) if S == 1 else (N * K, S)
    seed, step = seed % 2**64, step % 2**64
    group = np.arange(-(-cols // 8))[None, :]
    words = philox4x32_10((group + np.zeros((rows, 1), int), np.arange(rows)[:, None] + 0 * group, step & _LOW, step >> 32),
                          (seed & _LOW, seed >> 32))
    fields = np.stack([np.broadcast_to(w >> np.uint64(s), (rows, group.size)) & np.uint64(0xFFFF) for w in words for s in (0, 16)], -1)
    threshold = int(np.rint(float(np.float32(p)) * 65536))
    keep = fields.reshape(rows, -1)[:, :cols] >= threshold
    return keep.reshape(N, K, S), (65536 / (65536 - threshold) if threshold < 65536 else 0.0)


def _biased(x, bias):
    return np.asarray(x, np.float64) + (0 if bias is None else np.asarray(bias, np.float64)[None, :, None])


def dropout_forward(x, bias, relu, p, seed, step):
    keep, scale = dropout_keep(*x.shape, p, seed, step)
    z = _biased(x, bias)
    return np.where(keep, np.where(relu & (z < 0), 0.0, z) * scale, 0.0)


def dropout_backward(dy, x, bias, relu, p, seed, step):
    """-> dx, dbias."""
    keep, scale = dropout_keep(*dy.shape, p, seed, step)
    if relu:
        keep = keep & ~(_biased(x, bias) <= 0)
    dz = np.where(keep, np.asarray(dy, np.float64) * scale, 0.0)
    return dz, dz.sum((0, 2))


def logprobs_forward(x, labels, top):
    """x [rows][classes] -> logprob, entropy, stats [rows][2], top_class, top_logprob."""
    x = np.asarray(x, np.float64)
    rows, classes = x.shape
    logprob, entropy, stats = np.zeros(rows), np.zeros(rows), np.zeros((rows, 2))
    top_class, top_logprob = np.full((rows, top), -1, np.int32), np.full((rows, top), -np.inf)
    for i in range(rows):
        label = -1 if labels is None else int(labels[i])
        if np.isnan(x[i]).any() or np.isposinf(x[i]).any():
            entropy[i], stats[i], top_logprob[i] = np.nan, np.nan, np.nan
            logprob[i] = 0.0 if label < 0 else np.nan
            continue
        seen = np.flatnonzero(x[i] > -np.inf)
        if seen.size:
            m = x[i].max()
            e = np.exp(x[i][seen] - m)
            ls = np.log(e.sum())
            logp = np.full(classes, -np.inf)
            logp[seen] = (x[i][seen] - m) - ls
            q = e / e.sum()
            entropy[i] = -(q * np.where(q > 0, logp[seen], 0.0)).sum()
            order = seen[np.lexsort((seen, -(x[i][seen] + 0.0)))][:top]
            top_class[i, :order.size], top_logprob[i, :order.size] = order, logp[order]
        else:
            m, ls, logp = -np.inf, 0.0, np.full(classes, -np.inf)
        stats[i] = m, ls
        logprob[i] = 0.0 if label < 0 else (np.nan if label >= classes else logp[label])
    return logprob, entropy, stats, top_class, top_logprob


def logprobs_backward(x, labels, g, h):
    """g, h: dL/d(logprob), dL/d(entropy) by row, or None."""
    x = np.asarray(x, np.float64)
    rows, classes = x.shape
    _, entropy, stats, _, _ = logprobs_forward(x, None, 0)
    dx = np.zeros_like(x)
    for i in range(rows):
        label = -1 if labels is None else int(labels[i])
        gi = 0.0 if g is None or label < 0 else (float(g[i]) if label < classes else np.nan)
        hi = 0.0 if h is None else float(h[i])
        if np.isnan(stats[i]).any():
            dx[i] = np.where(np.isneginf(x[i]), 0.0, np.nan)
            continue
        seen = x[i] > -np.inf
        lp = (x[i][seen] - stats[i, 0]) - stats[i, 1]
        q = np.exp(lp)
        d = -q * gi - hi * np.where(q > 0, q * (np.where(q > 0, lp, 0.0) + entropy[i]), 0.0)
        dx[i][seen] = d
        if 0 <= label < classes and seen[label]:
            dx[i, label] += gi
    return dx
