"""The operators around a layer in training and at a network's end, as measurable cases.

  dropout        bias, ReLU and dropout of feature maps or feature rows: swconv_dropout_forward
  dropout_grad   its backward pass, with the bias gradient: swconv_dropout_backward
  logprobs       log probabilities of given classes (or tokens), entropy and the best alternatives:
                 swconv_logprobs_forward
  logprobs_grad  the gradient of a loss over log probabilities and entropies: swconv_logprobs_backward
  logprobs_step  both, as a training step calls them

With `own` false, `run` computes them in elementary torch operations; `exact` computes them in 64 bits.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}


# --------------------------------------------------------------------------------------------------------------
# cases
# --------------------------------------------------------------------------------------------------------------
def _dropout(name, op, dtype, N, K, S, p, relu=True, bias=True, gap=0):
    """gap: elements between one image's K x S values and the next image's (a channel group of a larger tensor)."""
    return {"name": name, "op": op, "dtype": dtype, "N": N, "K": K, "S": S, "p": p, "relu": relu, "bias": bias,
            "gap": gap}


def _logprobs(name, op, dtype, rows, classes, top, entropy=True, pad=0, masked=0.0):
    """pad: unused scores behind each row; masked: the share of classes that a mask has set to -inf."""
    return {"name": name, "op": op, "dtype": dtype, "rows": rows, "classes": classes, "top": top, "entropy": entropy,
            "pad": pad, "masked": masked}


def listed():
    return [
        # the rows in front of a classifier at a small batch: half a megabyte, latency is everything
        _dropout("dropout_features_small", "dropout", "f32", 32, 4096, 1, 0.5),
        # the output of the 56 x 56 layer, the largest feature maps of this repository's configurations
        _dropout("dropout_maps_56", "dropout", "f32", 32, 256, 56 * 56, 0.1),
        # one of two channel groups of 27 x 27 maps, inside the whole layer's tensor: odd planes, image strides
        _dropout("dropout_maps_27_group", "dropout", "f16", 32, 128, 27 * 27, 0.2, gap=128 * 27 * 27),
        # backward on the 13 x 13 maps: planes of 169, the bias gradient summed over images and pixels
        _dropout("dropout_grad_maps_13", "dropout_grad", "f32", 64, 384, 13 * 13, 0.25),
        # long rows of features in bfloat16, the largest dropout passes
        _dropout("dropout_features_large", "dropout", "bf16", 16384, 4096, 1, 0.1, relu=False),
        _dropout("dropout_grad_features_large", "dropout_grad", "bf16", 16384, 4096, 1, 0.1),
        # one step of serving: a single row over a vocabulary, five alternatives
        _logprobs("logprobs_one_row", "logprobs", "bf16", 1, 32768, 5),
        # a batch of rows while decoding, a vocabulary that divides by nothing, twenty alternatives
        _logprobs("logprobs_decode", "logprobs", "bf16", 64, 150001, 20, masked=0.01),
        # a classifier of 1000 classes judged by its five best
        _logprobs("logprobs_classifier_step", "logprobs_step", "f32", 256, 1000, 5),
        # fine-tuning with a padded vocabulary: ragged rows, both directions
        _logprobs("logprobs_step_ragged", "logprobs_step", "f16", 777, 50021, 0, pad=43),
        # scoring and training over long rows: the largest passes
        _logprobs("logprobs_large", "logprobs", "bf16", 4096, 131072, 1),
        _logprobs("logprobs_grad_large", "logprobs_grad", "bf16", 4096, 131072, 0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Rows of 1 to 16384 and planes of 7 to 64 pixels a side for dropout; 1 to 8192 rows of 10 to 262144 classes."""
    while True:
        dtype = rng.choice(["f32", "f16", "bf16"])
        if rng.random() < 0.45:
            op = rng.choice(["dropout", "dropout_grad"])
            if rng.random() < 0.5:
                N, K, S = _log(rng, 1, 64), _log(rng, 16, 512), _log(rng, 7, 64) * _log(rng, 7, 64)
                gap = rng.choice([0, 0, K * S, rng.randrange(1, 64)])
            else:
                N, K, S = _log(rng, 1, 16384), _log(rng, 10, 16384), 1
                gap = rng.choice([0, 0, rng.randrange(1, 64)])
            case = _dropout(None, op, dtype, N, K, S, round(rng.uniform(0.0, 0.6), 3), rng.random() < 0.6,
                            rng.random() < 0.7, gap)
            top = _dropout(None, "dropout_grad", "bf16", 16384, 4096, 1, 0.1)
        else:
            op = rng.choice(["logprobs", "logprobs", "logprobs_grad", "logprobs_step"])
            k = rng.choice([0, 0, 1, 5, 20, rng.randrange(0, 65)]) if op != "logprobs_grad" else 0
            case = _logprobs(None, op, dtype, _log(rng, 1, 8192), _log(rng, 10, 262144), k, rng.random() < 0.7,
                             rng.choice([0, 0, rng.randrange(1, 128)]), rng.choice([0.0, 0.0, 0.02, 0.5]))
            top = _logprobs(None, "logprobs_grad", "bf16", 4096, 131072, 0)
            if case["rows"] * case["classes"] * max(case["top"], 1) > 1 << 29:  # the plain form looks once per place
                continue
        del case["name"]
        if work(case)["bytes"] <= work(top)["bytes"]:
            return case


def work(case):
    """Tensors once in and once out.  Per element: bias, ReLU, comparison and scale; or difference, exp, two sums and
    the entropy's product (forward), difference, exp and two products (backward)."""
    op, size = case["op"], SIZE[case["dtype"]]
    if op.startswith("dropout"):
        n = case["N"] * case["K"] * case["S"]
        reads = 2 if op == "dropout_grad" and case["relu"] else 1
        return {"bytes": n * size * (reads + 1) + 8 * case["K"] * case["bias"], "flops": 4 * n}
    n, rows = case["rows"] * case["classes"], case["rows"]
    forward, backward = op != "logprobs_grad", op != "logprobs"
    nbytes = n * size * (forward + 2 * backward) + rows * (4 + forward * (16 + 8 * case["top"]) + backward * 20)
    return {"bytes": nbytes, "flops": n * (6 * forward + 6 * backward)}


# --------------------------------------------------------------------------------------------------------------
# what a user's program holds
# --------------------------------------------------------------------------------------------------------------
class _State:
    pass


def _image_views(buffer, N, K, S, gap):
    return buffer.as_strided((N, K, S), (K * S + gap, S, 1))


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = _State()
    s.case, s.dtype = dict(case), DTYPES[case["dtype"]]
    if case["op"].startswith("dropout"):
        N, K, S, gap = case["N"], case["K"], case["S"], case["gap"]
        length = N * (K * S + gap)
        s.stride = K * S + gap
        s.x = torch.randn(length, generator=gen, device="cuda").to(s.dtype)
        s.bias = torch.randn(K, generator=gen, device="cuda").mul_(0.1) if case["bias"] else None
        # the generator's state on the device: the seed and the training step
        s.rng = torch.tensor([0x5DEECE66D + 7919 * seed, 1000 + seed], dtype=torch.int64, device="cuda")
        s.offset = 3  # the layer's number in its network
        s.out = torch.zeros(length, dtype=s.dtype, device="cuda")
        s.out_view = _image_views(s.out, N, K, S, gap)
        s.x_view = _image_views(s.x, N, K, S, gap)
        if case["op"] == "dropout_grad":
            s.dy = torch.randn(length, generator=gen, device="cuda").mul_(0.01).to(s.dtype)
            s.dy_view = _image_views(s.dy, N, K, S, gap)
            s.dbias = torch.empty(K, device="cuda") if case["bias"] else None
            if own:
                from paper_1702_08597_amd import binding as sw
                s.work = torch.empty(sw.swconv_dropout_workspace_bytes(N, K, S), dtype=torch.uint8, device="cuda")
        return s
    rows, classes, k = case["rows"], case["classes"], case["top"]
    s.stride = classes + case["pad"]
    # scores of a trained model: a broad body and, in each row, one class that stands out
    s.scores = torch.randn((rows, s.stride), generator=gen, device="cuda").mul_(2.0)
    best = torch.randint(0, classes, (rows, 1), generator=gen, device="cuda")
    s.scores.scatter_(1, best, torch.rand((rows, 1), generator=gen, device="cuda").mul_(9.0).add_(5.0))
    other = torch.randint(0, classes, (rows,), generator=gen, device="cuda")
    likely = torch.rand(rows, generator=gen, device="cuda") < 0.6
    labels = torch.where(likely, best[:, 0], other)
    if case["masked"]:
        hidden = torch.rand((classes,), generator=gen, device="cuda") < case["masked"]
        hidden[0] = False
        s.scores[:, :classes].masked_fill_(hidden[None, :], float("-inf"))
        labels = torch.where(hidden[labels], s.scores[:, :classes].argmax(1), labels)
    # positions without a label, as the padding of a batch has them
    labels = torch.where(torch.rand(rows, generator=gen, device="cuda") < 0.05, torch.full_like(labels, -1), labels)
    s.labels = labels.to(torch.int32)
    s.scores = s.scores.to(s.dtype)
    if case["op"] != "logprobs_grad":
        s.logprob = torch.empty(rows, device="cuda")
        s.entropy = torch.empty(rows, device="cuda") if case["entropy"] else None
        s.stats = torch.empty((rows, 2), device="cuda")
        s.top_class = torch.empty((rows, k), dtype=torch.int32, device="cuda") if k else None
        s.top_logprob = torch.empty((rows, k), device="cuda") if k else None
        if own:
            from paper_1702_08597_amd import binding as sw
            nbytes = sw.swconv_logprobs_workspace_bytes(_dtype_code(case), rows, classes, k)
            s.work = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    else:
        # what the forward pass of the same step left
        f = _plain_logprobs(s.scores[:, :classes], s.labels, 0, case["entropy"])
        s.logprob, s.stats = f["logprob"], f["stats"]
        s.entropy = f["entropy"] if case["entropy"] else None
    if case["op"] != "logprobs":
        # a mean of negative log probabilities with a weight for each row, and an entropy bonus
        s.dlogprob = -(0.5 + torch.rand(rows, generator=gen, device="cuda")) / rows
        s.dentropy = torch.full((rows,), -0.01 / rows, device="cuda") if case["entropy"] else None
        s.dscores = torch.zeros((rows, s.stride), dtype=s.dtype, device="cuda")
    return s


def _dtype_code(case):
    from paper_1702_08597_amd import binding as sw
    return {"f32": sw.SWCONV_F32, "f16": sw.SWCONV_F16, "bf16": sw.SWCONV_BF16}[case["dtype"]]


def _ptr(t):
    return 0 if t is None else t.data_ptr()


# --------------------------------------------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------------------------------------------
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_1702_08597_amd import binding as sw
    c, stream, code = s.case, torch.cuda.current_stream().cuda_stream, _dtype_code(s.case)
    if c["op"] == "dropout":
        sw.swconv_dropout_forward(code, c["N"], c["K"], c["S"], s.x.data_ptr(), s.stride, _ptr(s.bias), c["relu"],
                                  c["p"], s.rng.data_ptr(), s.offset, stream, s.out.data_ptr(), s.stride)
        return s.out_view
    if c["op"] == "dropout_grad":
        sw.swconv_dropout_backward(code, c["N"], c["K"], c["S"], s.dy.data_ptr(), s.stride, s.x.data_ptr(), s.stride,
                                   _ptr(s.bias), c["relu"], c["p"], s.rng.data_ptr(), s.offset, s.work.data_ptr(),
                                   s.work.numel(), stream, s.out.data_ptr(), s.stride, _ptr(s.dbias))
        return (s.out_view, s.dbias) if c["bias"] else (s.out_view,)
    rows, classes = c["rows"], c["classes"]
    out = ()
    if c["op"] != "logprobs_grad":
        sw.swconv_logprobs_forward(code, rows, classes, s.scores.data_ptr(), s.stride, s.labels.data_ptr(), c["top"],
                                   s.work.data_ptr(), s.work.numel(), stream, s.logprob.data_ptr(), _ptr(s.entropy),
                                   s.stats.data_ptr(), _ptr(s.top_class), _ptr(s.top_logprob))
        out = tuple(t for t in (s.logprob, s.stats, s.entropy, s.top_class, s.top_logprob) if t is not None)
    if c["op"] != "logprobs":
        sw.swconv_logprobs_backward(code, rows, classes, s.scores.data_ptr(), s.stride, s.labels.data_ptr(),
                                    s.stats.data_ptr(), _ptr(s.entropy), s.dlogprob.data_ptr(), _ptr(s.dentropy),
                                    stream, s.dscores.data_ptr(), s.stride)
        out += (s.dscores[:, :classes],)
    return out


def _run_plain(s):
    c = s.case
    if c["op"].startswith("dropout"):
        keep, scale = _plain_keep(s)
        z = s.x_view.float()
        if s.bias is not None:
            z = z + s.bias[None, :, None]
        if c["op"] == "dropout":
            if c["relu"]:
                z = torch.where(z < 0, torch.zeros_like(z), z)
            y = torch.where(keep, z * scale, torch.zeros_like(z)).to(s.dtype)
            return y
        if c["relu"]:
            keep = keep & (z > 0)
        dz = torch.where(keep, s.dy_view.float() * scale, torch.zeros_like(z))
        return (dz.to(s.dtype), dz.sum((0, 2))) if c["bias"] else (dz.to(s.dtype),)
    scores = s.scores[:, :c["classes"]]
    out = ()
    if c["op"] != "logprobs_grad":
        f = _plain_logprobs(scores, s.labels, c["top"], c["entropy"])
        out = tuple(f[k] for k in ("logprob", "stats", "entropy", "top_class", "top_logprob") if k in f)
        stats, entropy = f["stats"], f.get("entropy")
    else:
        stats, entropy = s.stats, s.entropy
    if c["op"] != "logprobs":
        out += (_plain_logprobs_grad(scores, s.labels, stats, entropy, s.dlogprob, s.dentropy),)
    return out


_M0, _M1, _W0, _W1, _LOW = 0xD2511F53, 0xCD9E8D57, 0x9E3779B9, 0xBB67AE85, 0xFFFFFFFF


def _plain_keep(s):
    """keep[n][k][s] and the scale: 16-bit fields of philox4x32-10, compared with the rate.  Products of two 32-bit
    words wrap in int64 and keep all their 64 bits."""
    c = s.case
    N, K, S = c["N"], c["K"], c["S"]
    rows, cols = (N, K) if S == 1 else (N * K, S)
    threshold = round(c["p"] * 65536)
    scale = 65536.0 / (65536 - threshold) if threshold < 65536 else 0.0
    key0, key1 = s.rng[0] & _LOW, (s.rng[0] >> 32) & _LOW
    step = s.rng[1] + s.offset
    groups = (cols + 7) // 8
    c0 = torch.arange(groups, device="cuda").repeat(rows, 1)
    c1 = torch.arange(rows, device="cuda")[:, None].expand(rows, groups)
    c2, c3 = (step & _LOW).expand(rows, groups), ((step >> 32) & _LOW).expand(rows, groups)
    for _ in range(10):
        a, b = c0 * _M0, c2 * _M1
        c0, c1, c2, c3 = ((b >> 32) & _LOW) ^ c1 ^ key0, b & _LOW, ((a >> 32) & _LOW) ^ c3 ^ key1, a & _LOW
        key0, key1 = (key0 + _W0) & _LOW, (key1 + _W1) & _LOW
    fields = torch.stack([h for w in (c0, c1, c2, c3) for h in (w & 0xFFFF, w >> 16)], dim=-1)
    keep = fields.view(rows, groups * 8)[:, :cols] >= threshold
    return keep.reshape(N, K, S), scale


def _plain_logprobs(scores, labels, top, entropy):
    x = scores.float()
    rows = torch.arange(x.shape[0], device=x.device)
    m = x.amax(1, keepdim=True)
    d = x - m
    e = d.exp()
    total = e.sum(1, keepdim=True)
    ls = total.log()
    wanted = labels.long().clamp(min=0)
    logprob = torch.where(labels >= 0, d[rows, wanted] - ls[:, 0], torch.zeros_like(ls[:, 0]))
    out = {"logprob": logprob, "stats": torch.cat([m, ls], 1)}
    if entropy:
        out["entropy"] = ls[:, 0] - torch.where(e > 0, e * d, torch.zeros_like(e)).sum(1) / total[:, 0]
    if top:
        index = torch.empty((x.shape[0], top), dtype=torch.int32, device=x.device)
        value = torch.empty((x.shape[0], top), device=x.device)
        left = d.clone()
        for i in range(top):
            best, at = left.max(1)  # the first of equal ones
            value[:, i] = best - ls[:, 0]
            index[:, i] = torch.where(best > float("-inf"), at, torch.full_like(at, -1))
            left.scatter_(1, at[:, None], float("-inf"))
        out["top_class"], out["top_logprob"] = index, value
    return out


def _plain_logprobs_grad(scores, labels, stats, entropy, dlogprob, dentropy):
    logp = scores.float() - stats[:, :1] - stats[:, 1:]
    p = logp.exp()
    g = torch.where(labels >= 0, dlogprob, torch.zeros_like(dlogprob))
    factor = g[:, None].expand_as(p)
    if dentropy is not None:
        factor = torch.where(p > 0, factor + dentropy[:, None] * (logp + entropy[:, None]), torch.zeros_like(p))
    grad = -p * factor
    rows = torch.arange(p.shape[0], device=p.device)
    grad[rows, labels.long().clamp(min=0)] += g
    return grad.to(scores.dtype)


# --------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# --------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return _exact_dropout(s) if case["op"].startswith("dropout") else _exact_logprobs(s)


def _philox_words(counter, key):
    """philox4x32-10 in numpy: the product's halves from 64-bit words, the key schedule by multiples of its step."""
    x = [np.asarray(w, dtype=np.uint64) for w in counter]
    low = np.uint64(0xFFFFFFFF)
    for r in range(10):
        k0 = np.uint64((key[0] + r * 0x9E3779B9) % 2**32)
        k1 = np.uint64((key[1] + r * 0xBB67AE85) % 2**32)
        left, right = np.uint64(0xD2511F53) * x[0], np.uint64(0xCD9E8D57) * x[2]
        x = [(right >> np.uint64(32)) ^ x[1] ^ k0, right & low, (left >> np.uint64(32)) ^ x[3] ^ k1, left & low]
    return x


def _exact_dropout(s):
    c = s.case
    N, K, S = c["N"], c["K"], c["S"]
    rows, cols = (N, K) if S == 1 else (N * K, S)
    seed, step = (int(v) for v in s.rng.tolist())
    step = (step + s.offset) % 2**64
    group, row = np.meshgrid(np.arange(-(-cols // 8)), np.arange(rows))
    words = _philox_words((group, row, np.full(group.shape, step % 2**32), np.full(group.shape, step >> 32)),
                          (seed % 2**32, (seed >> 32) % 2**32))
    threshold = int(np.rint(c["p"] * 65536))
    u = np.stack(words, -1).astype(np.uint32).view(np.uint16)  # little-endian: the low half of each word first
    keep = torch.from_numpy(u.reshape(rows, -1)[:, :cols] >= threshold).cuda().view(N, K, S)
    z = s.x_view.double()
    if s.bias is not None:
        z = z + s.bias.double().view(1, K, 1)
    scale = 65536 / (65536 - threshold) if threshold < 65536 else 0.0
    if c["op"] == "dropout":
        return (z.clamp(min=0) if c["relu"] else z) * scale * keep
    dz = s.dy_view.double() * scale * (keep & (z > 0) if c["relu"] else keep)
    return (dz, dz.sum(2).sum(0)) if c["bias"] else (dz,)


def _exact_logprobs(s):
    c = s.case
    parts = []
    for r in range(0, c["rows"], max(1, (1 << 26) // c["classes"])):
        at = slice(r, r + max(1, (1 << 26) // c["classes"]))
        x, labels = s.scores[at, :c["classes"]].double(), s.labels[at].long()
        has = labels >= 0
        logp = torch.log_softmax(x, 1)
        p = logp.exp()
        plogp = torch.nan_to_num(p * logp, nan=0.0)  # a masked class adds nothing
        H = -plogp.sum(1)
        out = []
        if c["op"] != "logprobs_grad":
            m = x.max(1).values
            out.append(torch.where(has, logp.gather(1, labels.clamp(min=0)[:, None])[:, 0], 0.0))
            out.append(torch.stack([m, torch.logsumexp(x - m[:, None], 1)], 1))
            if c["entropy"]:
                out.append(H)
            if c["top"]:
                value, index = torch.sort(logp, dim=1, descending=True, stable=True)
                value, index = value[:, :c["top"]], index[:, :c["top"]].to(torch.int32)
                if c["classes"] < c["top"]:
                    short = (0, c["top"] - c["classes"])
                    value = torch.nn.functional.pad(value, short, value=float("-inf"))
                    index = torch.nn.functional.pad(index, short, value=-1)
                out += [torch.where(value > float("-inf"), index, -1), value.contiguous()]
        if c["op"] != "logprobs":
            g = torch.where(has, s.dlogprob[at].double(), 0.0)
            grad = -p * g[:, None]
            if c["entropy"]:
                grad -= s.dentropy[at].double()[:, None] * (plogp + p * H[:, None])
            grad.scatter_add_(1, labels.clamp(min=0)[:, None], g[:, None])
            out.append(grad)
        parts.append(out)
    return tuple(torch.cat(column) for column in zip(*parts))
