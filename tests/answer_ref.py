"""Plain forms of the operators on rows, in 64 bits on the CPU, for the tests."""
import math

import numpy as np
import torch

UNIT = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}  # half a step, relative
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134, torch.float32: 2.0 ** -150}  # half a step of the smallest values


def q4_layer(seed, cin, cout, group, scale_dtype=torch.float16, zeros=False, bias=True):
    """Random weights of a layer: packed values, scales, zero points, bias."""
    g = torch.Generator().manual_seed(seed)
    groups = -(-cin // group)
    q = torch.randint(0, 256, (cout, (cin + 1) // 2), generator=g, dtype=torch.uint8)
    scales = (torch.rand((cout, groups), generator=g) + 0.5).mul(0.1 / math.sqrt(cin)).to(scale_dtype)
    z = torch.randint(0, 16, (cout, groups), generator=g, dtype=torch.uint8) if zeros else None
    b = torch.randn((cout,), generator=g) if bias else None
    return q, scales, z, b


def q4_weights(q, scales, zeros, cin, group):
    """w[o, k] in 64 bits."""
    v = torch.stack([q & 15, q >> 4], -1).flatten(1)[:, :cin].double()
    of = torch.arange(cin) // group
    z = zeros.double()[:, of] if zeros is not None else 8.0
    return (v - z) * scales.double()[:, of]


def linear_q4(x, q, scales, zeros, bias, group, act="none"):
    """(y, bound): the product in 64 bits and how far a kernel may be from it that forms the products exactly, adds them up in
    fp32 in any order and rounds once to x's type.

    n products (three for each input in 32 bits, which counts in three parts) added in any order, each addition off by at most 2^-23 of
    its result (twice half a step: a matrix instruction may cut off instead of rounding): n 2^-23 sum |products|; a scale and the
    bias are two more operations.  Rounding: half a step of the result.

    More than 16 rows of a 16-bit type: each weight may be rounded to that type first - half a step of it, a little more where its scale
    enters in two parts, and half of fp16's smallest step (2^-25) of a weight brought to the output's largest scale (by less than twice
    its inverse)."""
    w = q4_weights(q, scales, zeros, x.shape[-1], group)
    xd = x.double().cpu()
    y = xd @ w.t()
    mag = xd.abs() @ w.abs().t()
    rounded = 0.0
    if x.shape[0] > 16 and x.dtype != torch.float32:
        rounded = 1.02 * UNIT[x.dtype] * mag + 2.0 ** -24 * xd.abs().sum(1, keepdim=True) * scales.double().abs().amax(1)
    if bias is not None:
        y = y + bias.double()
        mag = mag + bias.double().abs()
    if act != "none":
        y = y.clamp(min=0.0, max=6.0 if act == "relu6" else math.inf)
    sums = (x.shape[-1] * (3 if x.dtype == torch.float32 else 1) + 3) * 2.0 ** -23 * mag + rounded
    return y, sums + (y.abs() + sums) * UNIT[x.dtype] + TINY[x.dtype]


def log_probs(logits, given=None, top=0, temperature=1.0):
    """{"given", "entropy", "top", "top_ids"} in 64 bits, and {"log", "entropy"}: how far a kernel in fp32 may be off.

    With d = (x - max) / T and p = softmax, an exponential is off by 4 |d| 2^-24 (its argument takes four roundings) and 2^-21 of
    itself.  A thread adds up at most n = classes / 32 + 64 of them, each addition, and each change to a new maximum, off by 2^-22 at
    most.  So ln S is off by n 2^-22 + 4 sum p |d| 2^-24; a log probability by that and four roundings of its own d, which is what
    a caller adds as 2^-22 |log p|; and the entropy by the same errors of sum p d, each weighted with its d."""
    x = logits.double().cpu() / float(np.float32(temperature))
    rows, classes = x.shape
    some = x.amax(1, keepdim=True) > -math.inf
    d = torch.where(some, x - torch.where(some, x.amax(1, keepdim=True), 0.0), -math.inf)
    log_s = torch.where(some, d.exp().sum(1, keepdim=True).log(), 0.0)
    lp = d - log_s
    p = lp.exp()
    pd = torch.where(p > 0, p * d, 0.0)
    out = {"entropy": torch.where(some[:, 0], log_s[:, 0] - pd.sum(1), 0.0)}
    if given is not None:
        g = given.cpu().long()
        out["given"] = torch.where(g < 0, 0.0, torch.where(g < classes, lp.gather(1, g.clamp(0, classes - 1)), math.nan))
    if top:
        order = np.lexsort((np.broadcast_to(np.arange(classes), (rows, classes)), -logits.double().cpu().numpy()), axis=1)[:, :top]
        out["top_ids"] = torch.from_numpy(np.ascontiguousarray(order)).int()
        out["top"] = lp.gather(1, out["top_ids"].long())
    n = (classes / 32 + 64) * 2.0 ** -22
    absd = pd.abs().sum(1)
    ln = n + 4 * absd * 2.0 ** -24
    ent = (1 + absd) * ln + 4 * torch.where(p > 0, p * d * d, 0.0).sum(1) * 2.0 ** -24 + n * absd
    return out, {"log": ln, "entropy": ent}
