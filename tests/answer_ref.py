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
    bias are two more operations.  Rounding: half a step of the result."""
    w = q4_weights(q, scales, zeros, x.shape[-1], group)
    xd = x.double().cpu()
    y = xd @ w.t()
    mag = xd.abs() @ w.abs().t()
    if bias is not None:
        y = y + bias.double()
        mag = mag + bias.double().abs()
    if act != "none":
        y = y.clamp(min=0.0, max=6.0 if act == "relu6" else math.inf)
    sums = (x.shape[-1] * (3 if x.dtype == torch.float32 else 1) + 3) * 2.0 ** -23 * mag
    return y, sums + (y.abs() + sums) * UNIT[x.dtype] + TINY[x.dtype]
