"""The operators at the answer's end of a network, as measurable cases.

  linear      a fully connected layer whose weights are held in 4 bits with a scale (and, where asked for, a zero point) for each
              group of input channels: y = act(x w^T + bias), w[o, k] = scale[o, k / group] * (q[o, k] - zero[o, k / group])
  log_probs   for each row of logits: log probabilities of given classes, the entropy and the `top` most probable classes with
              their log probabilities, at a temperature

Fields of a case:

  op          "linear" | "log_probs"
  dtype       "f16" | "bf16" | "f32": activations in and out, or logits
  linear:     rows, cin, cout, group; scale ("f16" | "bf16" | "f32"); zeros, bias (truth values); act ("none" | "relu" | "relu6")
  log_probs:  rows, classes, given (classes asked for in each row), top, temperature; pitch (values between rows);
              mask "none" | "inf" (classes excluded by minus infinity) | "lowest" (by the type's lowest value)
"""
import math

import torch

own = False

_DTYPE = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
_BYTES = {"f16": 2, "bf16": 2, "f32": 4}
_DEV = "cuda:0"


def listed():
    def linear(name, rows, cin, cout, dtype, group, scale, zeros=False, bias=True, act="none"):
        return {"name": name, "op": "linear", "rows": rows, "cin": cin, "cout": cout, "dtype": dtype, "group": group, "scale": scale,
                "zeros": zeros, "bias": bias, "act": act}

    def log_probs(name, rows, classes, dtype, given, top, temperature=1.0, pitch=None, mask="none"):
        return {"name": name, "op": "log_probs", "rows": rows, "classes": classes, "dtype": dtype, "given": given, "top": top,
                "temperature": temperature, "pitch": pitch or classes, "mask": mask}

    return [
        # the classifier of one image: the last layer of the benchmark networks, where only latency counts
        linear("linear_1x1280_1001", 1, 1280, 1001, "f16", 32, "f16"),
        # one token through a square projection
        linear("linear_1x4096_4096", 1, 4096, 4096, "bf16", 128, "bf16", bias=False),
        # one token through a layer larger than what a pass can hide: bound by the weights' bytes
        linear("linear_1x8192_28672", 1, 8192, 28672, "f16", 128, "f16", bias=False),
        # odd sizes in the accurate type, with zero points
        linear("linear_3x1000_1537_f32", 3, 1000, 1537, "f32", 64, "f32", zeros=True, act="relu6"),
        # a batch of sequences that decode together, zero points and small groups
        linear("linear_16x5120_13824", 16, 5120, 13824, "f16", 64, "f16", zeros=True, act="relu"),
        # a short prompt, or many sequences: the products count as much as the bytes
        linear("linear_256x4096_12288", 256, 4096, 12288, "bf16", 128, "bf16"),
        # the answer for one image: label's log probability, entropy, the usual five best
        log_probs("log_probs_1x1001", 1, 1001, "f16", 1, 5),
        # the same for a batch of the throughput benchmark
        log_probs("log_probs_256x1001", 256, 1001, "f16", 1, 5),
        # one token over a large vocabulary: one row has to fill the GPU
        log_probs("log_probs_1x262144_f32", 1, 262144, "f32", 1, 20, temperature=0.7),
        # a decoding batch: odd vocabulary in padded rows, classes masked out, several candidates scored
        log_probs("log_probs_64x50257", 64, 50257, "bf16", 4, 8, pitch=50304, mask="inf"),
        # scoring a long text: bound by the logits' bytes
        log_probs("log_probs_2048x131072", 2048, 131072, "f16", 1, 5),
        # every pixel of a segmentation batch: many rows of few classes
        log_probs("log_probs_pixels_x21", 16 * 513 * 513, 21, "f16", 1, 1),
    ]


def _spread(rng, lo, hi):
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    """A case of the same ranges; sizes spread over their logarithm, odd ones among them."""
    dtype = rng.choice(["f16", "f16", "bf16", "f32"])
    if rng.random() < 0.5:
        cin, cout = _spread(rng, 33, 8192), _spread(rng, 17, 28672)
        if rng.random() < 0.5:
            cin, cout = (cin + 63) // 64 * 64, (cout + 63) // 64 * 64
        # the products of a row of 32 bits cost more: fewer of them
        rows = _spread(rng, 1, 32 if dtype == "f32" else 256)
        rows = max(1, min(rows, 256 * 4096 * 12288 // (cin * cout)))
        return {"op": "linear", "rows": rows, "cin": cin, "cout": cout, "dtype": dtype, "group": rng.choice([32, 64, 96, 128, 256]),
                "scale": rng.choice([dtype, "f32"]), "zeros": rng.random() < 0.5, "bias": rng.random() < 0.5, "act": rng.choice(["none", "none", "relu", "relu6"])}
    classes = _spread(rng, 8, 262144)
    rows = _spread(rng, 1, max(1, min(1 << 20, (1 << 28) // classes // _BYTES[dtype])))
    return {"op": "log_probs", "rows": rows, "classes": classes, "dtype": dtype, "given": rng.choice([0, 1, 1, 4]),
            "top": min(classes, rng.choice([0, 1, 5, 20, rng.randint(1, 32)])), "temperature": rng.choice([1.0, 0.7, round(rng.uniform(0.3, 2.0), 3)]),
            "pitch": classes if rng.random() < 0.6 else classes + rng.randint(1, 64), "mask": rng.choice(["none", "none", "inf", "lowest"])}


def _linear_inputs(case, seed):
    gen = torch.Generator(device=_DEV).manual_seed(seed)
    rows, cin, cout = case["rows"], case["cin"], case["cout"]
    groups = -(-cin // case["group"])
    # 4-bit values of weights that were near normal; two in a byte, the even channel in the low half
    half = -(-cin // 2)
    q = torch.empty((cout, half), dtype=torch.uint8, device=_DEV)
    step = max(1, (1 << 26) // (2 * half))
    for o in range(0, cout, step):  # in pieces: the normal values take eight times the bytes
        v = torch.randn((min(step, cout - o), 2 * half), generator=gen, device=_DEV).mul_(2.6).add_(8).round_().clamp_(0, 15).to(torch.uint8)
        q[o:o + step] = v[:, 0::2] | (v[:, 1::2] << 4)
    scales = torch.randn((cout, groups), generator=gen, device=_DEV).mul_(0.3).exp_().mul_(1.0 / (2.6 * math.sqrt(cin))).to(_DTYPE[case["scale"]])
    zeros = torch.randint(5, 12, (cout, groups), generator=gen, device=_DEV, dtype=torch.uint8) if case["zeros"] else None
    bias = torch.randn((cout,), generator=gen, device=_DEV).mul_(0.1) if case["bias"] else None
    # activations: a few channels are much larger than the rest
    x = torch.randn((rows, cin), generator=gen, device=_DEV)
    x *= torch.where(torch.rand((cin,), generator=gen, device=_DEV) < 0.01, 8.0, 1.0)
    return q, scales, zeros, bias, x.to(_DTYPE[case["dtype"]])


def _logit_inputs(case, seed):
    gen = torch.Generator(device=_DEV).manual_seed(seed)
    rows, classes, dtype = case["rows"], case["classes"], _DTYPE[case["dtype"]]
    logits = torch.zeros((rows, case["pitch"]), dtype=dtype, device=_DEV)
    common = torch.randn((classes,), generator=gen, device=_DEV).mul_(1.5)  # some classes are likely everywhere
    step = max(1, (1 << 28) // classes)
    for r in range(0, rows, step):
        v = torch.randn((min(step, rows - r), classes), generator=gen, device=_DEV).mul_(2.0).add_(common)
        if case["mask"] != "none":
            low = -math.inf if case["mask"] == "inf" else torch.finfo(dtype).min
            gone = torch.rand((classes,), generator=gen, device=_DEV) < 0.3
            none_left = torch.rand((v.shape[0], 1), generator=gen, device=_DEV) < 0.05  # rows in which nothing is allowed
            v.masked_fill_(gone | none_left, low)
        logits[r:r + step, :classes] = v.to(dtype)
    given = None
    if case["given"]:
        given = torch.randint(0, classes, (rows, case["given"]), generator=gen, device=_DEV, dtype=torch.int32)
        given[torch.rand(given.shape, generator=gen, device=_DEV) < 0.1] = -1  # nothing asked here
    return logits[:, :classes], given


def prepare(case, seed):
    if case["op"] == "linear":
        q, scales, zeros, bias, x = _linear_inputs(case, seed)
        if own:  # the layer as a program keeps it
            from paper_1907_01989_b200 import api
            kind = {"f16": api.GI_F16, "bf16": api.GI_BF16, "f32": api.GI_F32}
            act = {"none": api.GI_ACT_NONE, "relu": api.GI_ACT_RELU, "relu6": api.GI_ACT_RELU6}
            layer = api.LinearQ4(q, scales, zeros=zeros, bias=bias, cin=case["cin"], group=case["group"], dtype=kind[case["dtype"]],
                                 act=act[case["act"]], device=_DEV)
            return {"case": case, "layer": layer, "x": x, "y": torch.empty((case["rows"], case["cout"]), dtype=x.dtype, device=_DEV)}
        return {"case": case, "q": q, "scales": scales, "zeros": zeros, "bias": bias, "x": x}
    logits, given = _logit_inputs(case, seed)
    state = {"case": case, "logits": logits, "given": given}
    if own:  # result buffers that a program uses again
        from paper_1907_01989_b200 import api
        state["out"] = api.log_probs_out(case["rows"], case["given"], case["top"], _DEV)
    return state


def _linear_plain(s):
    case = s["case"]
    cin, group = case["cin"], case["group"]
    q = torch.stack([s["q"] & 15, s["q"] >> 4], dim=-1).flatten(1)[:, :cin].float()
    of = torch.arange(cin, device=q.device) // group
    q -= s["zeros"].float()[:, of] if s["zeros"] is not None else 8.0
    q *= s["scales"].float()[:, of]
    y = s["x"].float() @ q.t()
    if s["bias"] is not None:
        y += s["bias"]
    if case["act"] != "none":
        y = y.clamp(min=0.0, max=6.0 if case["act"] == "relu6" else None)
    return y.to(s["x"].dtype)


def _log_probs_plain(s):
    case, given = s["case"], s["given"]
    x = s["logits"].float()
    high = x.amax(1, keepdim=True)
    empty = high == -math.inf
    d = (x - high.masked_fill(empty, 0.0)) / case["temperature"]
    e = d.exp()
    total = e.sum(1, keepdim=True)
    log_total = total.log()
    out = {}
    if given is not None:
        at = d.gather(1, given.clamp(min=0).long()) - log_total
        out["given"] = torch.where(given < 0, 0.0, at.masked_fill(empty, -math.inf))
    inner = torch.where(e > 0, e * d, 0.0).sum(1, keepdim=True)
    out["entropy"] = (log_total - inner / total).masked_fill(empty, 0.0).squeeze(1)
    if case["top"]:
        # one whole number for each logit: ordered by value, then by the lower class
        bits = (x + 0.0).view(torch.int32)
        key = (bits ^ ((bits >> 31) & 0x7fffffff)).long() << 32
        key |= 0xffffffff - torch.arange(case["classes"], device=x.device)
        best = 0xffffffff - (key.topk(case["top"], dim=1).values & 0xffffffff)
        out["top"] = (d.gather(1, best) - log_total).masked_fill(empty, -math.inf)
        out["top_ids"] = best.int()
    return out


def run(state):
    if state["case"]["op"] == "linear":
        if own:
            return state["layer"].run(state["x"], state["y"])
        return _linear_plain(state)
    if not own:
        return _log_probs_plain(state)
    from paper_1907_01989_b200 import api
    case = state["case"]
    got = api.log_probs(state["logits"], given=state["given"], top=case["top"], temperature=case["temperature"], out=state["out"])
    return {k: v for k, v in got._asdict().items() if v is not None}


def work(case):
    if case["op"] == "linear":
        rows, cin, cout = case["rows"], case["cin"], case["cout"]
        groups = -(-cin // case["group"])
        weights = cout * (-(-cin // 2)) + cout * groups * (_BYTES[case["scale"]] + (1 if case["zeros"] else 0)) + (4 * cout if case["bias"] else 0)
        return {"bytes": weights + rows * (cin + cout) * _BYTES[case["dtype"]], "flops": 2 * rows * cin * cout}
    rows, classes = case["rows"], case["classes"]
    # difference, exponential and two sums (one with a product) for each logit
    return {"bytes": rows * (classes * _BYTES[case["dtype"]] + 8 * case["given"] + 4 + 8 * case["top"]), "flops": 5 * rows * classes}


def exact(case, seed):
    """The definitions in 64 bits, summed another way: group by group, and by the probabilities themselves."""
    if case["op"] == "linear":
        q, scales, zeros, bias, x = _linear_inputs(case, seed)
        y = torch.zeros((case["rows"], case["cout"]), dtype=torch.float64, device=_DEV)
        x = x.double()
        values = torch.empty((case["cout"], 2 * q.shape[1]), dtype=torch.uint8, device=_DEV)
        values[:, 0::2], values[:, 1::2] = q % 16, q // 16
        for g in range(scales.shape[1]):
            k0, k1 = g * case["group"], min((g + 1) * case["group"], case["cin"])
            zero = zeros[:, g].double() if zeros is not None else torch.full((case["cout"],), 8.0, dtype=torch.float64, device=_DEV)
            part = x[:, k0:k1] @ values[:, k0:k1].double().t() - x[:, k0:k1].sum(1, keepdim=True) * zero
            y += part * scales[:, g].double()
        if bias is not None:
            y += bias.double()
        return torch.relu(y) if case["act"] == "relu" else torch.minimum(torch.relu(y), torch.full_like(y, 6.0)) if case["act"] == "relu6" else y
    logits, given = _logit_inputs(case, seed)
    rows, classes, top = case["rows"], case["classes"], case["top"]
    out = {"entropy": torch.empty((rows,), dtype=torch.float64, device=_DEV)}
    if given is not None:
        out["given"] = torch.empty((rows, case["given"]), dtype=torch.float64, device=_DEV)
    if top:
        out["top"] = torch.empty((rows, top), dtype=torch.float64, device=_DEV)
        out["top_ids"] = None
    step = max(1, (1 << 27) // classes)
    for r in range(0, rows, step):
        z = logits[r:r + step].double() / case["temperature"]
        some = torch.isfinite(z).any(1, keepdim=True)
        lp = torch.where(some, z - torch.logsumexp(torch.where(some, z, 0.0), 1, keepdim=True), -math.inf)
        p = lp.exp()
        out["entropy"][r:r + step] = -torch.where(p > 0, p * lp, 0.0).sum(1)
        if given is not None:
            g = given[r:r + step].long()
            out["given"][r:r + step] = torch.where(g < 0, 0.0, lp.gather(1, g.clamp(min=0)))
        if top:
            out["top"][r:r + step] = lp.topk(top, dim=1).values
    return out
