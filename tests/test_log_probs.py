"""Log probabilities of classes, entropy and leading classes: gi_log_probs against a plain form in 64 bits."""
import math

import numpy as np
import pytest
import torch

import answer_ref as ref
from paper_1907_01989_b200 import api

INF = math.inf


def logits_of(seed, rows, classes, dtype, scale=3.0):
    return (torch.randn((rows, classes), generator=torch.Generator().manual_seed(seed)) * scale).to(dtype)


def check(x, given=None, top=0, temperature=1.0, dev=None, out=None):
    dev = x.cuda() if dev is None else dev
    got = api.log_probs(dev, None if given is None else given.cuda(), top, temperature, out)
    torch.cuda.synchronize()
    want, bound = ref.log_probs(x, given, top, temperature)
    if top:
        assert torch.equal(got.top_ids.cpu().view(-1, top), want["top_ids"])
    for name, v in (("given", got.given), ("top", got.top), ("entropy", got.entropy)):
        if v is None:
            continue
        w = want[name]
        v = v.double().cpu().view(w.shape)
        b = bound["entropy"] if name == "entropy" else bound["log"][:, None] + 2.0 ** -22 * w.abs()
        fine = torch.isfinite(w)
        assert torch.equal(torch.isnan(v), torch.isnan(w)) and torch.equal(v[~fine & ~torch.isnan(w)], w[~fine & ~torch.isnan(w)]), name
        err = torch.where(fine, v - w, 0.0).abs()
        assert (err <= torch.where(fine, b.expand_as(w), 1.0)).all(), f"{name}: off by {err.max().item():.3g}"
    return got


# ---------------------------------------------------------------- host
def test_refusals_before_any_launch():
    import ctypes as C
    L = api.lib()
    x, g, o = 0x10000, 0x20000, 0x30000

    def run(x=x, given=g, given_lp=o, entropy=o, ids=o, lp=o, **kw):
        d = dict(rows=4, classes=10, ld=10, dtype=api.GI_F16, temperature=1.0, n_given=1, top=2)
        d.update(kw)
        return L.gi_log_probs(C.byref(api.gi_log_probs_desc(**d)), x, given, given_lp, entropy, ids, lp, None)

    assert run(rows=0) == api.GI_OK
    for bad in (dict(rows=-1), dict(classes=0), dict(dtype=9), dict(temperature=0.0), dict(temperature=float("nan")), dict(temperature=INF), dict(temperature=-1.0),
                dict(n_given=-1), dict(top=-1), dict(top=33), dict(top=11), dict(ld=9), dict(ld=1 << 40), dict(x=None), dict(given=None), dict(given_lp=None),
                dict(ids=None), dict(lp=None), dict(x=x + 1), dict(given=g + 2), dict(lp=o + 1), dict(n_given=0, top=0, entropy=None), dict(n_given=65537)):
        assert run(**bad) == api.GI_E_INVALID, bad
    for bad in (dict(rows=(1 << 28) + 1), dict(classes=(1 << 24) + 1, ld=1 << 25)):
        assert run(**bad) == api.GI_E_UNSUPPORTED, bad
    assert L.gi_log_probs(None, x, g, o, o, o, o, None) == api.GI_E_INVALID


# ---------------------------------------------------------------- GPU
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("classes", [1, 2, 7, 8, 9, 21, 31, 64, 65, 100, 1001, 2047, 2048, 2049, 4099, 8192, 30001, 131072, 262144])
def test_classes(classes, dtype):
    rows = 5 if classes < 100000 else 2
    x = logits_of(classes, rows, classes, dtype)
    given = torch.randint(0, classes, (rows, 3), dtype=torch.int32, generator=torch.Generator().manual_seed(1))
    check(x, given, min(classes, 20))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("classes", [1, 3, 21, 64])
@pytest.mark.parametrize("pitch", [0, 5])
def test_many_rows_of_few_classes(classes, dtype, pitch):
    rows = 4096 + 77
    x = logits_of(classes, rows, classes, dtype)
    x[:, classes // 2] = -INF
    x[100] = -INF
    given = torch.randint(-1, classes + 1, (rows, 2), dtype=torch.int32, generator=torch.Generator().manual_seed(2))
    dev = torch.full((rows, classes + pitch), float("nan"), dtype=dtype, device="cuda")[:, :classes]
    dev.copy_(x)
    for top in {0, 1, min(classes, 4), classes if classes < 32 else 32}:
        check(x, given, top, 0.7, dev)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,classes", [(1, 1001), (300, 1001), (700, 5000), (2000, 2500), (148, 40000), (3, 200000), (2400, 5003), (2400, 8192)])
def test_rows(rows, classes):
    x = logits_of(rows, rows, classes, torch.float16)
    check(x, torch.zeros((rows, 1), dtype=torch.int32), 5)


@pytest.mark.gpu
@pytest.mark.parametrize("top", [0, 1, 2, 5, 31, 32])
@pytest.mark.parametrize("classes", [32, 1001, 3001, 70000])
def test_top(top, classes):
    """fp16 logits of few different values: ties everywhere."""
    x = (logits_of(top, 6, classes, torch.float32) * 0.5).round().to(torch.float16)
    x[1] = 2.0
    check(x, None, top)


@pytest.mark.gpu
@pytest.mark.parametrize("classes", [21, 1001, 2048, 5001, 100000])
@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_orders_that_defeat_a_guess(classes, dtype):
    """Rising, falling, and large elements that all belong to one thread's share (more than are collected at a time)."""
    n = torch.arange(classes, dtype=torch.float32)
    rise = n * (200.0 / classes)
    rows = [rise, rise.flip(0)]
    for period in (32 * 8, 32 * 4, 256 * 8, 256 * 4, 256 * 8 * 16):
        rows.append(torch.where(n % period < 40, 50.0 + n * (20.0 / classes), -n * (20.0 / classes)))
        rows.append(torch.where(n % period < 8, 50.0, 0.0))
    check(torch.stack(rows).to(dtype), None, min(classes, 20))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("classes", [21, 1001, 9000])
@pytest.mark.parametrize("rows", [6, 5000])
def test_masks(classes, dtype, rows):
    if rows == 5000 and classes > 1001:
        rows = 600
    x = logits_of(classes, rows, classes, dtype)
    low = torch.finfo(dtype).min
    x[0] = -INF                      # nothing left
    x[1] = low                       # the lowest value everywhere: uniform
    x[2, 1:] = -INF                  # one class left
    x[3, :] = -INF
    x[3, classes - 1] = low          # one left, of the lowest value
    x[4, ::2] = -INF
    x[5, ::3] = low
    given = torch.zeros((rows, 4), dtype=torch.int32)
    given[:, 1], given[:, 2], given[:, 3] = classes - 1, -5, classes
    got = check(x, given, 7)
    assert got.entropy[0] == 0 and got.entropy[2] == 0 and got.entropy[3] == 0
    assert abs(got.entropy[1].item() - math.log(classes)) < 1e-4
    assert got.top_ids[0].tolist() == list(range(7)) and (got.top[0] == -INF).all()


@pytest.mark.gpu
@pytest.mark.parametrize("rows,classes", [(3, 50257), (64, 60000), (400, 50257), (5, 1999), (2, 262144)])
@pytest.mark.parametrize("top", [1, 8, 32])
def test_rows_of_equal_logits(rows, classes, top):
    """Nothing left, one value everywhere, two values: every element reaches the bound, the lower classes come first."""
    x = torch.zeros((rows, classes), dtype=torch.bfloat16)
    x[0] = -INF
    x[1] = 3.0
    x[1, classes // 3::7] = 4.0
    if rows > 2:
        x[2, ::2] = -INF
    check(x, None, top)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("rows,classes", [(8, 21), (5000, 21), (8, 1001), (8, 20000)])
def test_not_a_number_and_infinity_stay_in_their_row(dtype, rows, classes):
    x = logits_of(3, rows, classes, dtype)
    given = torch.full((rows, 1), 4, dtype=torch.int32)
    clean = api.log_probs(x.cuda(), given.cuda(), 3)
    x[2, 7], x[5, 11] = float("nan"), INF
    got = api.log_probs(x.cuda(), given.cuda(), 3)
    keep = [r for r in range(rows) if r not in (2, 5)]
    for a, b in zip(clean, got):
        assert torch.equal(a[keep], b[keep])
    for r, c in ((2, 7), (5, 11)):
        assert torch.isnan(got.entropy[r]) and torch.isnan(got.given[r]).all() and torch.isnan(got.top[r]).all()
        assert got.top_ids[r, 0] == c and (got.top_ids[r] >= 0).all() and (got.top_ids[r] < classes).all()


@pytest.mark.gpu
@pytest.mark.parametrize("temperature", [1e-4, 0.3, 1.7, 100.0, 1e4])
@pytest.mark.parametrize("classes", [33, 1001, 20000])
def test_temperature(temperature, classes):
    x = logits_of(9, 40, classes, torch.float32)
    check(x, torch.full((40, 1), 3, dtype=torch.int32), 4, temperature)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,off", [(torch.float16, 1), (torch.float16, 3), (torch.bfloat16, 5), (torch.float32, 1)])
@pytest.mark.parametrize("rows,classes,pitch", [(9, 50, 57), (9, 1001, 1003), (5000, 21, 24), (4, 33333, 33340)])
def test_rows_inside_wider_tensors(dtype, off, rows, classes, pitch):
    """Any pitch and alignment; what lies beside the rows (NaN here) is not looked at."""
    x = logits_of(off, rows, classes, dtype)
    wide = torch.full((rows, pitch), float("nan"), dtype=dtype, device="cuda").view(-1)
    buf = torch.full((rows * pitch + 16,), float("nan"), dtype=dtype, device="cuda")
    dev = buf[off:off + rows * pitch].view(rows, pitch)[:, :classes]
    dev.copy_(x)
    check(x, torch.full((rows, 1), classes - 1, dtype=torch.int32), 6, 1.3, dev)
    del wide


@pytest.mark.gpu
def test_rows_far_beyond_32_bits():
    """Row offsets of more than 2^32 bytes."""
    rows, classes, pitch = 3, 1500, (1 << 30) + 8
    buf = torch.empty(2 * pitch + classes, dtype=torch.float16, device="cuda")
    dev = torch.as_strided(buf, (rows, classes), (pitch, 1))
    x = logits_of(4, rows, classes, torch.float16)
    dev.copy_(x)
    with pytest.raises(api.GiError):
        api.log_probs(dev, None, 3)  # above the largest pitch
    pitch = 1 << 30
    dev = torch.as_strided(buf, (rows, classes), (pitch, 1))
    dev.copy_(x)
    check(x, None, 3, dev=dev)


@pytest.mark.gpu
def test_many_rows_far_beyond_32_bits():
    rows, classes, pitch = 4100, 21, (1 << 20) + 5
    dev = torch.as_strided(torch.empty((rows - 1) * pitch + classes, dtype=torch.float16, device="cuda"), (rows, classes), (pitch, 1))
    x = logits_of(4, rows, classes, torch.float16)
    dev.copy_(x)
    check(x, None, 3, dev=dev)


@pytest.mark.gpu
def test_only_what_is_asked_for():
    x = logits_of(5, 12, 1001, torch.float16)
    got = check(x)
    assert got.given is None and got.top is None and got.top_ids is None and got.entropy.shape == (12,)
    out = api.log_probs_out(12, 0, 4, entropy=False)
    assert check(x, None, 4, out=out).entropy is None
    empty = api.log_probs(torch.empty((0, 10), dtype=torch.float16, device="cuda"), None, 2)
    assert empty.entropy.shape == (0,) and empty.top_ids.shape == (0, 2)
    maps = logits_of(6, 2 * 3 * 5, 21, torch.float16)
    got = api.log_probs(maps.view(2, 3, 5, 21).cuda(), None, 1)
    assert torch.equal(got.top_ids.cpu(), ref.log_probs(maps, None, 1)[0]["top_ids"])


@pytest.mark.gpu
def test_refusals_of_the_binding():
    x = torch.zeros((4, 10), dtype=torch.float16, device="cuda")
    given = torch.zeros((4, 1), dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        api.log_probs(x, given.long())
    with pytest.raises(ValueError):
        api.log_probs(x, given[:3])
    with pytest.raises(ValueError):
        api.log_probs(x, None, 2, out=api.log_probs_out(4, 0, 1))
    with pytest.raises(ValueError):
        api.log_probs(x.t())
    with pytest.raises(api.GiError):
        api.log_probs(x.double())
    with pytest.raises(api.GiError):
        api.log_probs(x, None, 11)
    with pytest.raises(api.GiError):
        api.log_probs(x[:1].expand(4, 10))


@pytest.mark.gpu
@pytest.mark.parametrize("rows,classes", [(1, 1001), (5000, 21), (2, 150000), (64, 50257)])
def test_same_bits_every_time_on_streams_and_in_graphs(rows, classes):
    x = logits_of(8, rows, classes, torch.float16).cuda()
    want = api.log_probs(x, None, 9)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = []
    for i in range(9):
        with torch.cuda.stream(streams[i % 3]):
            outs.append(api.log_probs(x, None, 9))
    torch.cuda.synchronize()
    for o in outs:
        assert all(torch.equal(a, b) for a, b in zip(o[1:], want[1:]))
    out = [api.log_probs_out(rows, 0, 9) for _ in range(2)]
    graphs = []
    for o in out:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            api.log_probs(x, None, 9, out=o)
        graphs.append(g)
    x.copy_(x.flip(1))
    with torch.cuda.stream(streams[0]):
        graphs[0].replay()
    graphs[1].replay()
    torch.cuda.synchronize()
    again = api.log_probs(x, None, 9)
    for o in out:
        assert all(torch.equal(a, b) for a, b in zip(o[1:], again[1:]))
    assert not torch.equal(again.top_ids, want.top_ids)


def order_of(x, top):
    """The leading classes: a NaN above all, of equals the lower class."""
    v = x.double().numpy()
    v = np.where(np.isnan(v), np.inf, np.where(np.isposinf(v), np.finfo(np.float64).max, v))
    return torch.from_numpy(np.lexsort((np.broadcast_to(np.arange(x.shape[1]), x.shape), -v), axis=1)[:, :top].copy()).int()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,classes", [(4096 + 130, 2), (4096 + 130, 8), (4096 + 130, 21), (4096 + 130, 33), (4096 + 130, 64),  # a thread a row
                                          (12, 8), (12, 21), (12, 1001),  # a warp a row
                                          (12, 5001), (12, 60000)])  # a CTA a row, a cluster
def test_not_a_number_leads_from_every_class(dtype, rows, classes):
    x = logits_of(classes, rows, classes, dtype)
    places = [[0], [classes // 2], [classes - 1], [0, classes - 1], list(range(classes)), [0, 1]]
    with_nan = [i * 2 for i in range(len(places))] + [rows - 1]  # the last row too: nothing lies behind it
    for r, cols in zip(with_nan, places + [[0]]):
        x[r, cols] = float("nan")
    x[1, classes - 1] = INF  # below a NaN, above all others
    x[2, 0] = INF
    for top in {2, 3, min(classes, 32)} - ({3} if classes < 3 else set()):
        got = api.log_probs(x.cuda(), None, top)
        torch.cuda.synchronize()
        assert torch.equal(got.top_ids.cpu(), order_of(x, top)), top
        assert torch.isnan(got.top[with_nan]).all() and torch.isnan(got.entropy[with_nan]).all()
        assert torch.isfinite(got.top[3:10:2]).all()


@pytest.mark.gpu
def test_calls_of_several_threads_at_once():
    """Sizes that share a kernel but not their need of shared memory, from threads of their own: none is refused, none is wrong."""
    import ctypes as C
    import threading
    run = api.lib().gi_log_probs
    results, cases = [], []
    for classes in (48, 64, 50, 63):
        x = logits_of(classes, 4096, classes, torch.float32).cuda()
        want, out, stream = api.log_probs(x, None, 1), api.log_probs_out(4096, 0, 1), torch.cuda.Stream()
        d = api.gi_log_probs_desc(4096, classes, classes, api.GI_F32, 1.0, 0, 1)
        cases.append((d, x, want, out, stream))
    torch.cuda.synchronize()

    def calls(d, x, want, out, stream):
        args = (C.byref(d), x.data_ptr(), None, None, out.entropy.data_ptr(), out.top_ids.data_ptr(), out.top.data_ptr(), stream.cuda_stream)
        results.append(sum(run(*args) != api.GI_OK for _ in range(20000)))
    threads = [threading.Thread(target=calls, args=c) for c in cases]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert results == [0] * len(cases)
    for _, _, want, out, _ in cases:
        assert all(torch.equal(a, b) for a, b in zip(out[1:], want[1:]))


@pytest.mark.gpu
def test_buffers_for_more_than_is_asked_for():
    """What was not asked for is None, not what an earlier call left in its buffer."""
    x = logits_of(5, 12, 1001, torch.float16).cuda()
    given = torch.zeros((12, 2), dtype=torch.int32, device="cuda")
    out = api.log_probs_out(12, 2, 4)
    full = api.log_probs(x, given, 4, out=out)
    assert all(a is b for a, b in zip(full, out))
    got = api.log_probs(x, None, 4, out=out)
    assert got.given is None and got.top is out.top and got.top_ids is out.top_ids and got.entropy is out.entropy
    got = api.log_probs(x, given, out=out)
    assert got.given is out.given and got.top is None and got.top_ids is None


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,classes", [(4100, 21), (9, 1001), (3, 70000)])
def test_logits_whose_difference_is_beyond_fp32(dtype, rows, classes):
    """The largest and the lowest logit are 6e38 apart: divided by a temperature that is a number again."""
    x = torch.full((rows, classes), -3e38).to(dtype)
    x[:, 3], x[:, 5], x[1, 7] = 3e38, 1e38, -INF
    given = torch.tensor([[0, 5, 7, 3]], dtype=torch.int32).repeat(rows, 1)
    for temperature in (3.0, 1000.0):
        got = check(x, given, 4, temperature)
        assert torch.isfinite(got.top).all()
    got = api.log_probs(x.cuda(), given.cuda(), 4, 1.0)  # here it is not
    assert (got.given[:, 0] == -INF).all() and (got.given[:, 3] == 0).all()


@pytest.mark.gpu
def test_logits_without_classes_are_refused():
    for shape in ((), (0,), (4, 0), (2, 2, 0)):
        with pytest.raises((ValueError, api.GiError)):
            api.log_probs(torch.zeros(shape, dtype=torch.float16, device="cuda"))
