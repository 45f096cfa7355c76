"""Fully connected layers with 4-bit weights: gi_linear_q4_* against a plain form in 64 bits."""
import numpy as np
import pytest
import torch

import answer_ref as ref
from paper_1907_01989_b200 import api

GI = {torch.float16: api.GI_F16, torch.bfloat16: api.GI_BF16, torch.float32: api.GI_F32}
ACT = {"none": api.GI_ACT_NONE, "relu": api.GI_ACT_RELU, "relu6": api.GI_ACT_RELU6}


def rows_of(seed, rows, cin, dtype):
    return torch.randn((rows, cin), generator=torch.Generator().manual_seed(seed)).to(dtype)


def check(x, layer, weights, group, act="none", y=None):
    got = layer.run(x.cuda(), y)
    torch.cuda.synchronize()
    want, bound = ref.linear_q4(x, *weights, group, act)
    err = (got.double().cpu() - want).abs()
    assert got.dtype == x.dtype and torch.isfinite(got).all()
    assert (err <= bound).all(), f"worst {(err / bound).max().item():.3f} of the bound"
    return got


def make(seed, cin, cout, group, dtype, scale=torch.float16, zeros=False, bias=True, act="none", device="cuda:0"):
    weights = ref.q4_layer(seed, cin, cout, group, scale, zeros, bias)
    q, s, z, b = weights
    return api.LinearQ4(q, s, z, b, cin=cin, group=group, dtype=GI[dtype], act=ACT[act], device=device), weights


# ---------------------------------------------------------------- host
def unpack_blob(blob, cin, cout, group, sb, zeros):
    """q, scale bytes, zero points and bias out of a packed blob: the layout that the kernel's comment states, restated.  sb: bytes
    of a scale."""
    nb, nu, ng = -(-cout // 16), -(-cin // 128), -(-cin // group)
    parts = 1 if group % 128 == 0 else 2 if group % 64 == 0 else 4
    zat = 1024 + parts * 16 * sb
    record = -(-(zat + (parts * 16 if zeros else 0)) // 32) * 32
    recs = blob[:nb * nu * record].reshape(nb, nu, record)
    words = np.ascontiguousarray(recs[..., :1024]).view(np.uint32).reshape(nb, nu, 2, 8, 4, 4)  # block, unit, half, g, t, word
    q = np.zeros((nb, 2, 8, nu, 128), dtype=np.uint8)
    for half in range(2):
        for s in range(4):
            for nib in range(8):
                row, off = nib % 2, 2 * (nib % 4 // 2) + nib // 4  # row g or g + 8; channel within four
                v = (words[:, :, half, :, :, s] >> (4 * nib)) & 15
                for t in range(4):
                    k = 64 * half + 32 * (s // 2) + 8 * t + 4 * (s % 2) + off
                    q[:, row, :, :, k] = v[..., t].transpose(0, 2, 1)
    sc, z = np.zeros((nb * 16, ng, sb), dtype=np.uint8), np.zeros((nb * 16, ng), dtype=np.uint8)
    for u in range(nu):
        for h in range(parts):
            gr = (u * 128 + h * (128 // parts)) // group
            if gr >= ng:
                continue
            at = 1024 + h * 16 * sb
            sc.reshape(nb, 2, 8, ng, sb)[:, :, :, gr] = recs[:, u, at:at + 16 * sb].reshape(nb, 8, 2, sb).transpose(0, 2, 1, 3)
            if zeros:
                z.reshape(nb, 2, 8, ng)[:, :, :, gr] = recs[:, u, zat + h * 16:zat + h * 16 + 16].reshape(nb, 8, 2).transpose(0, 2, 1)
    at = -(-nb * nu * record // 256) * 256
    bias = blob[at:at + nb * 64].view(np.float32)[:cout]
    return q.reshape(nb * 16, nu * 128)[:cout, :cin], sc[:cout], z[:cout], bias


@pytest.mark.parametrize("cin,cout,group,scale,zeros", [(64, 16, 32, torch.float16, False), (1, 1, 32, torch.float32, True), (97, 33, 32, torch.float16, True),
                                                        (1280, 41, 96, torch.bfloat16, True), (200, 17, 256, torch.float32, False)])
def test_pack_keeps_every_value_in_its_place(cin, cout, group, scale, zeros):
    layer, (q, s, z, b) = make(3, cin, cout, group, torch.float16, scale, zeros, device="cpu")
    sb = s.element_size()
    if scale == torch.bfloat16:  # kept in 32 bits beside rows of fp16
        s, sb = s.float(), 4
    got_q, got_s, got_z, got_b = unpack_blob(layer.blob.numpy(), cin, cout, group, sb, zeros)
    assert np.array_equal(got_q, torch.stack([q & 15, q >> 4], -1).flatten(1)[:, :cin].numpy())
    assert np.array_equal(got_s, s.view(torch.uint8).reshape(cout, -1, sb).numpy())
    assert not zeros or np.array_equal(got_z, z.numpy())
    assert np.array_equal(got_b, b.numpy())


def test_refusals_of_a_layer():
    import ctypes as C
    L, n = api.lib(), C.c_uint64(0)

    def status(**kw):
        d = dict(cin=64, cout=32, group=32, scale_dtype=api.GI_F16, has_zeros=0, dtype=api.GI_F16, act=0)
        d.update(kw)
        return L.gi_linear_q4_blob_bytes(C.byref(api.gi_linear_q4(**d)), C.byref(n))

    assert status() == api.GI_OK and n.value > 0
    for bad in (dict(cin=0), dict(cout=-1), dict(group=0), dict(scale_dtype=4), dict(dtype=0), dict(act=7), dict(has_zeros=2)):
        assert status(**bad) == api.GI_E_INVALID, bad
    for bad in (dict(group=16), dict(group=48), dict(cin=(1 << 20) + 1), dict(cout=(1 << 20) + 1)):
        assert status(**bad) == api.GI_E_UNSUPPORTED, bad
    assert L.gi_linear_q4_blob_bytes(None, C.byref(n)) == api.GI_E_INVALID
    assert L.gi_linear_q4_blob_bytes(C.byref(api.gi_linear_q4(64, 32, 32, 1, 0, 1, 0)), None) == api.GI_E_INVALID


def test_refusals_of_pack():
    q, s, z, b = ref.q4_layer(1, 64, 16, 32, zeros=True)
    z[3, 1] = 16
    with pytest.raises(api.GiError) as e:
        api.LinearQ4(q, s, z, b, cin=64, group=32, device="cpu")
    assert e.value.status == api.GI_E_INVALID and "above 15" in str(e.value)
    for kw in (dict(cin=66), dict(group=64)):
        with pytest.raises(ValueError):
            api.LinearQ4(q, s, None, b, **{"cin": 64, "group": 32, "device": "cpu", **kw})
    with pytest.raises(ValueError):
        api.LinearQ4(q, s.double(), None, b, cin=64, group=32, device="cpu")
    import ctypes as C
    d = api.gi_linear_q4(64, 16, 32, api.GI_F16, 1, api.GI_F16, 0)
    buf = torch.empty(1 << 14, dtype=torch.uint8)
    L = api.lib()
    assert L.gi_linear_q4_pack(C.byref(d), q.data_ptr(), s.data_ptr(), None, None, buf.data_ptr(), buf.numel()) == api.GI_E_INVALID  # zeros missing
    d.has_zeros = 0
    assert L.gi_linear_q4_pack(C.byref(d), q.data_ptr(), s.data_ptr(), None, None, buf.data_ptr(), 100) == api.GI_E_INVALID  # too small
    assert L.gi_linear_q4_pack(C.byref(d), None, s.data_ptr(), None, None, buf.data_ptr(), buf.numel()) == api.GI_E_INVALID


def test_refusals_of_run_before_any_launch():
    """Checked on the host: nothing here reaches a device."""
    import ctypes as C
    L = api.lib()
    d = api.gi_linear_q4(64, 32, 32, api.GI_F16, 0, api.GI_F16, 0)
    blob, x, y = 0x100000, 0x200000, 0x300000

    def run(blob=blob, x=x, ldx=64, y=y, ldy=32, rows=4):
        return L.gi_linear_q4_run(C.byref(d), blob, x, ldx, y, ldy, rows, None)

    assert run(rows=0) == api.GI_OK  # no rows: nothing to do
    assert run(rows=(1 << 30) + 1) == api.GI_E_UNSUPPORTED
    for bad in (dict(rows=-1), dict(blob=None), dict(x=None), dict(y=None), dict(blob=blob + 128), dict(x=x + 1), dict(y=y + 1), dict(ldx=63),
                dict(ldy=31), dict(ldx=(1 << 30) + 1), dict(y=x), dict(y=x + 64 * 2 * 3), dict(x=y + 32 * 2 * 3)):
        assert run(**bad) == api.GI_E_INVALID, bad


# ---------------------------------------------------------------- GPU
@pytest.mark.gpu
@pytest.mark.parametrize("cin,cout,group", [(1, 1, 32), (97, 33, 32), (1280, 1001, 96), (515, 40, 64), (4096, 300, 128), (200, 17, 1 << 30)])
@pytest.mark.parametrize("scale", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("zeros,bias", [(False, True), (True, False)])
def test_packed_on_the_device_byte_for_byte(cin, cout, group, scale, zeros, bias):
    for dtype in (torch.float16, torch.bfloat16):
        q, s, z, b = ref.q4_layer(cin, cin, cout, group, scale, zeros, bias)
        s[0] = 0
        if scale == torch.float32:
            s[cout // 2] *= 2.0 ** 140
            s[cout - 1] *= 2.0 ** -130
        kw = dict(cin=cin, group=group, dtype=GI[dtype])
        host = api.LinearQ4(q, s, z, b, **kw)
        dev = api.LinearQ4(q.cuda(), s.cuda(), None if z is None else z.cuda(), None if b is None else b.cuda(), **kw)
        assert dev.blob.device.type == "cuda" and torch.equal(host.blob.cpu(), dev.blob.cpu())


@pytest.mark.gpu
def test_refusals_of_packing_on_the_device():
    q, s, z, b = (t.cuda() for t in ref.q4_layer(1, 64, 16, 32, zeros=True))
    z[0, 0] = 16
    with pytest.raises(ValueError):
        api.LinearQ4(q, s, z, b, cin=64, group=32)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows", [1, 2, 3, 5, 8, 9, 16, 17, 31, 40, 130])
def test_rows(rows, dtype):
    layer, w = make(rows, 320, 200, 64, dtype)
    check(rows_of(rows, rows, 320, dtype), layer, w, 64)


@pytest.mark.gpu
@pytest.mark.parametrize("cin,cout", [(1, 1), (2, 3), (31, 16), (33, 17), (63, 15), (64, 128), (65, 129), (1000, 1001), (1280, 1001), (4099, 70), (9000, 40), (130, 5000)])
@pytest.mark.parametrize("dtype,rows", [(torch.float16, 1), (torch.bfloat16, 7), (torch.float32, 4), (torch.float16, 33)])
def test_sizes(cin, cout, dtype, rows):
    layer, w = make(cin + cout, cin, cout, 32, dtype, zeros=True)
    check(rows_of(7, rows, cin, dtype), layer, w, 32)


@pytest.mark.gpu
@pytest.mark.parametrize("group", [32, 64, 96, 128, 160, 1024, 1 << 30])
@pytest.mark.parametrize("scale", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("zeros", [False, True])
def test_groups_scales_and_zero_points(group, scale, zeros):
    for dtype, rows in ((torch.float16, 2), (torch.bfloat16, 12), (torch.float32, 1), (torch.bfloat16, 70)):
        layer, w = make(group % 1000, 710, 50, group, dtype, scale, zeros)
        check(rows_of(1, rows, 710, dtype), layer, w, group)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows", [17, 32, 33, 64, 100, 128, 250, 256, 257, 300, 513, 1000])
@pytest.mark.parametrize("cin", [1096, 1097, 1098])
def test_many_rows(rows, dtype, cin):
    """Rows in whole 16-byte units, in single elements, in 32-bit words."""
    layer, w = make(rows, cin, 300, 32, dtype, zeros=True)
    check(rows_of(rows, rows, cin, dtype), layer, w, 32)


@pytest.mark.gpu
@pytest.mark.parametrize("cin,cout", [(8, 1), (64, 128), (72, 129), (1000, 1001), (1288, 2000), (8192, 130), (4104, 4096)])
@pytest.mark.parametrize("dtype,rows,scale", [(torch.float16, 20, torch.float16), (torch.bfloat16, 70, torch.float32), (torch.float16, 260, torch.bfloat16)])
def test_many_rows_sizes(cin, cout, dtype, rows, scale):
    layer, w = make(cin + cout, cin, cout, 64, dtype, scale, zeros=cin > 1000)
    check(rows_of(7, rows, cin, dtype), layer, w, 64)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_scales_outside_fp16(dtype):
    """Scales of 2^-60 and 2^40, side by side in one layer: weights that fp16 cannot hold."""
    q, s, z, b = ref.q4_layer(2, 256, 40, 64, torch.float32, bias=False)
    s = s * torch.where(torch.arange(40) % 2 == 0, 2.0 ** -60, 2.0 ** 40)[:, None]
    layer = api.LinearQ4(q, s, cin=256, group=64, dtype=GI[dtype])
    for rows in (4, 50):
        x = rows_of(rows, rows, 256, dtype)
        x = x * 2.0 ** -40 if dtype == torch.bfloat16 else x * 2.0 ** -14
        got = layer.run(x.cuda())
        want, bound = ref.linear_q4(x, q, s, None, None, 64)
        keep = want.abs() < 6e4 if dtype == torch.float16 else want.abs() < 1e38
        assert ((got.double().cpu() - want).abs() <= bound)[keep].all()


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["none", "relu", "relu6"])
@pytest.mark.parametrize("bias", [False, True])
def test_epilogue(act, bias):
    layer, w = make(5, 256, 96, 128, torch.float16, bias=bias, act=act)
    x = rows_of(2, 6, 256, torch.float16) * 20
    got = check(x, layer, w, 128, act)
    assert act == "none" or (got == 0).any()
    assert act != "relu6" or got.max() <= 6


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("off", [0, 1, 3])
@pytest.mark.parametrize("rows", [3, 40])
def test_rows_inside_wider_tensors(dtype, off, rows):
    """Any pitch and any alignment of the elements; what lies beside the rows is neither used nor written."""
    cin, cout = 200, 77
    layer, w = make(9, cin, cout, 64, dtype)
    x = rows_of(3, rows, cin, dtype)
    wide = torch.full((rows, cin + 13), float("nan"), dtype=dtype, device="cuda")
    wide[:, off:off + cin] = x.cuda()
    out = torch.full((rows + 1, cout + 9), 123.0, dtype=dtype, device="cuda")
    y = out[:rows, off:off + cout]
    got = layer.run(wide[:, off:off + cin], y)
    assert got.data_ptr() == y.data_ptr()
    want, bound = ref.linear_q4(x, *w, 64)
    assert ((y.double().cpu() - want).abs() <= bound).all()
    out[:rows, off:off + cout] = 123.0
    assert (out == 123.0).all()


@pytest.mark.gpu
def test_32_bit_rows_count_with_all_their_digits():
    """x = 1 + 2^-23 against x = 1: the difference of the results is that of the inputs, times the weights."""
    cin, cout = 64, 16
    q = torch.full((cout, cin // 2), 0x99, dtype=torch.uint8)  # q = 9: weights of one scale
    layer = api.LinearQ4(q, torch.ones((cout, 1)), cin=cin, group=64, dtype=api.GI_F32)
    x = torch.zeros((3, cin), device="cuda")
    x[0, 5], x[1, 5], x[2, 5] = 1.0, 1.0 + 2.0 ** -23, 2.0 ** -100 * (1 + 2.0 ** -23)
    y = layer.run(x).double().cpu()
    assert (y[0] == 1.0).all() and (y[1] == 1.0 + 2.0 ** -23).all()
    assert (y[2] == 2.0 ** -100 * (1 + 2.0 ** -23)).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows", [4, 40])
def test_infinity_and_nan_stay_in_their_row(dtype, rows):
    layer, w = make(4, 128, 48, 32, dtype)
    x = rows_of(4, rows, 128, dtype)
    clean = layer.run(x.cuda())
    x[1, 17], x[2, 99] = float("inf"), float("nan")
    got = layer.run(x.cuda())
    keep = [r for r in range(rows) if r not in (1, 2)]
    assert torch.equal(got[keep], clean[keep])
    assert not torch.isfinite(got[1]).any() and torch.isnan(got[2]).all()


@pytest.mark.gpu
def test_no_rows_and_leading_axes():
    layer, w = make(6, 96, 40, 32, torch.float16)
    assert layer.run(torch.empty((0, 96), dtype=torch.float16, device="cuda")).shape == (0, 40)
    x = rows_of(6, 12, 96, torch.float16)
    got = layer.run(x.view(2, 2, 3, 96).cuda())
    assert got.shape == (2, 2, 3, 40) and torch.equal(got.view(12, 40), layer.run(x.cuda()))
    one = layer.run(x[0].cuda())
    want, bound = ref.linear_q4(x[:1], *w, 32)
    assert one.shape == (40,) and ((one.double().cpu() - want[0]).abs() <= bound[0]).all()


@pytest.mark.gpu
def test_refusals_of_the_binding():
    layer, _ = make(6, 96, 40, 32, torch.float16)
    x = torch.zeros((4, 96), dtype=torch.float16, device="cuda")
    for bad in (x.float(), x[:, :95], x.cpu(), torch.zeros((96, 4), dtype=torch.float16, device="cuda").t(), x.view(2, 2, 96)[:, :, ::2]):
        with pytest.raises(ValueError):
            layer.run(bad)
    with pytest.raises(ValueError):
        layer.run(x, torch.empty((3, 40), dtype=torch.float16, device="cuda"))
    with pytest.raises(api.GiError):
        layer.run(x, x.view(-1)[:160].view(4, 40))  # y on x
    with pytest.raises(api.GiError):
        layer.run(x[:1].expand(4, 96))  # rows at distance 0


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [1, 20, 100])
def test_same_bits_every_time_on_streams_and_in_graphs(rows):
    layer, w = make(8, 1024, 500, 128, torch.float16)
    x = rows_of(8, rows, 1024, torch.float16).cuda()
    want = layer.run(x)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = []
    for i in range(9):
        with torch.cuda.stream(streams[i % 3]):
            outs.append(layer.run(x))
    explicit = torch.empty_like(want)
    layer.run(x, explicit, stream=streams[0])
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs + [explicit])
    y, y2 = torch.zeros_like(want), torch.zeros_like(want)
    graphs = []
    for out in (y, y2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            layer.run(x, out)
        graphs.append(g)
    x.mul_(2)  # exact in fp16 here: a replay reads what is there now
    with torch.cuda.stream(streams[1]):
        graphs[1].replay()
    graphs[0].replay()
    torch.cuda.synchronize()
    again = layer.run(x)
    assert torch.equal(y, again) and torch.equal(y2, again) and not torch.equal(again, want)


@pytest.mark.gpu
def test_a_blob_written_just_before_the_call_is_the_one_used():
    """The kernel may start before its predecessor has ended: it must not have read the weights by then."""
    a, w = make(10, 2048, 512, 64, torch.float16)
    b, _ = make(11, 2048, 512, 64, torch.float16)
    x = rows_of(10, 1, 2048, torch.float16).cuda()
    ya, yb = a.run(x), b.run(x)
    torch.cuda.synchronize()
    keep = a.blob.clone()
    flip = keep ^ b.blob
    for i in range(20):
        y0 = a.run(x)
        a.blob.bitwise_xor_(flip)  # a kernel of torch turns one layer into the other
        y1 = a.run(x)
        a.blob.bitwise_xor_(flip)
        assert torch.equal(y0, ya) and torch.equal(y1, yb), i


@pytest.mark.gpu
@pytest.mark.parametrize("rows,pitch,dtype", [(3, 1 << 30, torch.float16), (20, (1 << 27) + 8, torch.bfloat16), (20, (1 << 27) + 3, torch.float16), (2, 1 << 30, torch.float32)])
def test_rows_far_beyond_32_bits(rows, pitch, dtype):
    """Row offsets of more than 2^32 bytes, in x and in y."""
    layer, w = make(1, 192, 40, 64, dtype)
    x = rows_of(2, rows, 192, dtype)
    wide = torch.as_strided(torch.empty((rows - 1) * pitch + 192, dtype=dtype, device="cuda"), (rows, 192), (pitch, 1))
    wide.copy_(x)
    check_near = ref.linear_q4(x, *w, 64)
    got = layer.run(wide)
    assert ((got.double().cpu() - check_near[0]).abs() <= check_near[1]).all()
    del wide
    far = torch.as_strided(torch.empty((rows - 1) * pitch + 40, dtype=dtype, device="cuda"), (rows, 40), (pitch, 1))
    layer.run(x.cuda(), far)
    assert torch.equal(far, layer.run(x.cuda()))


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [3, 16, 40])
@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_x_and_y_side_by_side_in_one_buffer(rows, dtype):
    """Columns of one tensor: the rows of x and y lie between one another, no element is in both."""
    cin, cout = 200, 77
    layer, w = make(9, cin, cout, 64, dtype)
    x = rows_of(3, rows, cin, dtype)
    want, bound = ref.linear_q4(x, *w, 64)
    for x_at, y_at in ((0, cin), (cout, 0), (3, cin + 5), (cout + 5, 2)):
        pitch = max(x_at + cin, y_at + cout) + 1
        both = torch.full((rows, pitch), 5.0, dtype=dtype, device="cuda")
        both[:, x_at:x_at + cin] = x.cuda()
        y = layer.run(both[:, x_at:x_at + cin], both[:, y_at:y_at + cout])
        assert ((y.double().cpu() - want).abs() <= bound).all()
        assert torch.equal(both[:, x_at:x_at + cin].cpu(), x)
        for at in (cin - 1, -(cout - 1)):  # one column in both
            at += x_at
            if 0 <= at and at + cout <= pitch:
                with pytest.raises(api.GiError):
                    layer.run(both[:, x_at:x_at + cin], both[:, at:at + cout])


@pytest.mark.gpu
def test_results_belong_to_the_stream_whose_handle_was_given():
    """Memory of a result that is dropped goes to no other stream: its own may still be writing it."""
    layer, _ = make(6, 256, 4096, 32, torch.float16)
    x = torch.zeros((512, 256), dtype=torch.float16, device="cuda")
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        torch.cuda.synchronize()
        y = layer.run(x, stream=stream)
        at = y.data_ptr()
        del y
        assert torch.empty((512, 4096), dtype=torch.float16, device="cuda").data_ptr() != at
        torch.cuda.synchronize()
        logits = torch.zeros((300000, 2), dtype=torch.float16, device="cuda")
        torch.cuda.synchronize()
        got = api.log_probs(logits, stream=stream)
        at = got.entropy.data_ptr()
        del got
        assert torch.empty((300000,), device="cuda").data_ptr() != at
    torch.cuda.synchronize()
    y = layer.run(x, stream=0)  # the default stream by its handle
    torch.cuda.synchronize()
    assert torch.equal(y, layer.run(x))


# ---------------------------------------------------------------- more than 16 rows of a 16-bit type: weights in two parts
def two_part_bound(x, weights, group, act="none"):
    """(y, bound): ref.linear_q4's for weights that are not rounded (its form for up to 16 rows), and what two parts of x's type leave out
    of a weight.  scale * (q - zero), with a scale in the type's digits D (8 or 11) and 4 digits of q - zero, has D + 4 of the 2 D + 1
    digits of two parts: nothing is left out.  A scale in 32 bits is taken as two parts: off by 2^-2D of itself at most (half a step of the
    second part, which is 2^-D of the first at most); its second part's product with q - zero and the second part of the weight are
    rounded, each by 2^-D of at most 2^-D of the weight: 2^-2D for both together, and as much again for their sum.  So 4 2^-2D at most.
    fp16: what lies below its smallest step 2^-24, where the output's largest scale is 2^11 or more: of two parts of a scale half a step,
    15 times, of the weight's parts at most 2 steps: 17 steps or 2^-31 of that scale."""
    q, s, z, _ = weights
    parts = [ref.linear_q4(x[r:r + 16], *weights, group, act) for r in range(0, x.shape[0], 16)]
    y, bound = torch.cat([p[0] for p in parts]), torch.cat([p[1] for p in parts])
    digits = 8 if x.dtype == torch.bfloat16 else 11
    more = 0.0
    if s.dtype == torch.float32:
        more = 4 * 2.0 ** (-2 * digits) * (x.double().abs() @ ref.q4_weights(q, s, z, x.shape[1], group).abs().t())
    if x.dtype == torch.float16:
        more = more + 2.0 ** -31 * x.double().abs().sum(1, keepdim=True) * s.double().abs().amax(1)
    return y, bound + 1.01 * more


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows", [16, 17, 40, 130, 300])
@pytest.mark.parametrize("scale", [torch.float16, torch.float32])
def test_scales_of_one_output_far_apart(dtype, rows, scale):
    """A group of large scales, which x passes over, beside groups of scales 2^25 times smaller."""
    q, s, z, b = ref.q4_layer(2, 640, 150, 128, scale, zeros=True, bias=False)
    s = (s.float() * 0.1).to(scale)
    s[:, 1] = 30000.0
    s[::2, 3] = 1e-3
    layer = api.LinearQ4(q, s, z, cin=640, group=128, dtype=GI[dtype])
    x = rows_of(rows, rows, 640, dtype)
    x[:, 128:256] = 0
    got = layer.run(x.cuda()).double().cpu()
    want, bound = two_part_bound(x, (q, s, z, None), 128)
    assert ((got - want).abs() <= bound).all(), ((got - want).abs() / bound).max()


@pytest.mark.gpu
@pytest.mark.parametrize("group", [32, 64, 96, 128, 160, 1024, 1 << 30])
@pytest.mark.parametrize("dtype,scale", [(torch.float16, torch.float16), (torch.float16, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float16),
                                         (torch.bfloat16, torch.float32)])
@pytest.mark.parametrize("zeros", [False, True])
def test_many_rows_keep_the_digits_of_weights(group, dtype, scale, zeros):
    """One-hot rows: y is a weight itself, rounded once; and sums of 700 products."""
    cin, cout = 700, 140
    layer, w = make(group % 1000, cin, cout, group, dtype, scale, zeros, bias=False)
    q, s, z, _ = w
    hot = torch.zeros((cin, cin), dtype=dtype)
    hot[torch.arange(cin), torch.arange(cin)] = 1.0
    got = layer.run(hot.cuda()).cpu()
    values = ref.q4_weights(q, s, z, cin, group).t()
    if scale == torch.float32:
        assert ((got.double() - values).abs() <= values.abs() * (ref.UNIT[dtype] + 4.1 * 2.0 ** (-16 if dtype == torch.bfloat16 else -22))).all()
    else:
        assert torch.equal(got, values.float().to(dtype))
    for rows in (17, 33, 129, 256, 400):
        x = rows_of(rows, rows, cin, dtype)
        got = layer.run(x.cuda()).double().cpu()
        want, bound = two_part_bound(x, w, group)
        assert ((got - want).abs() <= bound).all(), (rows, ((got - want).abs() / bound).max())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("cin,cout", [(256, 300), (4096, 40)])
def test_an_infinity_in_many_rows_gives_what_it_gives_in_few(dtype, cin, cout):
    q, s, z, b = ref.q4_layer(4, cin, cout, 64, torch.float32)
    layer = api.LinearQ4(q, s, z, b, cin=cin, group=64, dtype=GI[dtype])
    x = rows_of(4, 40, cin, dtype)
    x[3, 17], x[30, cin - 1], x[9, 0] = float("inf"), -float("inf"), float("nan")
    got = layer.run(x.cuda()).cpu()
    few = torch.cat([layer.run(x[r:r + 8].cuda()) for r in range(0, 40, 8)]).cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(few)) and torch.equal(torch.isinf(got), torch.isinf(few))
    there = torch.isinf(few)
    assert there.any() and torch.equal(got[there], few[there])


@pytest.mark.gpu
def test_a_layer_whose_rows_fill_shared_memory_to_the_last_byte():
    """One row of 64000 channels to 33168 outputs: what is staged of x, the rings and the sums end at a CTA's limit."""
    cin, cout, group = 64000, 33168, 128
    g = torch.Generator(device="cuda").manual_seed(1)
    q = torch.randint(0, 256, (cout, cin // 2), dtype=torch.uint8, device="cuda", generator=g)
    s = torch.rand((cout, cin // group), device="cuda", generator=g).add_(0.5).half()
    layer = api.LinearQ4(q, s, cin=cin, group=group)
    x = torch.zeros((1, cin), dtype=torch.float16, device="cuda")
    want = torch.zeros((cout,), dtype=torch.float64, device="cuda")
    for k, v in ((0, 1.0), (127, -2.0), (31999, 0.5), (32000, 3.0), (51235, 1.5), (63999, -1.0)):
        x[0, k] = v
        want += v * ((q[:, k // 2] >> (4 * (k % 2)) & 15).double() - 8) * s[:, k // group].double()
    got = layer.run(x)[0].double()
    # six products, a rounding of each sum in fp32; half a step of the result
    assert ((got - want).abs() <= want.abs() * 2.0 ** -11 + 6 * 6 * 8 * 1.5 * 3 * 2.0 ** -23).all()


def test_a_layer_in_host_memory_is_not_run():
    """It can be packed there (and copied elsewhere); a launch would read host pointers."""
    layer, _ = make(6, 96, 40, 32, torch.float16, device="cpu")
    x = torch.zeros((4, 96), dtype=torch.float16)
    for stream in (None, 0):
        with pytest.raises(ValueError, match="CUDA"):
            layer.run(x, torch.empty((4, 40), dtype=torch.float16), stream=stream)
        with pytest.raises(ValueError, match="CUDA"):
            layer.run(x, stream=stream)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,scale,group,zeros", [(torch.float16, torch.float32, 32, True), (torch.bfloat16, torch.float32, 32, True), (torch.float16, torch.float16, 128, False),
                                                     (torch.bfloat16, torch.bfloat16, 64, True), (torch.bfloat16, torch.float32, 128, False)])
@pytest.mark.parametrize("rows,cin", [(256, 304), (256, 515), (600, 72), (129, 640)])
def test_tiles_of_256_rows(dtype, scale, group, zeros, rows, cin):
    """Outputs enough for every SM: the largest tiles, whose stages are the fewest."""
    cout = 9700
    layer, w = make(cin, cin, cout, group, dtype, scale, zeros)
    x = rows_of(rows, rows, cin, dtype)
    got = layer.run(x.cuda()).double().cpu()
    want, bound = two_part_bound(x, w, group)
    assert ((got - want).abs() <= bound).all(), ((got - want).abs() / bound).max()
    assert api.gi_device_status() == 0
