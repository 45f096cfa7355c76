"""4-bit weights inside a graph, and a network's answers: graph -> logits -> log probabilities, as they are used together."""
import ctypes as C

import numpy as np
import pytest

from paper_1907_01989_b200 import api
from paper_1907_01989_b200 import workloads as wl


def q4_graph(batch, H, W, cin, cout, group=32, zeros=False, relu=None, residual=False, scale_dtype=np.float16, follow=False):
    """input -> 1x1 conv with 4-bit weights (+ residual input) (+ activation) (-> fp16 1x1 conv)."""
    b = wl.GraphBuilder("q4", batch, 900 + cin + cout)
    x = b.input(H, W, cin)
    other = b.input(H, W, cout) if residual else None
    y = b.conv2d(x, cout, 1, 1)
    if residual:
        y = b.add(y, other)
    if relu:
        y = b.activation(y, relu)
    if follow:
        y = b.conv2d(y, 24, 1, 1)
    b.output(y)
    spec = b.g
    op = spec.ops[0]
    op.q4 = wl.quantize_q4(op.weights, group, zeros, scale_dtype)
    op.weights = op.q4.values(cin)
    return spec


# ---------------------------------------------------------------- host
@pytest.mark.parametrize("cin,group,zeros", [(64, 32, False), (33, 32, True), (200, 96, True), (1280, 1280, False)])
def test_quantize_is_within_half_a_step(cin, group, zeros):
    w = np.random.default_rng(cin).standard_normal((11, cin)).astype(np.float32)
    w[3] = 0
    q = wl.quantize_q4(w, group, zeros, np.float32)
    got = q.values(cin).reshape(w.shape)
    step = q.scales[:, np.arange(cin) // group]
    # half a step, and where the zero point was rounded half a step more; a hair for the roundings of fp32
    assert (np.abs(got - w) <= step * (1.0 if zeros else 0.5) * (1 + 1e-5)).all()
    assert (got[3] == 0).all()


def test_compile_chooses_the_4_bit_kernel_for_few_pixels():
    for batch, H, W, want in ((1, 1, 1, True), (4, 1, 1, True), (5, 1, 1, False), (1, 2, 4, True), (1, 7, 1, True), (1, 3, 3, False)):
        ex = api.graph_from_spec(q4_graph(batch, H, W, 320, 40), api.GI_F16)[0].compile()
        assert ("linear_q4" in [api.KERNEL_NAMES[x.kernel] for x in ex.launches()]) is want, (batch, H, W)
    spec = q4_graph(1, 1, 1, 1280, 1001)
    ex = api.graph_from_spec(spec, api.GI_F16)[0].compile()
    plain = q4_graph(1, 1, 1, 1280, 1001)
    plain.ops[0].q4 = None
    assert ex.info.weight_bytes < api.graph_from_spec(plain, api.GI_F16)[0].compile().info.weight_bytes / 3
    for kw in (dict(pointwise=api.GI_PW_SIMT), dict(pointwise=api.GI_PW_RULE)):
        assert "linear_q4" not in [api.KERNEL_NAMES[x.kernel] for x in api.graph_from_spec(spec, api.GI_F16)[0].compile(**kw).launches()]
    assert "linear_q4" not in [api.KERNEL_NAMES[x.kernel] for x in api.graph_from_spec(spec, api.GI_F32)[0].compile().launches()]


def test_refusals_of_4_bit_weights():
    q, s = np.zeros((8, 16), np.uint8), np.ones((8, 1), np.float16)

    def status(kind=api.GI_OP_CONV2D, k=1, q=q.ctypes.data, s=s.ctypes.data, zeros=None, scale=api.GI_F16, group=32):
        g = api.Graph(1, api.GI_F16)
        d = api.gi_op_desc()
        w = api.gi_q4_weights(q, s, zeros, scale, group)
        d.kind, d.kh, d.kw, d.stride_h, d.stride_w, d.dilation_h, d.dilation_w, d.cout = kind, k, k, 1, 1, 1, 1, 8
        d.inputs[0], d.inputs[1] = g.input(4, 4, 32), -1
        d.weight_dtype, d.weights = api.GI_Q4, C.addressof(w)
        t = C.c_int32(-1)
        return api.lib().gi_add_op(g._h, C.byref(d), C.byref(t))

    z = np.full((8, 1), 16, np.uint8)
    assert status() == api.GI_OK
    for bad in (dict(q=None), dict(s=None), dict(scale=0), dict(group=0), dict(group=-32), dict(zeros=z.ctypes.data)):
        assert status(**bad) == api.GI_E_INVALID, bad
    for bad in (dict(group=16), dict(k=3), dict(kind=api.GI_OP_DEPTHWISE_CONV2D, k=3)):
        assert status(**bad) == api.GI_E_UNSUPPORTED, bad


# ---------------------------------------------------------------- GPU
@pytest.mark.gpu
@pytest.mark.parametrize("batch,H,W", [(1, 1, 1), (3, 1, 1), (4, 1, 1), (1, 7, 1), (1, 2, 4), (2, 1, 3), (1, 3, 3), (5, 7, 7)])
@pytest.mark.parametrize("cin,cout,kw", [(1280, 1001, {}), (33, 7, dict(zeros=True)), (96, 64, dict(relu=wl.ACT_RELU6, group=64, scale_dtype=np.float32)),
                                         (130, 18, dict(residual=True, relu=wl.ACT_RELU)), (64, 30, dict(follow=True, relu=wl.ACT_RELU6, residual=True))])
@pytest.mark.parametrize("planner", [api.GI_PLAN_GREEDY_BY_SIZE, api.GI_PLAN_NAIVE])
def test_graph_matches_the_oracle(batch, H, W, cin, cout, kw, planner):
    import gpu_util as gu
    from oracle import graph as og
    spec = q4_graph(batch, H, W, cin, cout, **kw)
    rng = np.random.default_rng(5)
    xs = [rng.uniform(-1, 1, (batch,) + tuple(spec.shapes[t])).astype(np.float16).astype(np.float32) for t in spec.inputs]
    run = gu.DeviceRun(spec, planner=planner, guard_bytes=4096)
    if batch * ((H * W + 1) // 2 * 2) <= 8:
        assert "linear_q4" in [api.KERNEL_NAMES[x.kernel] for x in run.ex.launches()]
    got = run.run(xs)
    ref = og.run(spec, xs, storage="f16")
    for t in spec.outputs:
        gu.assert_close(got[t], ref[t], api.GI_F16, f"tensor {t}")
    assert run.guard_intact()


@pytest.mark.gpu
@pytest.mark.parametrize("zeros", [False, True])
def test_fp32_storage_and_the_built_in_arena(zeros):
    import torch
    import gpu_util as gu
    from oracle import graph as og
    spec = q4_graph(2, 1, 1, 130, 45, zeros=zeros, relu=wl.ACT_RELU6, follow=True)
    x = np.random.default_rng(3).uniform(-1, 1, (2, 1, 1, 130)).astype(np.float16).astype(np.float32)
    got = gu.DeviceRun(spec, storage=api.GI_F32).run([x])
    gu.assert_close(got[spec.outputs[0]], og.run(spec, [x], storage="f32")[spec.outputs[0]], api.GI_F32)
    ex = api.graph_from_spec(spec, api.GI_F16)[0].compile()
    ex.bind("cuda:0")
    assert "linear_q4" in [api.KERNEL_NAMES[k.kernel] for k in ex.launches()]
    xin = torch.from_numpy(x).half().cuda()
    a, b = (torch.full((2, 1, 1, 24), float("nan"), dtype=torch.float16, device="cuda") for _ in range(2))
    ex.run([xin], [a])
    ex.arena.fill_(0xFF)
    ex.run_static([xin], [b])
    torch.cuda.synchronize()
    assert torch.equal(a, b) and torch.isfinite(a).all()
    assert len(ex.run_timed([xin], [b])) == ex.info.n_ops


@pytest.mark.gpu
@pytest.mark.parametrize("batch", [1, 4, 8, 12])
@pytest.mark.parametrize("graphs", [False, True])
def test_network_to_answers(batch, graphs):
    """MobileNetV2 with a 4-bit classifier through the host pipeline: answers of the logits that gi_run leaves."""
    import torch
    import answer_ref as ref
    import gpu_util as gu
    from oracle import graph as og
    from paper_1907_01989_b200.pipeline import HostPipeline
    spec = wl.with_q4_classifier(wl.mobilenet_v2(batch, size=96))
    ex = api.graph_from_spec(spec, api.GI_F16)[0].compile()
    assert ("linear_q4" in [api.KERNEL_NAMES[x.kernel] for x in ex.launches()]) is (batch <= 4)
    ex.bind("cuda:0")
    shape_in = (batch,) + tuple(spec.shapes[spec.inputs[0]])
    shape_out = (batch,) + tuple(spec.shapes[spec.outputs[0]])
    pipe = HostPipeline(ex, [shape_in], [shape_out], torch.float16, "cuda:0", graphs=graphs, top=5)
    assert bool(pipe.graphs) is graphs
    results = []
    for images in (range(batch), range(7, 7 + batch), range(batch)):
        x = torch.from_numpy(wl.make_input(spec, images=list(images))).half().pin_memory()
        out = [torch.empty((batch, 5)).pin_memory(), torch.empty((batch, 5), dtype=torch.int32).pin_memory(), torch.empty((batch,)).pin_memory()]
        pipe.submit([x], out)
        results.append((x, out))
    pipe.synchronize()
    y = torch.empty(shape_out, dtype=torch.float16, device="cuda:0")
    for x, (lp, ids, entropy) in results:
        ex.run([x.cuda()], [y])
        torch.cuda.synchronize()
        gu.assert_close(y.float().cpu().numpy(), og.run(spec, [x.float().numpy()], storage="f16")[spec.outputs[0]], api.GI_F16, "logits")
        want, bound = ref.log_probs(y.view(batch, -1), None, 5)
        assert torch.equal(ids, want["top_ids"])
        assert ((lp.double() - want["top"]).abs() <= bound["log"][:, None] + 2.0 ** -22 * want["top"].abs()).all()
        assert ((entropy.double() - want["entropy"]).abs() <= bound["entropy"]).all()
    assert all(torch.equal(a, b) for a, b in zip(results[0][1], results[2][1]))


@pytest.mark.gpu
def test_segmentation_to_classes_of_pixels():
    """Logits of every pixel -> its class, on the device."""
    import torch
    import answer_ref as ref
    spec = wl.mobilenet_v2_segmentation(1, size=97)
    ex = api.graph_from_spec(spec, api.GI_F16)[0].compile()
    ex.bind("cuda:0")
    x = torch.from_numpy(wl.make_input(spec)).half().cuda()
    y = torch.empty((1,) + tuple(spec.shapes[spec.outputs[0]]), dtype=torch.float16, device="cuda:0")
    ex.run([x], [y])
    got = api.log_probs(y, top=1)
    want, bound = ref.log_probs(y.view(-1, y.shape[-1]), None, 1)
    assert torch.equal(got.top_ids.cpu(), want["top_ids"])
    assert ((got.entropy.double().cpu() - want["entropy"]).abs() <= bound["entropy"]).all()


@pytest.mark.gpu
def test_many_rows_between_kernels_that_take_all_tensor_memory():
    """Each kernel may start while the one in front of it ends: a layer of many rows between 1x1 convolutions on tensor memory, over and
    over on one stream."""
    import torch
    import answer_ref as ref
    spec = wl.mobilenet_v2(32, size=96)
    ex = api.graph_from_spec(spec, api.GI_F16)[0].compile(pointwise=api.GI_PW_TC_LANE, cross_op=api.GI_XOP_OFF)
    assert "pointwise_ts" in [api.KERNEL_NAMES[x.kernel] for x in ex.launches()]
    ex.bind("cuda:0")
    x = torch.from_numpy(wl.make_input(spec)).half().cuda()
    y = torch.empty((32, 1, 1, 1001), dtype=torch.float16, device="cuda:0")
    q, s, z, b = ref.q4_layer(1, 512, 4096, 64)
    layer = api.LinearQ4(q, s, z, b, cin=512, group=64)
    rows = torch.randn((300, 512), generator=torch.Generator().manual_seed(1)).half().cuda()
    ex.run([x], [y])
    out = layer.run(rows)
    torch.cuda.synchronize()
    first, first_out = y.clone(), out.clone()
    for _ in range(30):
        layer.run(rows, out)
        ex.run([x], [y])
        layer.run(rows, out)
        layer.run(rows[:40], out[:40])
        layer.run(rows, out)
    torch.cuda.synchronize()
    assert torch.equal(y, first) and torch.equal(out, first_out)
    assert api.gi_device_status() == 0


@pytest.mark.gpu
def test_captured_behind_work_of_two_streams():
    """A capture in which both operators follow kernels of another stream as well."""
    import torch
    import answer_ref as ref
    q, s, z, b = ref.q4_layer(1, 256, 1001, 64)
    layer = api.LinearQ4(q, s, z, b, cin=256, group=64)
    a, c = (torch.randn((30, 256), generator=torch.Generator().manual_seed(i)).half().cuda() for i in (1, 2))
    x, y = torch.empty_like(a), torch.empty((30, 1001), dtype=torch.float16, device="cuda")
    out = api.log_probs_out(30, 0, 4)
    want_y = layer.run(a + c)
    want = api.log_probs(want_y, top=4)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        main = torch.cuda.current_stream()
        side.wait_stream(main)
        with torch.cuda.stream(side):
            t = a * 1
        u = c * 1
        main.wait_stream(side)
        torch.add(t, u, out=x)
        layer.run(x, y)
        side.wait_stream(main)
        with torch.cuda.stream(side):
            e = y * 1
        layer.run(x, y)
        main.wait_stream(side)
        api.log_probs(y, top=4, out=out)
    for _ in range(3):
        x.zero_()
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want_y) and torch.equal(e, want_y)
        assert all(torch.equal(p, r) for p, r in zip(out[1:], want[1:]))


@pytest.mark.gpu
def test_pipeline_refuses_buffers_that_are_not_its_answers():
    """Three buffers of the answers' shapes and types: anything else would be left out, cast or stretched without a word."""
    import torch
    from paper_1907_01989_b200.pipeline import HostPipeline
    spec = q4_graph(2, 1, 1, 64, 30)
    ex = api.graph_from_spec(spec, api.GI_F16)[0].compile()
    ex.bind("cuda:0")
    pipe = HostPipeline(ex, [(2, 1, 1, 64)], [(2, 1, 1, 30)], torch.float16, "cuda:0", top=3)
    x = torch.zeros((2, 1, 1, 64)).half().pin_memory()
    good = [torch.empty((2, 3)).pin_memory(), torch.empty((2, 3), dtype=torch.int32).pin_memory(), torch.empty((2,)).pin_memory()]
    for bad in (good[:2], good + good[:1], [good[1], good[0], good[2]], [good[0], good[1], torch.empty((2, 1)).pin_memory()],
                [torch.empty((4, 3)).pin_memory()[:2].t().contiguous().t(), torch.empty((3,), dtype=torch.int32), good[2]]):
        with pytest.raises(ValueError):
            pipe.submit([x], bad)
    pipe.submit([x], good)
    pipe.synchronize()
    assert torch.isfinite(good[0]).all() and (good[1] >= 0).all()
    with pytest.raises(ValueError):
        HostPipeline(ex, [(2, 1, 1, 64)], [(2, 1, 1, 30)], torch.float16, "cuda:0", top=31)
    with pytest.raises(ValueError):
        HostPipeline(ex, [(2, 1, 1, 64)], [(2, 1, 1, 30)], torch.float16, "cuda:0", top=33)
