"""The operators together as a student with a frozen and a trained half uses them: planar features are quantised, a frozen layer multiplies them in 8 bits,
a trained layer behind it is stepped by st_adamw on the gradients that autograd gives, new buffers each step; its weights are then quantised in turn.
And the context's own Adam against st_adamw on the same gradients."""
import numpy as np
import pytest

import synth_inputs as si
import paper_2003_10735_b200 as st
from test_gpu_adamw import Ref, f64, put, U

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(autouse=True)
def side_stream():
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        yield s
    s.synchronize()


def quantized(x, stream):
    rows, cols = x.shape
    q, s = torch.zeros(rows, -(-cols // 16) * 16, dtype=torch.int8, device="cuda")[:, :cols], torch.zeros(rows, device="cuda")
    st.st_quantize_rows(x, q, s, cuda_stream=stream)
    return q, s


@pytest.mark.parametrize("bits", [32, 8])
def test_a_frozen_layer_in_8_bits_and_a_trained_one(bits, side_stream):
    stream = side_stream.cuda_stream
    torch.manual_seed(1)
    k, c, classes, h, w = 200, 96, 7, 19, 23
    planes = torch.randn(k, h, w, device="cuda").relu()
    weight, bias = torch.randn(c, k, device="cuda"), torch.randn(c, device="cuda")
    labels = torch.randint(0, classes, (h * w,), device="cuda")
    xq, xs = quantized(planes.view(k, -1).t(), stream)
    wq, ws = quantized(weight, stream)
    tokens = torch.zeros(h * w, c, device="cuda")
    st.st_int8_matmul(xq, xs, wq, ws, tokens, bias=bias, relu=True, cuda_stream=stream)

    params = [torch.randn(classes, c, device="cuda") * 0.1, torch.zeros(classes, device="cuda")]
    leaves = [p.clone().requires_grad_() for p in params]
    kinds = (torch.float32, torch.float32) if bits == 32 else (torch.int8, torch.uint8)
    m, v = ([torch.zeros(p.shape, dtype=t, device="cuda") for p in params] for t in kinds)
    scales = [[torch.zeros(-(-p.numel() // st.ST_ADAMW_BLOCK), device="cuda") for p in params] for _ in range(2)] if bits == 8 else [None, None]
    opt = st.st_adamw_create([p.detach() for p in leaves], m, v, None, scales[0], scales[1], lr=0.01, weight_decay=[0.1, 0.0], max_norm=0.5, cuda_stream=stream)
    refs = [Ref(f64(p).reshape(-1), bits, 0.01, 0.9, 0.999, 1e-8, wd) for p, wd in zip(params, (0.1, 0.0))]
    norm = torch.zeros(1, device="cuda")
    for _ in range(4):
        loss = torch.nn.functional.cross_entropy(tokens @ leaves[0].t() + leaves[1], labels)
        grads = torch.autograd.grad(loss, leaves)
        # the gradients are those of the formula: (softmax - onehot) over the number of tokens, back through the layer
        with torch.no_grad():
            p = torch.softmax((tokens.double() @ leaves[0].double().t() + leaves[1].double()), 1)
            d = (p - torch.nn.functional.one_hot(labels, classes)) / labels.numel()
            for g, want in zip(grads, (d.t() @ tokens.double(), d.sum(0))):
                assert (g.double() - want).norm() <= 1e-5 * want.norm()
        g64 = [f64(g).reshape(-1) for g in grads]
        total = np.sqrt(sum(float(np.sum(g * g)) for g in g64))
        factor = float(np.float32(min(1.0, 0.5 / (total + 1e-6))))
        for r, g, leaf, mm, vv in zip(refs, g64, leaves, m, v):
            if bits == 32:
                r.m, r.v = f64(mm).reshape(-1), f64(vv).reshape(-1)
            r.p, r.bound = f64(leaf).reshape(-1), np.zeros(r.p.size)
            r.step(g, factor)
        st.st_adamw_set_grads(opt, [g.contiguous() for g in grads])
        st.st_adamw_step(opt, norm_out=norm)
        assert abs(norm.item() - total) <= 2 * U * total
        for r, leaf, mm in zip(refs, leaves, m):
            assert np.all(np.abs(f64(leaf).reshape(-1) - r.p) <= r.bound)
            if bits == 8:
                assert np.array_equal(mm.cpu().numpy().reshape(-1), r.cm)
    # the trained layer leaves in 8 bits too: its logits differ from the fp32 ones by what rounding tokens and weights to steps of
    # 1/254 of a row's largest value allows
    tq, ts = quantized(tokens, stream)
    lq, ls = quantized(leaves[0].detach(), stream)
    logits = torch.zeros(h * w, classes, device="cuda")
    st.st_int8_matmul(tq, ts, lq, ls, logits, bias=leaves[1].detach(), cuda_stream=stream)
    with torch.no_grad():
        full = tokens.double() @ leaves[0].double().t() + leaves[1].double()
        off = 0.5 * ts.double()[:, None] * leaves[0].double().abs().sum(1) + 0.5 * ls.double() * tokens.double().abs().sum(1)[:, None] + 0.25 * c * ts.double()[:, None] * ls.double()
        assert bool(((logits.double() - full).abs() <= off * (1 + 1e-5) + 1e-5).all())
    st.st_adamw_destroy(opt)


def test_the_contexts_adam_and_st_adamw_take_the_same_steps(side_stream):
    """Adam inside a context (Section 5.2) and st_adamw without weight decay, fed with the gradients that the context reports, from the same student."""
    stream = side_stream.cuda_stream
    c_in, C, h, w = 8, 4, 11, 13
    theta = si.initial_head_params(c_in, 0, C, 1003)
    cls = si.voronoi_map(4 * h, 4 * w, 6, C, 2001)
    ctx = st.st_init_head(c_in=c_in, n_classes=C, feat_h=h, feat_w=w, gemm_precision=0, lr=0.01, cuda_stream=stream, init_params=theta, optimizer=1)
    st.st_set_frozen_features(ctx, 0, put(si.label_informed_features(c_in, h, w, cls, 4, 3).reshape(-1), "f32"))
    st.st_set_labels(ctx, 0, torch.from_numpy(np.ascontiguousarray(cls)).cuda())
    p, m, v, g = put(theta, "f32"), torch.zeros(theta.size, device="cuda"), torch.zeros(theta.size, device="cuda"), torch.zeros(theta.size, device="cuda")
    opt = st.st_adamw_create([p], [m], [v], [g], lr=0.01, weight_decay=0.0, cuda_stream=stream)
    packed = torch.zeros(ctx.n_params, device="cuda")
    for step in range(1, 6):
        st.st_distill_step(ctx, 1)
        g.copy_(torch.from_numpy(st.st_read_tensor(ctx, 0, st.ST_TENSOR_PARAM_GRAD)).cuda())
        st.st_adamw_step(opt)
        st.st_pack_updated_params(ctx, 0, packed)
        # both round each step to fp32; a step is at most lr (1 - b1) / sqrt(1 - b2) = 3.2 lr long, moments are off by 13 u and 16 u
        assert (p - packed).abs().max().item() <= step * (14 * U * 0.032 + 16 * U * 0.032 + 4 * U * float(np.abs(theta).max() + 0.2))
    assert st.st_adamw_step_count(opt) == 5
    st.st_adamw_destroy(opt)
    st.st_destroy(ctx)


def test_an_error_of_an_earlier_call_is_not_the_operators(side_stream):
    """A step that finds no memory for its confusion matrices leaves the runtime's last error behind.  What is enqueued after that succeeds and says so:
    a caller that is told otherwise would step twice."""
    stream = side_stream.cuda_stream
    S, C = 8000, 255                                    # 64 matrices a stream: 266 GB, one request that cannot be met
    ctx = st.st_init_head(n_streams=S, c_in=1, n_classes=C, feat_h=1, feat_w=1, cuda_stream=stream, init_params=np.zeros(S * 2 * C, np.float32))
    feature, label = torch.zeros(1, device="cuda"), torch.zeros(16, dtype=torch.uint8, device="cuda")
    for i in range(S):
        st.st_set_frozen_features(ctx, i, feature)
        st.st_set_labels(ctx, i, label)
    conf = np.empty((S, 1, C, C), np.int64)             # never touched

    def fails_for_want_of_memory():
        with pytest.raises(st.StError) as ei:
            st.st_distill_step(ctx, 1, None, conf)
        assert ei.value.status == st.ST_ERR_OOM

    p, m, v, g = put(np.ones(1000), "f32"), torch.zeros(1000, device="cuda"), torch.zeros(1000, device="cuda"), put(np.ones(1000), "f32")
    opt = st.st_adamw_create([p], [m], [v], [g], lr=0.1, max_norm=1.0, cuda_stream=stream)
    out = torch.zeros(1000, device="cuda")
    x = torch.randn(300, 20, device="cuda")
    planes = torch.randn(700, 20, device="cuda")
    q, s = torch.zeros(20, 704, dtype=torch.int8, device="cuda")[:, :700], torch.zeros(300, device="cuda")
    for call in (lambda: st.st_adamw_step(opt), lambda: st.st_adamw_set_grads(opt, [g]), lambda: st.st_adamw_set_lr(opt, 0.2),
                 lambda: st.st_adamw_read_moments(opt, [out]), lambda: st.st_adamw_write_moments(opt, [out]),
                 lambda: st.st_quantize_rows(x, torch.zeros(300, 32, dtype=torch.int8, device="cuda")[:, :20], s, cuda_stream=stream),
                 lambda: st.st_quantize_rows(planes.t(), q, s, cuda_stream=stream)):
        fails_for_want_of_memory()
        call()
    assert st.st_adamw_step_count(opt) == 1
    st.st_adamw_destroy(opt)
    st.st_destroy(ctx)
