"""GPU parity of the 8-bit integer layers.  Integers and scales of st_quantize_rows equal numpy's from the exact quotients; sums of
st_int8_matmul are exact, and the four fp32 operations behind them are those of numpy in the same order, so results are equal bit for bit."""
import os

import numpy as np
import pytest

import oracle
import synth_inputs as si
import paper_2003_10735_b200 as st

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(autouse=True)
def side_stream():
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        yield s
    s.synchronize()


def stream():
    return torch.cuda.current_stream().cuda_stream


# ---------------------------------------------------------------------------- rows to integers
def ref_quantize(x):
    """(integers, scales) of a float64 array that holds exact fp32 values."""
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        top = np.max(np.abs(x), axis=1)
        scale = np.where(np.isfinite(top), (top.astype(np.float32) / np.float32(127)), np.float32("nan")).astype(np.float32)
        q = np.rint(x / scale.astype(np.float64)[:, None])
        q[~(scale > 0)] = 0
    return np.clip(q, -127, 127).astype(np.int8), scale


def run_quantize(x, ldq=None, shift=0):
    """Integers and scales of a CUDA matrix; checks that nothing is written beside them."""
    rows, cols = x.shape
    ldq = ldq or -(-cols // 16) * 16
    buf = torch.full((rows * ldq + shift + 64,), 77, dtype=torch.int8, device="cuda")
    q = buf[shift:shift + rows * ldq].view(rows, ldq)[:, :cols]
    scale = torch.full((rows + 2,), -5.0, device="cuda")
    st.st_quantize_rows(x, q, scale[1:1 + rows], cuda_stream=stream())
    assert (buf[:shift] == 77).all() and (buf[shift + rows * ldq:] == 77).all() and scale[0] == -5 and scale[-1] == -5
    if ldq > cols:
        assert (buf[shift:shift + rows * ldq].view(rows, ldq)[:, cols:] == 77).all()
    return q.cpu().numpy(), scale[1:1 + rows].cpu().numpy()


def check_quantize(x, **kw):
    want_q, want_s = ref_quantize(x.double().cpu().numpy())
    got_q, got_s = run_quantize(x, **kw)
    assert np.array_equal(got_s, want_s, equal_nan=True)
    assert np.array_equal(got_q, want_q)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 16), (3, 17), (33, 255), (65, 256), (8, 511), (7, 512), (5, 513), (9, 1024), (4, 1025), (5, 2048), (3, 4099),
                                       (2, 8192), (2, 8200), (3, 20001), (1, 40000), (1000, 48)])
def test_rows_of_tokens(kind, rows, cols):
    torch.manual_seed(rows * 1000 + cols)
    x = (torch.randn(rows, cols, device="cuda") * torch.rand(cols, device="cuda").mul(4).exp()).to(TYPES[kind])
    check_quantize(x)
    check_quantize(x, ldq=cols, shift=1)                # integers at odd addresses
    wide = torch.randn(rows, cols + 5, device="cuda").to(TYPES[kind])
    check_quantize(wide[:, 3:3 + cols])                 # rows that begin anywhere


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("cols,h,w", [(1, 5, 7), (4, 8, 8), (21, 11, 13), (256, 9, 32), (255, 3, 21), (257, 6, 11), (300, 1, 33), (1000, 2, 17), (4333, 3, 25), (700, 40, 130), (5000, 1, 1)])
def test_pixels_of_planar_maps(kind, cols, h, w):
    torch.manual_seed(cols)
    planes = (torch.randn(cols, h, w, device="cuda") * 3).relu().to(TYPES[kind])
    check_quantize(planes.view(cols, -1).t())
    check_quantize(planes.view(cols, -1).t(), ldq=cols + 3, shift=2)
    check_quantize(planes.view(cols, -1).t()[::3])      # neither stride is 1


def test_quotients_next_to_a_half():
    """Rows built so that quotients lie on halves, and one step of fp32 beside them."""
    rng = np.random.default_rng(0)
    rows = []
    for k in range(400):
        top = np.float32(rng.uniform(0.5, 2) * 2.0 ** rng.integers(-120, 120))
        s = np.float32(top / np.float32(127))
        half = (rng.integers(-126, 126, 62) + 0.5) * np.float64(s)
        near = half.astype(np.float32)
        rows.append(np.concatenate([[top], near, np.nextafter(near, np.float32(np.inf)), np.nextafter(near, np.float32(-np.inf)), [0.0]]).astype(np.float32))
    x = np.stack(rows)
    x = np.clip(x, -np.abs(x[:, :1]), np.abs(x[:, :1]))
    check_quantize(torch.from_numpy(x).cuda())
    check_quantize(torch.from_numpy(np.ascontiguousarray(x.T)).cuda().t())


@pytest.mark.parametrize("planar,cols", [(False, 40), (False, 41), (False, 5000), (True, 40), (True, 301)])
def test_rows_that_are_zero_tiny_or_not_finite(planar, cols):
    x = torch.randn(12, cols, device="cuda")
    x[0] = 0
    x[1] = 0; x[1, 3] = 1e-45                           # the least fp32: its scale underflows
    x[2] = x[2] * 1e-39                                 # scales that fp32 holds with few bits
    x[3] = x[3] * 1e-43
    x[4, 5] = float("nan")
    x[5, 6] = float("inf")
    x[6, 7] = float("-inf"); x[6, 8] = float("nan")
    x[7] = x[7] * 1e37
    x[8] = 0; x[8, 0] = -0.0
    x[9] = -torch.finfo(torch.float32).max
    check_quantize(x.t().contiguous().t() if planar else x)


def test_quantize_offsets_beyond_32_bits():
    rows, cols = 5, 1 << 29
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    x[:, -1] = torch.tensor([1.0, -2, 3, -4, 5], device="cuda")
    x[:, 7] = 0.5
    q = torch.zeros(rows, cols, dtype=torch.int8, device="cuda")
    scale = torch.zeros(rows, device="cuda")
    st.st_quantize_rows(x, q, scale, cuda_stream=stream())
    want_q, want_s = ref_quantize(x[:, [7, -1]].double().cpu().numpy())
    assert np.array_equal(q[:, [7, -1]].cpu().numpy(), want_q) and np.array_equal(scale.cpu().numpy(), want_s)
    assert int(q.ne(0).sum()) == int(np.count_nonzero(want_q))


@pytest.mark.parametrize("planar", [False, True])
def test_as_many_columns_as_a_row_may_have(planar):
    """2^31 - 1 columns: counts of columns that are rounded up, and places of a row's last values, lie next to the end of 32-bit integers."""
    cols = 2 ** 31 - 1
    rows = 2 if planar else 1
    flat = torch.zeros(rows * cols + 3, dtype=torch.bfloat16, device="cuda")
    x = flat[3:].as_strided((rows, cols), (1, rows) if planar else (cols, 1))         # row-major: its last values lie behind the last whole piece
    at = torch.tensor([0, 255, 256, 2 ** 30 + 5] + list(range(cols - 300, cols)), device="cuda")
    x[:, at] = (torch.arange(1, at.numel() * rows + 1, device="cuda") % 97 - 48).view(rows, -1).to(torch.bfloat16)
    q, scale = torch.zeros(rows, cols, dtype=torch.int8, device="cuda"), torch.zeros(rows, device="cuda")
    st.st_quantize_rows(x, q, scale, cuda_stream=stream())
    want_q, want_s = ref_quantize(x[:, at].double().cpu().numpy())
    assert np.array_equal(scale.cpu().numpy(), want_s) and np.array_equal(q[:, at].cpu().numpy(), want_q)
    assert sum(int(torch.count_nonzero(part)) for r in range(rows) for part in q[r].split(2 ** 30)) == int(np.count_nonzero(want_q))


# ---------------------------------------------------------------------------- products
def matrix(rows, cols, seed, pitch=None, shift=0, extremes=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    pitch = pitch or -(-cols // 16) * 16
    buf = torch.full((rows * pitch + shift,), 101, dtype=torch.int8, device="cuda")         # what lies between rows must not count
    q = buf[shift:].view(rows, pitch)[:, :cols]
    q.copy_(torch.full((rows, cols), -128, device="cuda") if extremes else torch.randint(-128, 128, (rows, cols), generator=g, device="cuda"))
    return q


def ref_matmul(x, sx, w, sw, bias, relu, kind):
    acc = torch.matmul(x.double(), w.double().t()).cpu().numpy()                            # exact: below 2^53
    y = acc.astype(np.int64).astype(np.float32) * sx.cpu().numpy()[:, None] * sw.cpu().numpy()[None, :]
    if bias is not None:
        y = y + bias.cpu().numpy()
    if relu:
        y = np.where(y < 0, np.float32(0), y)
    return torch.from_numpy(y).to(TYPES[kind])


def check_matmul(m, n, k, kind="bf16", bias=True, relu=False, seed=0, px=None, pw=None, py=None, shift_x=0, shift_w=0, shift_y=0, extremes=False):
    torch.manual_seed(seed + 1)
    x, w = matrix(m, k, seed + 2, px, shift_x, extremes), matrix(n, k, seed + 3, pw, shift_w, extremes)
    sx, sw = torch.rand(m, device="cuda") * 0.02 + 1e-3, torch.rand(n, device="cuda") * 0.02 + 1e-3
    b = torch.randn(n, device="cuda") if bias else None
    py = py or n
    buf = torch.full((m * py + shift_y + 32,), 3.0, dtype=TYPES[kind], device="cuda")
    y = buf[shift_y:shift_y + m * py].view(m, py)[:, :n]
    st.st_int8_matmul(x, sx, w, sw, y, bias=b, relu=relu, cuda_stream=stream())
    want = ref_matmul(x, sx, w, sw, b, relu, kind)
    got = y.cpu()
    assert torch.equal(got, want), (m, n, k, (got != want).nonzero()[:5].tolist(), got[got != want][:5], want[got != want][:5])
    assert (buf[:shift_y] == 3).all() and (buf[shift_y + m * py:] == 3).all()
    if py > n:
        assert (buf[shift_y:shift_y + m * py].view(m, py)[:, n:] == 3).all()


SHAPES = [(1, 1, 1), (1, 256, 64), (2, 7, 33), (5, 130, 100), (16, 64, 128), (17, 65, 129), (23, 1000, 1531), (31, 200, 4096), (64, 256, 256), (100, 300, 513),
          (127, 127, 127), (128, 128, 128), (129, 129, 129), (200, 513, 700), (256, 512, 2048), (300, 40, 96), (1000, 1000, 1000), (3000, 256, 512), (20000, 64, 48),
          (40000, 129, 32), (1, 4096, 4096), (4, 5000, 8200), (700, 2500, 160)]


@pytest.mark.parametrize("m,n,k", SHAPES)
def test_products(m, n, k):
    check_matmul(m, n, k, "bf16", seed=m)
    check_matmul(m, n, k, "f32", bias=False, relu=True, seed=n)


# shapes that each width of tile, with and without weights that stay, one round and several, two and four groups that store, and each token count of
# the cluster form is taken for
@pytest.mark.parametrize("m,n,k", [(30, 4096, 2048), (60, 4100, 4096), (100, 1000, 300), (16, 130, 8192), (3, 20000, 256), (9000, 64, 700), (20011, 384, 384),
                                   (4100, 1024, 1024), (30000, 256, 512), (30001, 250, 1024), (4099, 4096, 512), (3001, 5000, 2500), (2048, 2304, 3000),
                                   (8193, 700, 4096), (300, 20000, 2048), (4097, 4095, 4100)])
@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_products_of_every_form(m, n, k, kind):
    check_matmul(m, n, k, kind, relu=True, seed=k)


@pytest.mark.parametrize("m,n,k", [(1, 33, 70), (50, 257, 300), (333, 100, 64), (5000, 300, 200)])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_products_of_any_layout(m, n, k, kind):
    check_matmul(m, n, k, kind, py=n + 3)                                       # rows of y that allow no wide stores
    check_matmul(m, n, k, kind, relu=True, px=-(-k // 16) * 16 + 64, pw=-(-k // 16) * 16 + 32, shift_y=1)
    check_matmul(m, n, k, kind, bias=False, px=k + 1, pw=k + 2, shift_x=1, shift_w=3)        # nothing that TMA could read
    check_matmul(m, n, k, kind, shift_x=16, shift_w=48, py=-(-n // 16) * 16)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shift", [0, 1, 2, 3])
@pytest.mark.parametrize("pitch", [331, 332, 334, 345])
def test_rows_of_y_at_every_alignment(kind, shift, pitch):
    check_matmul(1000, 331, 200, kind, py=pitch, shift_y=shift, relu=True)
    check_matmul(3000, 300, 2100, kind, py=pitch, shift_y=shift)        # columns behind y's end stay


def test_sums_at_the_end_of_the_integers():
    """K = 131071 products of (-128)^2: the largest sum that 32 bits hold."""
    for m, n in ((1, 3), (130, 20), (300, 300)):
        check_matmul(m, n, 131071, "f32", extremes=True)


def test_scales_that_are_not_finite_reach_y():
    x, w = matrix(40, 64, 1), matrix(50, 64, 2)
    sx, sw = torch.ones(40, device="cuda"), torch.ones(50, device="cuda")
    sx[3] = float("nan"); sw[7] = float("inf")
    y = torch.zeros(40, 50, device="cuda")
    st.st_int8_matmul(x, sx, w, sw, y, relu=True, cuda_stream=stream())
    assert torch.isnan(y[3]).all() and torch.isfinite(y[4, :7]).all()
    acc = torch.matmul(x.double(), w.double().t())
    keep = torch.arange(40, device="cuda") != 3
    assert torch.equal(torch.isinf(y[keep, 7]), acc[keep, 7] > 0)


def test_product_offsets_beyond_32_bits():
    m, n, k = 9_000_000, 256, 256
    x = torch.zeros(m, k, dtype=torch.int8, device="cuda")
    x[-300:] = torch.randint(-128, 128, (300, k), device="cuda")
    w, sw = matrix(n, k, 5), torch.rand(n, device="cuda")
    sx = torch.rand(m, device="cuda")
    y = torch.full((m, n), 9.0, dtype=torch.bfloat16, device="cuda")
    st.st_int8_matmul(x, sx, w, sw, y, cuda_stream=stream())
    want = ref_matmul(x[-300:], sx[-300:], w, sw, None, False, "bf16")
    assert torch.equal(y[-300:].cpu(), want) and (y[:1000] == 0).all() and (y[m // 2:m // 2 + 1000] == 0).all()


def test_clusters_of_several_streams_at_once():
    """Small products whose clusters share SMs, on four streams: each block needs tensor memory before its cluster can go on."""
    streams = [torch.cuda.Stream() for _ in range(4)]
    shapes = [(16, 1024, 512), (60, 1024, 4096), (100, 1024, 8192)]
    sets = [(matrix(m, k, i), matrix(n, k, i + 5), torch.rand(m, device="cuda"), torch.rand(n, device="cuda")) for i, (m, n, k) in enumerate(shapes)]
    ys = [[torch.zeros(m, n, device="cuda") for m, n, _ in shapes] for _ in streams]
    st.st_int8_matmul(sets[0][0], sets[0][2], sets[0][1], sets[0][3], ys[0][0], cuda_stream=stream())
    torch.cuda.synchronize()
    for _ in range(40):
        for i, ((x, w, sx, sw)) in enumerate(sets):
            for s, y in zip(streams, ys):
                st.st_int8_matmul(x, sx, w, sw, y[i], cuda_stream=s.cuda_stream)
    torch.cuda.synchronize()
    for i, (x, w, sx, sw) in enumerate(sets):
        want = ref_matmul(x, sx, w, sw, None, False, "f32")
        assert all(torch.equal(y[i].cpu(), want) for y in ys)


def test_products_on_two_streams_and_replayed():
    """Calls share no workspace: two streams at once, and a captured call replayed between eager ones."""
    other = torch.cuda.Stream()
    sets = []
    for i, (m, n, k) in enumerate([(3, 4096, 2048), (2000, 512, 512), (60, 700, 4096)]):
        x, w = matrix(m, k, i), matrix(n, k, i + 10)
        sx, sw = torch.rand(m, device="cuda"), torch.rand(n, device="cuda")
        sets.append((x, sx, w, sw, [torch.zeros(m, n, device="cuda") for _ in range(3)]))
    for x, sx, w, sw, ys in sets:
        st.st_int8_matmul(x, sx, w, sw, ys[0], cuda_stream=stream())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, capture_error_mode="thread_local"):
        for x, sx, w, sw, ys in sets:
            st.st_int8_matmul(x, sx, w, sw, ys[1], cuda_stream=torch.cuda.current_stream().cuda_stream)
    for _ in range(20):
        with torch.cuda.stream(other):
            graph.replay()
        for x, sx, w, sw, ys in sets:
            st.st_int8_matmul(x, sx, w, sw, ys[2], cuda_stream=stream())
    torch.cuda.synchronize()
    for *_, ys in sets:
        assert torch.equal(ys[0], ys[1]) and torch.equal(ys[0], ys[2])


def test_refusals():
    x, w, s, y = matrix(8, 32, 0), matrix(8, 32, 1), torch.ones(8, device="cuda"), torch.zeros(8, 8, device="cuda")

    def refused(f):
        with pytest.raises(st.StError) as ei:
            f()
        assert ei.value.status == st.ST_ERR_INVALID_ARG
        return str(ei.value)

    assert "current device" in refused(lambda: st.st_int8_matmul(x.cpu(), s, w, s, y))
    assert "current device" in refused(lambda: st.st_int8_matmul(x, s, w, s.cpu(), y))
    assert "current device" in refused(lambda: st.st_int8_matmul(x, s, w, s, y.cpu()))
    assert "overlap" in refused(lambda: st.st_int8_matmul(x, s, w, s, x.view(torch.float32)[:, :8].as_strided((8, 8), (8, 1)), bias=None))
    assert "overlap" in refused(lambda: st.st_int8_matmul(x, s, w, s, y, bias=y[0]))
    f = torch.randn(8, 32, device="cuda")
    assert "current device" in refused(lambda: st.st_quantize_rows(f.cpu(), x, s))
    assert "current device" in refused(lambda: st.st_quantize_rows(f, x, s.cpu()))
    assert "overlap" in refused(lambda: st.st_quantize_rows(f, f.view(torch.int8)[:, :32], s))
    raw = torch.zeros(401, dtype=torch.uint8, device="cuda")
    odd = raw[1:].data_ptr()
    lib = st.load_library()
    assert lib.st_quantize_rows(odd, st.ST_F32, 4, 8, 8, 1, x.data_ptr(), 32, s.data_ptr(), stream() or None) == st.ST_ERR_INVALID_ARG
    assert "aligned" in st.st_last_error(None)
    assert lib.st_int8_matmul(x.data_ptr(), 32, s.data_ptr(), w.data_ptr(), 32, s.data_ptr(), None, 0, 8, 8, 32, odd, st.ST_BF16, 8, stream() or None) == st.ST_ERR_INVALID_ARG
    # the same integers as tokens and as weights are no fault
    st.st_int8_matmul(x, s, x, s, y, cuda_stream=stream())
    assert torch.equal(y.cpu(), ref_matmul(x, s, x, s, None, False, "f32"))


@pytest.mark.parametrize("m,n,k", [(300, 200, 1024), (4, 1000, 4096), (4096, 4096, 4096)])
def test_a_wait_that_runs_out_is_reported(m, n, k, monkeypatch):
    """The first stage of every block expects bytes that never come: the waits give up, and the next call says so."""
    x, w, sx, sw, y = matrix(m, k, 0), matrix(n, k, 1), torch.ones(m, device="cuda"), torch.ones(n, device="cuda"), torch.zeros(m, n, device="cuda")
    st.st_int8_matmul(x, sx, w, sw, y, cuda_stream=stream())
    monkeypatch.setenv("ST_TEST_STALL_INT8", "1")
    st.st_int8_matmul(x, sx, w, sw, y, cuda_stream=stream())
    torch.cuda.synchronize()
    monkeypatch.delenv("ST_TEST_STALL_INT8")
    with pytest.raises(st.StError) as ei:
        st.st_int8_matmul(x, sx, w, sw, y, cuda_stream=stream())
    assert ei.value.status == st.ST_ERR_CUDA and "gave up" in str(ei.value)
    st.st_int8_matmul(x, sx, w, sw, y, cuda_stream=stream())
    assert torch.equal(y.cpu(), ref_matmul(x, sx, w, sw, None, False, "f32"))


def test_a_product_that_gave_up_is_told_of_on_its_own_stream(monkeypatch):
    """A call on another stream is neither refused nor told; the call on the same stream is told, and its own product is there."""
    m, n, k = 300, 200, 1024
    x, w, sx, sw = matrix(m, k, 0), matrix(n, k, 1), torch.rand(m, device="cuda"), torch.rand(n, device="cuda")
    ys = [torch.zeros(m, n, device="cuda") for _ in range(3)]
    other = torch.cuda.Stream()
    st.st_int8_matmul(x, sx, w, sw, ys[0], cuda_stream=stream())
    monkeypatch.setenv("ST_TEST_STALL_INT8", "1")
    st.st_int8_matmul(x, sx, w, sw, ys[0], cuda_stream=stream())
    monkeypatch.delenv("ST_TEST_STALL_INT8")
    torch.cuda.synchronize()
    st.st_int8_matmul(x, sx, w, sw, ys[1], cuda_stream=other.cuda_stream)
    with pytest.raises(st.StError) as ei:
        st.st_int8_matmul(x, sx, w, sw, ys[2], cuda_stream=stream())
    assert ei.value.status == st.ST_ERR_CUDA and "gave up" in str(ei.value)
    torch.cuda.synchronize()
    want = ref_matmul(x, sx, w, sw, None, False, "f32")
    assert torch.equal(ys[1].cpu(), want) and torch.equal(ys[2].cpu(), want)
    st.st_int8_matmul(x, sx, w, sw, ys[2], cuda_stream=stream())


def test_a_product_that_gave_up_inside_a_graph_is_told_of_by_the_next_call(monkeypatch):
    """The stream that was captured may see no call again: whichever product comes next on the device tells of it, once, and is there itself."""
    m, n, k = 40, 200, 1024
    x, w, sx, sw = matrix(m, k, 0), matrix(n, k, 1), torch.rand(m, device="cuda"), torch.rand(n, device="cuda")
    ys = [torch.zeros(m, n, device="cuda") for _ in range(3)]
    st.st_int8_matmul(x, sx, w, sw, ys[0], cuda_stream=stream())
    torch.cuda.synchronize()
    monkeypatch.setenv("ST_TEST_STALL_INT8", "1")
    graph, captured = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=captured, capture_error_mode="thread_local"):
        st.st_int8_matmul(x, sx, w, sw, ys[1], cuda_stream=torch.cuda.current_stream().cuda_stream)
    monkeypatch.delenv("ST_TEST_STALL_INT8")
    st.st_int8_matmul(x, sx, w, sw, ys[2], cuda_stream=stream())            # nothing has run yet
    graph.replay()
    torch.cuda.synchronize()
    ys[2].zero_()
    with pytest.raises(st.StError) as ei:
        st.st_int8_matmul(x, sx, w, sw, ys[2], cuda_stream=stream())
    assert ei.value.status == st.ST_ERR_CUDA and "graph gave up" in str(ei.value)
    torch.cuda.synchronize()
    assert torch.equal(ys[2].cpu(), ref_matmul(x, sx, w, sw, None, False, "f32"))
    st.st_int8_matmul(x, sx, w, sw, ys[2], cuda_stream=stream())


@pytest.mark.parametrize("k,n", [(96, 48), (97, 33)])
def test_matrices_that_lie_beside_each_other_in_one_buffer(k, n):
    """Integers behind the rows that they are made from, products behind the integers: no byte is shared, and nothing else changes."""
    m, pitch = 150, 1024
    g = torch.Generator(device="cuda").manual_seed(k)
    buf = torch.randint(0, 256, (m + 1, pitch), dtype=torch.uint8, generator=g, device="cuda")[:m]
    x = buf[:, :4 * k].view(torch.float32)
    x.copy_(torch.randn(m, k, generator=g, device="cuda"))
    q = buf[:, 4 * k:5 * k].view(torch.int8)
    y0 = -(-5 * k // 4) * 4
    y = buf[:, y0:y0 + 4 * n].view(torch.float32)
    scale, w, sw = torch.zeros(m, device="cuda"), matrix(n, k, 3), torch.rand(n, device="cuda")
    before = buf.clone()
    st.st_quantize_rows(x, q, scale, cuda_stream=stream())
    want_q, want_s = ref_quantize(x.double().cpu().numpy())
    assert np.array_equal(q.cpu().numpy(), want_q) and np.array_equal(scale.cpu().numpy(), want_s)
    st.st_int8_matmul(q, scale, w, sw, y, cuda_stream=stream())
    assert torch.equal(y.cpu(), ref_matmul(q, scale, w, sw, None, False, "f32"))
    before[:, 4 * k:5 * k], before[:, y0:y0 + 4 * n] = buf[:, 4 * k:5 * k], buf[:, y0:y0 + 4 * n]
    assert torch.equal(buf, before)
    planes = torch.zeros(60, 256, device="cuda")                    # pixels of planes, integers behind each plane
    st.st_quantize_rows(planes[:, :50].t(), planes.view(torch.int8)[:50, 400:460], torch.zeros(50, device="cuda"), cuda_stream=stream())
    for call in (lambda: st.st_quantize_rows(x, buf[:, 4 * k - 1:5 * k - 1].view(torch.int8), scale),                      # a byte shared
                 lambda: st.st_quantize_rows(x, buf[:, pitch - 1:].view(torch.int8).as_strided((m, k), (pitch, 1)), scale),          # in the next row
                 lambda: st.st_int8_matmul(q, scale, w, sw, buf.view(torch.float32).as_strided((m, n), (pitch // 4 + 1, 1), y0 // 4)),     # another pitch
                 lambda: st.st_int8_matmul(q, scale, w, sw, y, bias=y[3])):
        with pytest.raises(st.StError) as ei:
            call()
        assert ei.value.status == st.ST_ERR_INVALID_ARG and "overlap" in str(ei.value)


# ---------------------------------------------------------------------------- with a context
@pytest.mark.parametrize("h,w,k", [(10, 37, 96), (45, 80, 200)])
def test_the_front_parts_last_layer_in_8_bits(h, w, k):
    """A planar map is quantised, the front part's last 1x1 layer multiplies it into the feature cache, the head is trained on it: the same as
    with the layer's output given as a feature map."""
    c_in, C, S = 64, 5, 2
    torch.manual_seed(0)
    weight, bias = torch.randn(c_in, k, device="cuda"), torch.randn(c_in, device="cuda")
    wq, ws = torch.zeros(c_in, -(-k // 16) * 16, dtype=torch.int8, device="cuda")[:, :k], torch.zeros(c_in, device="cuda")
    st.st_quantize_rows(weight, wq, ws, cuda_stream=stream())
    theta = np.tile(si.initial_head_params(c_in, 0, C, 1000), S)
    ctxs = [st.st_init_head(n_streams=S, c_in=c_in, n_classes=C, feat_h=h, feat_w=w, gemm_precision=1, lr=0.02, momentum=0.9,
                            cuda_stream=stream(), init_params=theta) for _ in range(2)]
    for s in range(S):
        planes = torch.randn(k, h, w, device="cuda").relu() * (s + 1)
        xq, xs = torch.zeros(h * w, -(-k // 16) * 16, dtype=torch.int8, device="cuda")[:, :k], torch.zeros(h * w, device="cuda")
        st.st_quantize_rows(planes.view(k, -1).t(), xq, xs, cuda_stream=stream())
        st.st_set_frozen_features_int8(ctxs[0], s, xq, xs, wq, ws, bias, relu=True)
        y = torch.zeros(h * w, c_in, device="cuda")
        st.st_int8_matmul(xq, xs, wq, ws, y, bias=bias, relu=True, cuda_stream=stream())
        st.st_set_frozen_features(ctxs[1], s, y.t().contiguous().view(c_in, h, w))
        labels = torch.randint(0, C, (4 * h, 4 * w), dtype=torch.uint8, device="cuda")
        for c in ctxs:
            st.st_set_labels(c, s, labels)
        assert np.array_equal(st.st_read_tensor(ctxs[0], s, st.ST_TENSOR_FEATURES), st.st_read_tensor(ctxs[1], s, st.ST_TENSOR_FEATURES))
        # the layer in fp32 is near: 1/254 of a row's and of a channel's largest value, per product
        full = (planes.view(k, -1).t() @ weight.t() + bias).relu()
        assert (y - full).norm() < 0.02 * full.norm()
    outs = []
    for c in ctxs:
        loss = torch.zeros(S, 3, device="cuda")
        st.st_distill_step(c, 3, loss)
        packed = torch.zeros(c.n_params, device="cuda")
        st.st_pack_updated_params(c, 1, packed)
        outs.append((loss.clone(), packed.clone()))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
    with pytest.raises(ValueError):
        st.st_set_frozen_features_int8(ctxs[0], 0, xq[:-1], xs[:-1], wq, ws)
    with pytest.raises(st.StError):
        st.st_set_frozen_features_int8(ctxs[0], S, xq, xs, wq, ws)
    plain = st.st_init_head(c_in=c_in, n_classes=C, feat_h=h, feat_w=w, cuda_stream=stream(), init_params=theta[:theta.size // S])
    with pytest.raises(st.StError) as ei:
        st.st_set_frozen_features_int8(plain, 0, xq, xs, wq, ws)
    assert ei.value.status == st.ST_ERR_UNSUPPORTED
    for c in ctxs + [plain]:
        st.st_destroy(c)


@pytest.mark.parametrize("h,w,k", [(6, 11, 4096), (45, 80, 200)])
def test_a_feature_cache_left_incomplete_is_the_contexts_to_report(h, w, k, monkeypatch):
    """A wait that runs out while the feature cache is filled (few pixels: the form that splits K; many: tiles) is reported by the context's
    next call that waits, once, and by nobody else's product."""
    c_in, C = 64, 5
    x, wq, sx, sw = matrix(h * w, k, 0), matrix(c_in, k, 1), torch.rand(h * w, device="cuda") * 1e-3, torch.rand(c_in, device="cuda") * 1e-2
    y = torch.zeros(h * w, c_in, dtype=torch.bfloat16, device="cuda")
    st.st_int8_matmul(x, sx, wq, sw, y, cuda_stream=stream())
    ctx = st.st_init_head(c_in=c_in, n_classes=C, feat_h=h, feat_w=w, gemm_precision=1, cuda_stream=stream(),
                          init_params=si.initial_head_params(c_in, 0, C, 1000))
    st.st_set_labels(ctx, 0, torch.zeros(4 * h, 4 * w, dtype=torch.uint8, device="cuda"))
    monkeypatch.setenv("ST_TEST_STALL_INT8", "1")
    st.st_set_frozen_features_int8(ctx, 0, x, sx, wq, sw)
    monkeypatch.delenv("ST_TEST_STALL_INT8")
    torch.cuda.synchronize()
    st.st_int8_matmul(x, sx, wq, sw, y, cuda_stream=stream())               # another caller's product: nothing of it gave up
    assert torch.equal(y.cpu(), ref_matmul(x, sx, wq, sw, None, False, "bf16"))
    with pytest.raises(st.StError) as ei:
        st.st_distill_step(ctx, 1, np.zeros(1, np.float32))
        st.st_read_tensor(ctx, 0, st.ST_TENSOR_FEATURES)
    assert ei.value.status == st.ST_ERR_CUDA and "gave up waiting" in str(ei.value)
    st.st_set_frozen_features_int8(ctx, 0, x, sx, wq, sw)
    got = st.st_read_tensor(ctx, 0, st.ST_TENSOR_FEATURES).reshape(c_in, h * w)
    assert np.array_equal(got, y.float().cpu().numpy().T)
    st.st_destroy(ctx)
