"""GPU parity of st_adamw: one optimiser over many tensors, moments in 32 and in 8 bits, against the formulas in 64 bits.

Bounds count roundings.  With u = 2^-24 (half a step of fp32, relative):
  m   b1 m + (1 - b1) f g: the coefficients (1 each), f (1), f g (1), (1 - b1) f g (1), the sum (1): 5 u of |b1 m| + |(1 - b1) f g|
  v   the same with g twice: 8 u of b2 v + (1 - b2) (f g)^2
  u   the update lr1 m / (root r2 + eps): m as above; the root 4 + 1, r2 1, its product with the sum 1, eps 1, the quotient 1, lr, its factor,
      lr_scale and their products 5: 14 u of |update|, and the error of m through the same quotient
  p   decay: lr, wd, two products 4 u of |lr wd p|; the two sums 2 u of |p|
and parameters of 16 bits are off by half a step of their type on top.  With 8-bit moments the levels and scales are defined by fp32
operations, so they are equal to numpy's."""
import numpy as np
import pytest

import paper_2003_10735_b200 as st

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

U = 2.0 ** -24
BLOCK = st.ST_ADAMW_BLOCK
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_STEP = {"f32": 0.0, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}


@pytest.fixture(autouse=True)
def side_stream():
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        yield s
    s.synchronize()


def stream():
    return torch.cuda.current_stream().cuda_stream


def put(values, kind, shift=0):
    """A CUDA tensor of the values that begins `shift` elements into an allocation."""
    v = torch.as_tensor(values)
    dtype = kind if isinstance(kind, torch.dtype) else TYPES[kind]
    buf = torch.zeros(v.numel() + shift, dtype=dtype, device="cuda")
    buf[shift:] = v.to(dtype).cuda()
    return buf[shift:]


def f64(t):
    return t.detach().double().cpu().numpy()


class Ref:
    """The formulas for one tensor, in 64 bits; with 8-bit moments the levels as fp32 operations give them."""

    def __init__(self, p, bits, lr, b1, b2, eps, wd, t=0):
        n = p.size
        self.p, self.bits, self.lr, self.b1, self.b2, self.eps, self.wd, self.t = p.astype(np.float64), bits, lr, b1, b2, eps, wd, t
        self.m, self.v = np.zeros(n), np.zeros(n)
        k = -(-n // BLOCK)
        self.cm, self.cv = np.zeros(n, np.int8), np.zeros(n, np.uint8)
        self.ms, self.vs = np.zeros(k, np.float32), np.zeros(k, np.float32)
        self.bound = np.zeros(n)        # how far fp32 parameters may be off by now

    def _rep(self, s, n):
        return np.repeat(s, BLOCK)[:n]

    def decoded(self):
        n, f = self.p.size, np.float32
        with np.errstate(invalid="ignore", over="ignore"):
            c, d = self.cm.astype(np.int32), self.cv.astype(np.int32)
            return (c * np.abs(c)).astype(f) * self._rep(self.ms, n), (d * d).astype(f) * self._rep(self.vs, n)

    def encode(self, m, root):
        f, n = np.float32, m.size
        for b in range(self.ms.size):
            s = slice(b * BLOCK, min((b + 1) * BLOCK, n))
            with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
                top, top_root = np.max(np.abs(m[s])), np.max(root[s])                 # NaN where there is one
                ms = f(0) if top < f(2.0 ** -100) else f(top / f(127 * 127))
                vs = f(top_root / f(255 * 255))
                im, iv = f(1) / ms if ms > 0 else f(0), f(1) / vs if vs > 0 else f(0)
                level = lambda r, most: np.minimum(np.floor(np.sqrt((r.astype(f)).astype(np.float64)) + 0.5), most)  # noqa: E731
                cm = np.nan_to_num(level(np.abs(m[s]) * im, 127), nan=0.0)
                cv = np.nan_to_num(level(root[s] * iv, 255), nan=0.0)
            self.ms[b], self.vs[b] = ms, vs
            self.cm[s] = np.where(m[s] < 0, -cm, cm).astype(np.int8)
            self.cv[s] = np.where(root[s] > 0, np.maximum(cv, 1), cv).astype(np.uint8)

    def step(self, g, factor=1.0, lr=None):
        lr = self.lr if lr is None else lr
        self.t += 1
        f, t = np.float32, self.t
        c1, r2 = 1 - self.b1 ** t, 1 / np.sqrt(1 - self.b2 ** t)
        with np.errstate(invalid="ignore", over="ignore"):
            if self.bits == 32:
                gf = g * factor
                sm = np.abs(self.b1 * self.m) + np.abs((1 - self.b1) * gf)
                self.m = self.b1 * self.m + (1 - self.b1) * gf
                self.v = self.b2 * self.v + (1 - self.b2) * gf * gf
                m, root = self.m, np.sqrt(self.v)
                m_off = 5 * U * sm
            else:
                m0, r0 = self.decoded()
                gf = g.astype(f) * f(factor)
                m32 = m0 * f(self.b1) + gf * f(1 - self.b1)
                root32 = np.sqrt((r0 * r0) * f(self.b2) + (gf * gf) * f(1 - self.b2))
                self.encode(m32, root32)
                m, root, m_off = m32.astype(np.float64), root32.astype(np.float64), 0.0
            den = root * r2 + self.eps
            update = lr / c1 * m / den
            self.bound = self.bound + lr / c1 * m_off / den + 14 * U * np.abs(update) + 4 * U * np.abs(lr * self.wd * self.p) + 2 * U * np.abs(self.p)
            self.p = self.p - lr * self.wd * self.p - update


def make(sizes, bits, param="f32", grad="f32", master=False, shift=0, seed=0, lr=1e-2, b1=0.9, b2=0.99, eps=1e-8, wd=0.05, **kw):
    rng = np.random.default_rng(seed)
    values = [rng.normal(0, 0.5, n).astype(np.float32) for n in sizes]
    params = [put(v, param, shift) for v in values]
    masters = [put(v, "f32", shift) for v in values] if master else None
    kinds = (torch.float32, torch.float32) if bits == 32 else (torch.int8, torch.uint8)
    m = [put(np.zeros(n), kinds[0], shift) for n in sizes]
    v = [put(np.zeros(n), kinds[1], shift) for n in sizes]
    scales = [[put(np.zeros(-(-n // BLOCK)), "f32") for n in sizes] for _ in range(2)] if bits == 8 else [None, None]
    grads = [put(np.zeros(n), grad, shift) for n in sizes]
    opt = st.st_adamw_create(params, m, v, grads, scales[0], scales[1], masters, lr=lr, beta1=b1, beta2=b2, eps=eps, weight_decay=wd,
                             cuda_stream=stream(), **kw)
    start = masters if master else params
    t = kw.get("first_step", 0)
    refs = [Ref(f64(p), bits, lr, b1, b2, eps, wd if np.isscalar(wd) else wd[i], t) for i, p in enumerate(start)]
    return opt, params, masters, m, v, scales, grads, refs


def new_grads(rng, grads, kind, std=0.1):
    out = []
    for g in grads:
        x = torch.from_numpy(rng.normal(0, std, g.numel()) * (rng.random(g.numel()) < 0.9)).to(TYPES[kind])
        g.copy_(x.cuda())
        out.append(f64(g))
    return out


def check(made, param, master, bits):
    _, params, masters, m, v, scales, _, refs = made
    for i, r in enumerate(refs):
        if r.p.size == 0:
            continue
        off = r.bound
        got = f64(masters[i]) if master else f64(params[i])
        if master or param == "f32":
            assert np.all(np.abs(got - r.p) <= off), (i, np.max(np.abs(got - r.p) - off))
        if master:
            assert torch.equal(params[i], masters[i].to(params[i].dtype)), i
        elif param != "f32":
            tiny = 2.0 ** -25 if param == "f16" else 0.0
            assert np.all(np.abs(got - r.p) <= off + HALF_STEP[param] * np.abs(r.p) + tiny), i
        if bits == 32:
            assert np.all(np.abs(f64(m[i]) - r.m) <= r.m_bound) and np.all(np.abs(f64(v[i]) - r.v) <= r.v_bound), i
        else:
            assert np.array_equal(m[i].cpu().numpy(), r.cm), i
            assert np.array_equal(v[i].cpu().numpy(), r.cv), i
            assert np.array_equal(scales[0][i].cpu().numpy(), r.ms, equal_nan=True), i
            assert np.array_equal(scales[1][i].cpu().numpy(), r.vs, equal_nan=True), i


def run_steps(made, param, grad, master, bits, steps, factor=None, seed=3):
    """Steps; 32-bit moments and 16-bit parameters are taken over by the reference after each, so that every step is checked by itself."""
    opt, params, masters, m, v, _, grads, refs = made
    rng = np.random.default_rng(seed)
    for _ in range(steps):
        g = new_grads(rng, grads, grad)
        f = 1.0 if factor is None else factor(g)
        for r, x, p, a, mm, vv in zip(refs, g, params, masters or params, m, v):
            if bits == 32:
                r.m, r.v = f64(mm), f64(vv)
                r.m_bound = 5 * U * (np.abs(r.b1 * r.m) + np.abs((1 - r.b1) * f * x)) + 2.0 ** -149
                r.v_bound = 8 * U * (r.b2 * r.v + (1 - r.b2) * (f * x) ** 2) + 2.0 ** -149
            r.p, r.bound = f64(a), np.zeros(r.p.size)
            r.step(x, f)
        st.st_adamw_step(opt)
        check(made, param, master, bits)


SIZES = [1, 2, 255, 256, 257, 0, 2047, 2048, 2049, 5003, 31, 4096]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param,grad,master,shift", [
    ("f32", "f32", False, 0), ("f32", "bf16", False, 0), ("f32", "f16", False, 3), ("bf16", "bf16", False, 0), ("bf16", "f32", True, 0),
    ("f16", "f16", True, 0), ("f16", "f32", False, 1), ("f32", "f32", True, 0), ("bf16", "bf16", True, 5)])
def test_steps_match_the_formulas(bits, param, grad, master, shift):
    made = make(SIZES, bits, param, grad, master, shift)
    run_steps(made, param, grad, master, bits, 3)
    assert st.st_adamw_step_count(made[0]) == 3
    st.st_adamw_destroy(made[0])


@pytest.mark.parametrize("bits", [32, 8])
def test_clipping_and_late_steps(bits):
    made = make([300, 4099, 17], bits, max_norm=0.5, first_step=1000)

    def factor(g):
        norm = np.sqrt(sum(float(np.sum(x * x)) for x in g))
        return float(np.float32(min(1.0, 0.5 / (norm + 1e-6))))

    run_steps(made, "f32", "f32", False, bits, 2, factor)
    norm = torch.zeros(1, device="cuda")
    g = new_grads(np.random.default_rng(9), made[6], "f32")
    st.st_adamw_step(made[0], 0.25, norm)
    want = 0.25 * np.sqrt(sum(float(np.sum(x * x)) for x in g))
    assert abs(norm.item() - want) <= 2 * U * want
    assert st.st_adamw_step_count(made[0]) == 1003


def test_each_tensor_has_its_decay_and_its_share_of_the_learning_rate():
    sizes, wd, share = [40, 50, 60], [0.0, 0.5, 0.1], [1.0, 0.1, 3.0]
    made = make(sizes, 32, wd=wd, lr_scale=share, lr=0.02)
    for r, s in zip(made[7], share):
        r.lr = 0.02 * s
    run_steps(made, "f32", "f32", False, 32, 2)
    # a new learning rate holds from the next step on
    st.st_adamw_set_lr(made[0], 0.004)
    for r, s in zip(made[7], share):
        r.lr = 0.004 * s
    run_steps(made, "f32", "f32", False, 32, 1, seed=5)


@pytest.mark.parametrize("betas", [(0.0, 0.99), (0.9, 0.0), (0.0, 0.0)])
def test_decay_rates_of_zero(betas):
    for bits in (32, 8):
        run_steps(make([700], bits, b1=betas[0], b2=betas[1]), "f32", "f32", False, bits, 2)


@pytest.mark.parametrize("bits", [32, 8])
def test_tensors_without_a_gradient_are_left_alone(bits):
    made = make([300, 400, 500], bits)
    opt, params, _, m, v, scales, grads, refs = made
    run_steps(made, "f32", "f32", False, bits, 1)
    st.st_adamw_set_grads(opt, [grads[0], None, grads[2]])
    kept = [t.clone() for t in (params[1], m[1], v[1])]
    norm = torch.zeros(1, device="cuda")
    st.st_adamw_step(opt, norm_out=norm)
    for a, b in zip(kept, (params[1], m[1], v[1])):
        assert torch.equal(a, b)
    want = np.sqrt(sum(float(np.sum(f64(grads[i]) ** 2)) for i in (0, 2)))
    assert abs(norm.item() - want) <= 2 * U * want
    assert st.st_adamw_step_count(opt) == 2


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_norm_that_is_not_finite_skips_the_step(bits, bad):
    made = make([600, 100], bits, skip_nonfinite=True)
    opt, params, _, m, v, scales, grads, refs = made
    run_steps(made, "f32", "f32", False, bits, 1)
    kept = [t.clone() for t in params + m + v]
    g = grads[1][50].item()
    grads[1][50] = bad
    st.st_adamw_step(opt)
    assert all(torch.equal(a, b) for a, b in zip(kept, params + m + v)) and st.st_adamw_step_count(opt) == 1
    grads[1][50] = g
    run_steps(made, "f32", "f32", False, bits, 1, seed=8)
    assert st.st_adamw_step_count(opt) == 2


def test_a_gradient_that_is_not_finite_stays_in_its_block():
    made = make([1000], 8)
    opt, params, _, m, v, scales, grads, refs = made
    new_grads(np.random.default_rng(1), grads, "f32")
    grads[0][300] = float("nan")
    refs[0].step(f64(grads[0]))
    st.st_adamw_step(opt)
    got = f64(params[0])
    assert np.isnan(got[300]) and np.isfinite(np.delete(got, 300)).all()
    out = [torch.zeros(1000, device="cuda") for _ in range(2)]
    st.st_adamw_read_moments(opt, [out[0]], [out[1]])
    for o in out:
        bad = ~np.isfinite(f64(o))
        assert bad[256:512].all() and not bad[:256].any() and not bad[512:].any()


def test_moments_that_fade_away_end_at_zero():
    """Without gradients m shrinks by b1 each step; in 8 bits it ends at 0 before its scale leaves the range of fp32."""
    made = make([300], 8, b1=0.5, b2=0.5, wd=0.0)
    opt, params, _, m, v, scales, grads, refs = made
    new_grads(np.random.default_rng(1), grads, "f32")
    g = f64(grads[0])
    refs[0].step(g)
    st.st_adamw_step(opt)
    grads[0].zero_()
    for _ in range(130):
        refs[0].step(np.zeros(300))
        st.st_adamw_step(opt)
    check((opt, [], None, m, v, scales, grads, []), "f32", False, 8)
    assert np.array_equal(m[0].cpu().numpy(), refs[0].cm) and np.array_equal(v[0].cpu().numpy(), refs[0].cv)
    assert np.array_equal(scales[1][0].cpu().numpy(), refs[0].vs) and (refs[0].ms == 0).all() and (refs[0].cm == 0).all()
    assert torch.isfinite(params[0]).all()


@pytest.mark.parametrize("b2,steady,shrunk", [(0.99, (0.95, 1.05), (0.93, 1.08)), (0.999, (1.0, 1.3), (2.0, 6.0))])
def test_moments_in_8_bits_over_thousands_of_steps(b2, steady, shrunk):
    """3,000 steps against the definition, level by level, and against fp32 moments.  After the first 1,000 the gradients of half of each block fall tenfold.
    The ranges of the medians are those that the header gives: with beta2 0.99 sqrt(v) follows, with 0.999 it does not."""
    n = 2 * BLOCK
    eight, full = make([n], 8, b2=b2, wd=0.0, lr=1e-4), make([n], 32, b2=b2, wd=0.0, lr=1e-4)
    rng, ref = np.random.default_rng(12), eight[7][0]
    falls = np.arange(n) % BLOCK >= BLOCK // 2
    for t in range(3000):
        g = torch.from_numpy((rng.normal(0, 1e-3, n) * np.where(falls & (t >= 1000), 0.1, 1.0)).astype(np.float32))
        for made in (eight, full):
            made[6][0].copy_(g)
            st.st_adamw_step(made[0])
        ref.step(g.double().numpy())
    assert np.array_equal(eight[3][0].cpu().numpy(), ref.cm) and np.array_equal(eight[4][0].cpu().numpy(), ref.cv)
    assert np.array_equal(eight[5][0][0].cpu().numpy(), ref.ms) and np.array_equal(eight[5][1][0].cpu().numpy(), ref.vs)
    m, v = [torch.zeros(n, device="cuda")], [torch.zeros(n, device="cuda")]
    st.st_adamw_read_moments(eight[0], m, v)
    ratio = np.sqrt(f64(v[0]) / f64(full[4][0]))
    assert steady[0] <= np.median(ratio[~falls]) <= steady[1] and shrunk[0] <= np.median(ratio[falls]) <= shrunk[1], (np.median(ratio[~falls]), np.median(ratio[falls]))
    if b2 == 0.99:
        assert np.all(np.abs(ratio[~falls] - 1) <= 0.07)
    off, held = f64(m[0]) - f64(full[3][0]), f64(full[3][0])
    assert np.sqrt(np.mean(off[~falls] ** 2)) <= 0.03 * np.sqrt(np.mean(held[~falls] ** 2))
    assert torch.isfinite(eight[1][0]).all()


@pytest.mark.parametrize("shift", [0, 1])
def test_levels_next_to_their_borders(shift):
    """Second moments whose root lies on a border between two of the upper levels, or up to four steps of fp32 beside it: the levels are those that the
    fp32 operations of the definition give, by the path of whole vectors and by that of single values."""
    f, blocks, b2 = np.float32, 2000, 0.5               # 1 - b2 is exact, and so is its product
    rng = np.random.default_rng(11)
    g = np.empty((blocks, BLOCK), f)
    g[:, 0] = rng.uniform(0.5, 2, blocks).astype(f)
    top = np.sqrt((g[:, 0] * g[:, 0]) * f(1 - b2))      # the block's largest root, and the scale of the step
    scale = (top / f(255 * 255)).astype(f)
    level = rng.integers(150, 254, (blocks, BLOCK - 1)) + 0.5
    root = level ** 2 * scale.astype(np.float64)[:, None]
    near = (root / np.sqrt(1 - b2)).astype(f).view(np.int32) + rng.integers(-4, 5, root.shape)
    g[:, 1:] = near.astype(np.int32).view(f)
    made = make([g.size], 8, shift=shift, b1=0.0, b2=b2, wd=0.0)
    made[6][0].copy_(torch.from_numpy(g.reshape(-1)).cuda())
    made[7][0].step(g.reshape(-1).astype(np.float64))
    st.st_adamw_step(made[0])
    assert np.array_equal(made[4][0].cpu().numpy(), made[7][0].cv) and np.array_equal(made[3][0].cpu().numpy(), made[7][0].cm)
    assert np.array_equal(made[5][1][0].cpu().numpy(), made[7][0].vs)


@pytest.mark.parametrize("bits", [32, 8])
def test_moments_go_out_and_come_back(bits):
    sizes = [5, 1000, 256, 3]
    made = make(sizes, bits, shift=1)
    run_steps(made, "f32", "f32", False, bits, 2)
    opt, _, _, m, v, scales, _, refs = made
    out = [[put(np.full(n, 7.0), "f32", i % 2) for i, n in enumerate(sizes)] for _ in range(2)]
    st.st_adamw_read_moments(opt, *out)
    for i, r in enumerate(refs):
        if bits == 8:
            dm, dr = r.decoded()
            assert np.array_equal(out[0][i].cpu().numpy(), dm) and np.array_equal(out[1][i].cpu().numpy(), dr * dr)
        else:
            assert torch.equal(out[0][i], m[i]) and torch.equal(out[1][i], v[i])
    # into a second optimiser of the same width: the same values; levels of the same width come back exactly
    other = make(sizes, bits, shift=0)
    st.st_adamw_write_moments(other[0], *out)
    back = [[torch.zeros(n, device="cuda") for n in sizes] for _ in range(2)]
    st.st_adamw_read_moments(other[0], *back)
    for i in range(len(sizes)):
        if bits == 32:
            assert torch.equal(back[0][i], out[0][i]) and torch.equal(back[1][i], out[1][i])
        else:           # scale = top / 127^2 again, a rounding up and one down: 2 u; the levels are the same
            assert torch.equal(other[3][i], m[i]) and torch.equal(other[4][i], v[i])
            np.testing.assert_allclose(back[0][i].cpu().numpy(), out[0][i].cpu().numpy(), rtol=4 * U, atol=0)
    # one moment alone, and a tensor left out
    before = [t.clone() for t in other[4]], other[3][2].clone()
    st.st_adamw_write_moments(other[0], [torch.ones(n, device="cuda") if i != 2 else None for i, n in enumerate(sizes)], None)
    assert all(torch.equal(a, b) for a, b in zip(before[0], other[4])) and torch.equal(before[1], other[3][2])


def test_reading_two_moments_into_the_same_place_is_refused():
    opt = make([300, 40], 32)[0]
    out = [torch.full((n,), 7.0, device="cuda") for n in (300, 40, 300, 40)]
    for m, v in ((out[:2], [out[0], out[3]]), ([out[0], out[0][260:]], out[2:]), ([out[0], out[0][:40]], None)):
        with pytest.raises(st.StError) as ei:
            st.st_adamw_read_moments(opt, m, v)
        assert ei.value.status == st.ST_ERR_INVALID_ARG and "overlap" in str(ei.value)
    assert all((o == 7).all() for o in out)
    st.st_adamw_write_moments(opt, [out[0], out[1]], [out[0], out[1]])          # what is only read may be the same
    st.st_adamw_read_moments(opt, [out[0], out[1]], [out[2], out[3]])
    assert all((o == 7).all() for o in out)


def test_values_at_the_ends_of_the_range_step_like_others():
    """Moments that are 0, subnormal or near fp32's end, in one warp with ordinary ones."""
    vals = np.array([0.0, 1e-45, 1e-40, 1.2e-38, 1e-37, 1e-31, 1e-30, 1e-20, 1e-8, 1.0, 1e10, 1e30, 3e38])
    m0, v0 = [x.reshape(-1) for x in np.meshgrid(np.concatenate([-vals, vals]), vals)]
    n = m0.size
    for g0 in (0.0, 1e-3):
        made = make([n], 32, wd=0.0, eps=1e-12, lr=1e-3)
        opt, params, _, m, v, _, grads, refs = made
        st.st_adamw_write_moments(opt, [put(m0, "f32")], [put(v0, "f32")])
        grads[0].fill_(g0)
        r = refs[0]
        r.m, r.v = f64(m[0]), f64(v[0])
        before = f64(params[0])
        st.st_adamw_step(opt)
        r.step(f64(grads[0]))
        tiny = 2.0 ** -149
        assert np.all(np.abs(f64(m[0]) - r.m) <= 5 * U * np.abs(r.m) + 5 * U * g0 + tiny)
        assert np.all(np.abs(f64(v[0]) - r.v) <= 8 * U * r.v + tiny)
        # v of a few subnormal steps has that much relative error, and its root half of it
        rough = 0.5 * tiny / np.maximum(r.v, tiny)
        step = before - r.p
        off = r.bound + rough * np.abs(step) + 4 * U * np.abs(step)
        # quotients m / (sqrt(v) + eps) that fp32 holds: beyond FLT_MAX they are infinite, and so is the step
        ok = np.abs(step) * (1 - 0.9) / 1e-3 < 3.4e38
        assert np.all(np.abs(f64(params[0]) - r.p)[ok] <= off[ok] + tiny)


def test_negative_second_moments_are_taken_as_zero():
    for bits in (32, 8):
        made = make([10], bits)
        st.st_adamw_write_moments(made[0], None, [put(np.linspace(-1, 1, 10), "f32")])
        out = torch.zeros(10, device="cuda")
        st.st_adamw_read_moments(made[0], None, [out])
        assert (f64(out)[:5] == 0).all() and (f64(out)[5:] > 0).all()


def test_gradients_that_are_replaced_stay_until_their_step_is_done(side_stream):
    """The optimiser works on another stream than the one that gradients come from, and is behind: the memory of gradients that it was given before
    does not go to tensors of the other stream meanwhile."""
    n, own = 300_000, torch.cuda.Stream()
    p, m, v = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    before, after = torch.ones(n, device="cuda"), torch.full((n,), 1.0, device="cuda")
    side_stream.synchronize()
    opt = st.st_adamw_create([p], [m], [v], [before], lr=0.1, weight_decay=0.0, cuda_stream=own.cuda_stream)
    st.st_adamw_set_grads(opt, [before])
    st.st_adamw_step(opt)                               # kernels are loaded before the wait
    own.synchronize()
    with torch.cuda.stream(own):
        torch.cuda._sleep(200_000_000)                  # a tenth of a second
    st.st_adamw_step(opt)
    st.st_adamw_set_grads(opt, [after])
    del before
    other = [torch.full((n,), float("nan"), device="cuda") for _ in range(4)]
    side_stream.synchronize()
    assert not own.query()                              # the step has not run yet
    own.synchronize()
    assert torch.isfinite(p).all() and len(other) == 4
    st.st_adamw_destroy(opt)


def test_more_tensors_than_one_launch_can_name():
    n = 1000
    sizes = [1 + i % 7 for i in range(n)]
    made = make(sizes, 32, b2=0.9)
    opt, params, _, m, v, _, grads, refs = made
    rng = np.random.default_rng(4)
    moved = [put(rng.normal(0, 1, s), "f32") for s in sizes]
    st.st_adamw_set_grads(opt, moved)
    st.st_adamw_step(opt)
    out = [torch.zeros(s, device="cuda") for s in sizes]
    st.st_adamw_read_moments(opt, out, None)
    for i in range(n):
        r = refs[i]
        r.step(f64(moved[i]))
        assert np.all(np.abs(f64(params[i]) - r.p) <= r.bound), i
        assert np.all(np.abs(f64(out[i]) - r.m) <= 5 * U * np.abs(r.m)), i


def test_the_norm_is_the_same_every_time():
    made = make([100_000, 7, 333_333], 32)
    new_grads(np.random.default_rng(2), made[6], "f32")
    seen = set()
    for _ in range(5):
        norm = torch.zeros(1, device="cuda")
        st.st_adamw_step(made[0], norm_out=norm)
        seen.add(norm.item())
    assert len(seen) == 1


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_the_norm_does_not_depend_on_where_gradients_lie(kind):
    """The sum of squares is (1 + 2^-24)^2, whose root lies between two fp32 numbers, and four squares that double loses or keeps, depending on what they are added to."""
    u, tiny = 2.0 ** -12, 1.25 * 2.0 ** -27
    up = 1.0 if kind != "f16" else 2.0 ** 14            # fp16 holds nothing below 2^-24
    g = np.zeros(700)
    g[256:264] = np.array([1, u, tiny, tiny, 2.0 ** -24, u, tiny, tiny]) * up
    seen = set()
    for shift in (0, 1, 2, 3, 4, 8):
        made = make([700], 32, grad=kind, shift=shift)
        made[6][0].copy_(torch.from_numpy(g).to(TYPES[kind]).cuda())
        assert np.array_equal(f64(made[6][0]), g)       # the type holds them
        norm = torch.zeros(1, device="cuda")
        st.st_adamw_step(made[0], norm_out=norm)
        seen.add(norm.item())
    assert len(seen) == 1, seen


def test_norm_of_gradients_whose_squares_leave_fp32():
    made = make([64, 64], 32)
    made[6][0].fill_(1e25)
    made[6][1].fill_(1e-30)
    norm = torch.zeros(1, device="cuda")
    st.st_adamw_step(made[0], norm_out=norm)
    assert abs(norm.item() / 8e25 - 1) < 4 * U
    made[6][0].fill_(1e-30)
    st.st_adamw_step(made[0], norm_out=norm)
    assert abs(norm.item() / (1e-30 * np.sqrt(128)) - 1) < 4 * U


def test_captured_steps(side_stream):
    """A captured step counts on when it is replayed, and sees learning rates and gradients set between replays."""
    a, b = make([5000, 40], 8, max_norm=1.0), make([5000, 40], 8, max_norm=1.0)
    rng = np.random.default_rng(6)
    g = new_grads(rng, a[6], "f32")
    for x, y in zip(a[6], b[6]):
        y.copy_(x)
    st.st_adamw_step(a[0]); st.st_adamw_step(b[0])              # modules are loaded before the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side_stream, capture_error_mode="thread_local"):
        st.st_adamw_step(a[0])
        st.st_adamw_step(a[0])
    moved = [torch.randn_like(x) for x in a[6]]
    for k in range(3):
        if k == 1:
            for o in (a, b):
                st.st_adamw_set_lr(o[0], 0.05)
        if k == 2:
            for o in (a, b):
                st.st_adamw_set_grads(o[0], moved)
        graph.replay()
        st.st_adamw_step(b[0]); st.st_adamw_step(b[0])
    assert st.st_adamw_step_count(a[0]) == st.st_adamw_step_count(b[0]) == 7
    for x, y in zip(a[1] + a[3] + a[4], b[1] + b[3] + b[4]):
        assert torch.equal(x, y)


def test_offsets_beyond_32_bits():
    n = 2 ** 31 + 300
    p = torch.full((n,), 0.5, dtype=torch.bfloat16, device="cuda")
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    m, v = torch.zeros(n, dtype=torch.int8, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda")
    s = [torch.zeros(-(-n // BLOCK), device="cuda") for _ in range(2)]
    tail = 1000
    vals = torch.randn(tail, device="cuda").to(torch.bfloat16)
    g[-tail:] = vals
    opt = st.st_adamw_create([p], [m], [v], [g], [s[0]], [s[1]], lr=0.1, weight_decay=0.0, cuda_stream=stream())
    norm = torch.zeros(1, device="cuda")
    st.st_adamw_step(opt, norm_out=norm)
    want = f64(vals)
    assert abs(norm.item() - np.linalg.norm(want)) <= 2 * U * np.linalg.norm(want)
    moved = f64(p[-tail:])
    assert np.all(np.abs(moved - (0.5 - 0.1 * np.sign(want))) <= 2.0 ** -8 * 0.7)       # the first step is lr long
    assert (p[:n - tail] == 0.5).all().item()
    st.st_adamw_destroy(opt)


def test_refusals():
    ok = lambda n=100: torch.zeros(n, device="cuda")  # noqa: E731
    p, m, v, g = ok(), ok(), ok(), ok()

    def refused(*a, **kw):
        with pytest.raises(st.StError) as ei:
            st.st_adamw_create(*a, lr=0.1, cuda_stream=stream(), **kw)
        assert ei.value.status == st.ST_ERR_INVALID_ARG
        return str(ei.value)

    assert "not memory" in refused([p], [m.cpu()], [v], [g])
    assert "not memory" in refused([p], [m], [v], [g.cpu()])
    assert "overlap" in refused([p], [m], [m], [g])
    assert "overlap" in refused([p, p], [m, ok()], [v, ok()], [g, ok()])                # the same tensor twice
    assert "overlap" in refused([p], [m], [v], [p])                                     # a gradient that the step would overwrite
    raw = torch.zeros(404, dtype=torch.uint8, device="cuda")
    assert "overlap" in refused([ok(50)], [raw[:200].view(torch.float32)], [raw[196:396].view(torch.float32)], [ok(50)])
    bad = float("nan")
    assert "finite" in refused([p], [m], [v], [g], weight_decay=bad)
    opt = st.st_adamw_create([p], [m], [v], [g], lr=0.1, cuda_stream=stream())
    for call in (lambda: st.st_adamw_set_lr(opt, -1.0), lambda: st.st_adamw_step(opt, bad), lambda: st.st_adamw_set_grads(opt, [g.cpu()]),
                 lambda: st.st_adamw_set_grads(opt, [m]), lambda: st.st_adamw_step(opt, norm_out=p), lambda: st.st_adamw_read_moments(opt, [v], None),
                 lambda: st.st_adamw_write_moments(opt, [ok().cpu()], None)):
        with pytest.raises(st.StError) as ei:
            call()
        assert ei.value.status == st.ST_ERR_INVALID_ARG and "st_adamw" in st.st_adamw_last_error(opt)
    with pytest.raises(ValueError):
        st.st_adamw_set_grads(opt, [ok(99)])
    with pytest.raises(TypeError):
        st.st_adamw_set_grads(opt, [g.double()])
    st.st_adamw_step(opt)                                                               # nothing above has harmed it
    assert st.st_adamw_step_count(opt) == 1
    st.st_adamw_destroy(opt)
    with pytest.raises(st.StError):
        st.st_adamw_step(opt)
