"""What the speed of the operators around the distillation step is measured on: the optimiser of the tensors that a context does
not hold (full distillation trains the whole student; a teacher is fine-tuned), and the 8-bit integer layers of the part that is
never trained.

A case is one pass through one of four operators:

  adamw     one AdamW step over many tensors at once, moments in 32 or in 8 bits, with or without the clipping of the gradients'
            norm.  With 8-bit moments the pass also exports them as fp32 values, as a checkpoint does.
  quantise  rows (tokens, pixels, output channels) to 8-bit integers with one scale per row, from row-major tokens or from planar
            feature maps.
  product   8-bit integer matrix product with a scale per token and a scale per output channel, bias and ReLU.
  linear    the two together: a layer of the frozen part on activations that arrive in 16 bits.

With `own` false the operators are computed in their plain form, with elementary torch operations; with `own` true by the
framework's entry points.
"""
import math
import random

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_BLOCK = 256            # moments in 8 bits: values that share a scale


def _adamw(name=None, tensors=2, total=5397, bits=32, param="f32", grad="f32", master=False, clip=0.0, packed=False):
    c = {"op": "adamw", "tensors": tensors, "total": total, "bits": bits, "param": param, "grad": grad, "master": master, "clip": clip,
         "packed": packed}
    return dict(c, name=name) if name else c


def _matrix(op, name=None, m=1, n=256, k=256, x="bf16", y="bf16", bias=True, relu=False, planar=False):
    c = {"op": op, "m": m, "k": k}
    c.update({"x": x, "planar": planar} if op == "quantise" else {"n": n, "y": y, "bias": bias, "relu": relu})
    c.update({"x": x} if op == "linear" else {})
    return dict(c, name=name) if name else c


def listed():
    return [
        # the classifier of the benchmark's head alone (21 x 256 weights, 21 biases): the smallest step there is, its latency
        _adamw("adamw head"),
        # full distillation of the paper's student (0.48 M parameters) in fp32, packed as the update buffer is, gradients clipped
        _adamw("adamw student packed", 97, 480_000, clip=1.0, packed=True),
        # fine-tuning the paper's teacher (44.34 M parameters): bf16 copies for the matrix products, fp32 masters, clipped
        _adamw("adamw teacher master", 161, 44_340_000, param="bf16", grad="bf16", master=True, clip=1.0),
        # a large model in fp32, no clipping: pure streaming
        _adamw("adamw large", 290, 150_000_000),
        # the two-layer head with a 3x3 layer (595,477 parameters), fp16 gradients, moments in 8 bits: small and ragged
        _adamw("adamw 8-bit head", 4, 595_477, bits=8, grad="f16"),
        # a large model whose memory is short: bf16 parameters without masters, moments in 8 bits, clipped
        _adamw("adamw 8-bit large", 290, 200_000_000, bits=8, param="bf16", grad="bf16", clip=1.0),
        # the feature map of a 720p frame as the front part leaves it, planar fp32, to 8-bit pixels
        _matrix("quantise", "quantise 720p planar", m=180 * 320, k=256, x="f32", planar=True),
        # tokens of odd number and width
        _matrix("quantise", "quantise odd rows", m=4099, k=1111, x="bf16"),
        # one token through a wide layer: bound by the weights
        _matrix("product", "product one token", m=1, n=4096, k=4096),
        # a few tokens, odd in every size
        _matrix("product", "product odd few", m=23, n=1000, k=1531, y="f32", relu=True),
        # a pointwise layer of the front part over a 720p feature map: bound by activations
        _matrix("product", "product 720p map", m=180 * 320, n=256, k=512, relu=True),
        # a wide layer over many tokens, quantisation included: bound by the tensor cores
        _matrix("linear", "linear large", m=8192, n=4096, k=4096),
    ]


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(("adamw", "adamw", "quantise", "product", "product", "linear"))
    if op == "adamw":
        bits = rng.choice((32, 32, 8))
        total = _log_int(rng, 5_000, 120_000_000)
        param = rng.choice(("f32", "f32", "bf16", "f16"))
        return _adamw(None, min(_log_int(rng, 1, 300), total // 64), total, bits, param, rng.choice((param, "f32", "bf16", "f16")),
                      param != "f32" and rng.random() < 0.6, rng.choice((0.0, 0.5, 1.0)), bits == 32 and rng.random() < 0.3)
    if op == "quantise":
        m = _log_int(rng, 1, 100_000)
        return _matrix(op, None, m, k=min(_log_int(rng, 16, 8192), 64_000_000 // m), x=rng.choice(("f32", "bf16", "f16")), planar=rng.random() < 0.4)
    m, n, k = _log_int(rng, 1, 60_000), _log_int(rng, 16, 8192), _log_int(rng, 32, 8192)
    most = 8192 * 4096 * 4096
    while m * n * k > most or m * (n + k) > 150_000_000:
        m, n, k = (m + 1) // 2, (n + 15) // 2, (k + 31) // 2
    return _matrix(op, None, m, n, k, rng.choice(("bf16", "f16", "f32")), rng.choice(("bf16", "bf16", "f16", "f32")), rng.random() < 0.7, rng.random() < 0.4)


# ---------------------------------------------------------------------------- inputs
def _sizes(case):
    """Sizes of the case's tensors: spread like a network's layers, one value at least, `total` together."""
    n, total = case["tensors"], case["total"]
    rng = random.Random(n * 1_000_003 + total)
    w = [math.exp(rng.gauss(0, 2)) for _ in range(n)]
    sizes = [1 + int((total - n) * x / sum(w)) for x in w]
    sizes[0] += total - sum(sizes)
    return sizes


def _places(case):
    """Where each tensor begins in the flat buffers: back to back, or at multiples of 256 values as an allocator would put them."""
    sizes, at, places = _sizes(case), 0, []
    for s in sizes:
        places.append(at)
        at += s if case["packed"] else -(-s // _BLOCK) * _BLOCK
    return sizes, places, -(-at // _BLOCK) * _BLOCK


_LR, _B1, _B2, _EPS, _WD, _STEPS = 1e-3, 0.9, 0.999, 1e-8, 0.01, 200


def _prepare_adamw(case, gen):
    sizes, places, flat = _places(case)
    dev = "cuda"
    used = torch.zeros(flat, dtype=torch.bool, device=dev)
    for s, p in zip(sizes, places):
        used[p:p + s] = True

    def normal(std):
        return torch.randn(flat, generator=gen, device=dev).mul_(std).mul_(used)

    state = {"op": "adamw", "case": case, "t": _STEPS, "scale": 1.0}
    value = normal(0.02)
    state["param"] = value.to(_TYPES[case["param"]])
    state["master"] = value if case["master"] else None
    # gradients of layers differ in size; a tenth of them are zero (inactive units)
    grad = normal(1e-3).mul_(torch.rand(flat, generator=gen, device=dev) < 0.9)
    state["grad"] = grad.to(_TYPES[case["grad"]])
    del grad
    if case["bits"] == 32:
        state["m"] = normal(3e-4)
        state["v"] = normal(1e-3).square_()
    else:
        state["m"] = torch.randn(flat, generator=gen, device=dev).mul_(40).round_().clamp_(-127, 127).mul_(used).to(torch.int8)
        state["v"] = torch.randint(1, 256, (flat,), generator=gen, device=dev, dtype=torch.int16).mul_(used).to(torch.uint8)
        n = flat // _BLOCK
        state["m_scale"] = torch.randn(n, generator=gen, device=dev).mul_(0.5).exp_().mul_(3e-3 / 127 ** 2)
        state["v_scale"] = torch.randn(n, generator=gen, device=dev).mul_(0.5).exp_().mul_(4e-3 / 255 ** 2)
    state["norm"] = torch.zeros(1, device=dev)
    del used, value
    if own:
        import paper_2003_10735_b200 as st

        def views(t, of=1):
            return None if t is None else [t[p // of:p // of + -(-s // of)] for s, p in zip(sizes, places)]

        eight = case["bits"] == 8
        state["opt"] = st.st_adamw_create(
            params=views(state["param"]), grads=views(state["grad"]), exp_avg=views(state["m"]), exp_avg_sq=views(state["v"]),
            exp_avg_scale=views(state["m_scale"], _BLOCK) if eight else None,
            exp_avg_sq_scale=views(state["v_scale"], _BLOCK) if eight else None, masters=views(state["master"]), lr=_LR, beta1=_B1,
            beta2=_B2, eps=_EPS, weight_decay=_WD, max_norm=case["clip"], first_step=_STEPS, cuda_stream=torch.cuda.current_stream().cuda_stream)
        if eight:
            state["m_out"], state["v_out"] = torch.zeros(flat, device=dev), torch.zeros(flat, device=dev)
            state["out_views"] = views(state["m_out"]), views(state["v_out"])
    return state


def _pitch(k):
    """Rows of 8-bit integers begin at multiples of 16 bytes."""
    return -(-k // 16) * 16


def _integers(rows, cols, gen):
    q = torch.zeros(rows, _pitch(cols), dtype=torch.int8, device="cuda")
    q[:, :cols] = torch.randn(rows, cols, generator=gen, device="cuda").mul_(36).round_().clamp_(-127, 127).to(torch.int8)
    return q[:, :cols]


def _activations(case, gen):
    """Activations behind a ReLU-like unit with a few large channels, as they reach a layer."""
    m, k = case["m"], case["k"]
    shape = (k, m) if case.get("planar") else (m, k)
    x = torch.randn(shape, generator=gen, device="cuda")
    big = torch.rand(k, generator=gen, device="cuda").mul_(3).exp_()
    x.mul_(big[:, None] if case.get("planar") else big)
    x = torch.where(x > 0, x, x * 0.1).to(_TYPES[case["x"]])
    return x.t() if case.get("planar") else x


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    if case["op"] == "adamw":
        return _prepare_adamw(case, gen)
    state = {"op": case["op"], "case": case}
    m, k = case["m"], case["k"]
    if case["op"] in ("quantise", "linear"):
        state["x"] = _activations(case, gen)
        state["q"] = torch.zeros(m, _pitch(k), dtype=torch.int8, device="cuda")[:, :k]
        state["q_scale"] = torch.zeros(m, device="cuda")
    else:
        state["q"] = _integers(m, k, gen)
        state["q_scale"] = torch.rand(m, generator=gen, device="cuda").add_(0.2).mul_(0.02)
    if case["op"] != "quantise":
        n = case["n"]
        state["w"] = _integers(n, k, gen)
        state["w_scale"] = torch.rand(n, generator=gen, device="cuda").add_(0.2).mul_(0.03 / math.sqrt(k))
        state["bias"] = torch.randn(n, generator=gen, device="cuda") if case["bias"] else None
        state["y"] = torch.zeros(m, n, dtype=_TYPES[case["y"]], device="cuda")
    return state


# ---------------------------------------------------------------------------- plain forms
def _nearest_level(r, scale, most):
    """The level c = 0..most whose c^2 * scale is nearest in the root: c = floor(sqrt(r / scale) + 1/2), in 64 bits next to the borders."""
    inv = torch.where(scale > 0, 1 / scale, 0.0)
    return (r * inv).double().sqrt_().add_(0.5).floor_().clamp_(max=most).float()


def _plain_adamw(s):
    case = s["case"]
    s["t"] += 1
    t = s["t"]
    lr1, r2 = _LR / (1 - _B1 ** t), 1 / math.sqrt(1 - _B2 ** t)
    g = s["grad"].float()
    if case["clip"]:
        norm = g.double().square().sum().sqrt()
        g = g * (case["clip"] / (norm + 1e-6)).clamp(max=1.0).float()
        s["norm"].copy_(norm)
    if case["bits"] == 8:
        cm, cv = s["m"].float().view(-1, _BLOCK), s["v"].float().view(-1, _BLOCK)
        m, root = cm * cm.abs() * s["m_scale"][:, None], cv * cv * s["v_scale"][:, None]
        m, v = m.view(-1), (root * root).view(-1)
    else:
        m, v = s["m"], s["v"]
    m = m * _B1 + g * (1 - _B1)
    v = v * _B2 + (g * g) * (1 - _B2)
    root = v.sqrt()
    p = s["master"] if s["master"] is not None else s["param"].float()
    p = p * (1 - _LR * _WD) - lr1 * m / (root * r2 + _EPS)
    s["param"].copy_(p)
    if s["master"] is not None:
        s["master"].copy_(p)
    out = {"param": s["param"], "master": s["master"], "norm": s["norm"] if case["clip"] else None}
    if case["bits"] == 32:
        s["m"].copy_(m)
        s["v"].copy_(v)
        return dict(out, m=s["m"], v=s["v"])
    m, root = m.view(-1, _BLOCK), root.view(-1, _BLOCK)
    top, top_root = m.abs().amax(1), root.amax(1)
    m_scale = torch.where(top < 2.0 ** -100, 0.0, (top.double() / 127 ** 2).float())
    v_scale = (top_root.double() / 255 ** 2).float()
    cm = _nearest_level(m.abs(), m_scale[:, None], 127) * m.sign()
    cv = _nearest_level(root, v_scale[:, None], 255)
    cv = torch.where(root > 0, cv.clamp(min=1), cv)
    s["m"].copy_(cm.view(-1))
    s["v"].copy_(cv.view(-1))
    s["m_scale"].copy_(m_scale)
    s["v_scale"].copy_(v_scale)
    root = cv * cv * v_scale[:, None]
    return dict(out, m=(cm * cm.abs() * m_scale[:, None]).view(-1), v=(root * root).view(-1))


def _plain_quantise(x):
    scale = (x.float().abs().amax(1).double() / 127).float()
    q = torch.where(scale[:, None] > 0, x.double() / scale.double()[:, None], 0.0)      # 64 bits: values next to a border
    return q.round_().clamp_(-127, 127).to(torch.int8), scale


def _plain_product(s, q, scale):
    y = (q.float() @ s["w"].float().t()) * scale[:, None] * s["w_scale"]
    if s["bias"] is not None:
        y = y + s["bias"]
    if s["case"]["relu"]:
        y = y.clamp(min=0)
    return y.to(s["y"].dtype)


def _plain(s):
    if s["op"] == "adamw":
        return _plain_adamw(s)
    if s["op"] == "quantise":
        q, scale = _plain_quantise(s["x"])
        return {"q": q, "scale": scale}         # the integers themselves are the result: they have to be equal
    if s["op"] == "linear":
        return {"y": _plain_product(s, *_plain_quantise(s["x"]))}
    return {"y": _plain_product(s, s["q"], s["q_scale"])}


# ---------------------------------------------------------------------------- one pass
def run(s):
    if not own:
        return _plain(s)
    import paper_2003_10735_b200 as st
    stream = torch.cuda.current_stream().cuda_stream
    if s["op"] == "adamw":
        clip = s["case"]["clip"]
        st.st_adamw_step(s["opt"], norm_out=s["norm"] if clip else None)
        out = {"param": s["param"], "master": s["master"], "norm": s["norm"] if clip else None}
        if s["case"]["bits"] == 32:
            return dict(out, m=s["m"], v=s["v"])
        st.st_adamw_read_moments(s["opt"], *s["out_views"])
        return dict(out, m=s["m_out"], v=s["v_out"])
    if s["op"] in ("quantise", "linear"):
        st.st_quantize_rows(s["x"], s["q"], s["q_scale"], cuda_stream=stream)
        if s["op"] == "quantise":
            return {"q": s["q"], "scale": s["q_scale"]}
    st.st_int8_matmul(s["q"], s["q_scale"], s["w"], s["w_scale"], s["y"], bias=s["bias"], relu=s["case"]["relu"], cuda_stream=stream)
    return {"y": s["y"]}


def work(case):
    if case["op"] == "adamw":
        n = case["total"]
        size = {"f32": 4, "bf16": 2, "f16": 2}
        per = size[case["grad"]] + (size[case["param"]] + 8 if case["master"] else 2 * size[case["param"]])
        per += 16 if case["bits"] == 32 else 4 + 16 / _BLOCK + 8
        return {"bytes": n * per, "flops": n * 15}
    m, k = case["m"], case["k"]
    size = {"f32": 4, "bf16": 2, "f16": 2}
    if case["op"] == "quantise":
        return {"bytes": m * k * (size[case["x"]] + 1) + 4 * m, "flops": 3 * m * k}
    n = case["n"]
    read = m * k * (size[case["x"]] if case["op"] == "linear" else 1) + n * k + 4 * (m + n) + (4 * n if case["bias"] else 0)
    return {"bytes": read + m * n * size[case["y"]], "flops": 2 * m * n * k}


# ---------------------------------------------------------------------------- 64 bits
def _f32(x):
    return x.float().double()


def _exact_adamw(s, case):
    """Moments that are held in 8 bits are defined by fp32 operations, each rounded (the level of a value next to a border depends on
    it), so those roundings are made here too; parameters follow from the moments without rounding."""
    t = _STEPS + 1
    g = s["grad"].double()
    out = {"norm": None}
    factor = 1.0
    if case["clip"]:
        out["norm"] = torch.linalg.vector_norm(g).reshape(1)
        factor = min(1.0, float(case["clip"] / (out["norm"] + 1e-6)))
        factor = float(torch.tensor(factor, dtype=torch.float32)) if case["bits"] == 8 else factor
    g = g * factor
    value = (s["master"] if s["master"] is not None else s["param"]).double()
    if case["bits"] == 32:
        out["m"] = torch.lerp(g, s["m"].double(), _B1)
        out["v"] = torch.lerp(g * g, s["v"].double(), _B2)
        m, root = out["m"], out["v"].sqrt()
    else:
        g = _f32(g)

        def old(codes, scale):
            c = codes.double().view(-1, _BLOCK)
            return _f32(c * c.abs() * scale.double()[:, None])

        def mix(a, b, beta):
            keep, take = (torch.tensor([beta, 1 - beta], dtype=torch.float32)).double().tolist()
            return _f32(_f32(a * keep) + _f32(b * take))

        g = g.view(-1, _BLOCK)
        m = mix(old(s["m"], s["m_scale"]), g, _B1)
        root = old(s["v"], s["v_scale"])
        root = _f32(mix(_f32(root * root), _f32(g * g), _B2).sqrt())

        def held(a, most, low):
            scale = _f32(a.amax(1, keepdim=True) / most ** 2)
            scale[a.amax(1, keepdim=True) < low] = 0
            ratio = _f32(a * _f32(torch.where(scale > 0, 1 / scale, 0)))
            c = torch.minimum((ratio.sqrt() + 0.5).floor(), torch.full_like(ratio, most))
            return c, scale

        c, scale = held(m.abs(), 127, 2.0 ** -100)
        out["m"] = (c * c * scale * m.sign()).view(-1)
        c, scale = held(root, 255, 0.0)
        c[(root > 0) & (c == 0)] = 1
        out["v"] = (c * c * scale).square().view(-1)
        m, root = m.view(-1), root.view(-1)
    p = value - _LR * _WD * value - _LR / (1 - _B1 ** t) * m / (root / math.sqrt(1 - _B2 ** t) + _EPS)
    out["param"], out["master"] = p, p if s["master"] is not None else None
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "adamw":
        return _exact_adamw(s, case)
    if case["op"] in ("quantise", "linear"):
        x = s["x"].double()
        scale = _f32(torch.linalg.vector_norm(x, ord=math.inf, dim=1) / 127)
        q = torch.div(x, scale[:, None]).nan_to_num_(0.0).round_().clamp_(-127, 127)
        if case["op"] == "quantise":
            return {"q": q.to(torch.int8), "scale": scale}
    else:
        q, scale = s["q"].double(), s["q_scale"].double()
    y = torch.einsum("mk,nk->mn", q, s["w"].double())
    y = y * scale[:, None] * s["w_scale"].double()
    if case["bias"]:
        y = y + s["bias"].double()
    return {"y": y.relu() if case["relu"] else y}
