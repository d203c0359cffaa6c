"""Root-mean-square norms with the residual's addition, their gradient, 8-bit tensors with scales and their products as cases
with a size: plain forms in elementary torch operations, and the calls that a user makes of the lazy arrays' entry points.

A case is a dict of plain values: `kind` names the operator, the rest its sizes and options.  `prepare` makes the
tensors that a program holds before the call, `run` is one pass, `exact` the same values in binary64, written apart.

8-bit values are e4m3 (largest 448).  128 neighbours along the axis that a product sums over share a scale, of a row each ("rows":
scales (M, ceil(K / 128))) or of 128 rows together ("blocks": (ceil(M / 128), ceil(K / 128))): max|x| / 448, 2^-126 at least.  8-bit
results come back as e4m3 tensors beside their scales.  Scales of rows lie with neighbouring rows side by side."""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_contexts = {}


def listed():
    return [
        # the norm before a projection for the new tokens of 8 running sequences: a call whose time is latency
        dict(name="norm_token", kind="norm", dtype="bf16", rows=8, heads=1, d=4096, residual=True, eight=True, offset=0.0),
        # the same for long prompts: the residual stream is read and written, the norm goes to the next product in 8 bits
        dict(name="norm_prompt", kind="norm", dtype="bf16", rows=16384, heads=1, d=8192, residual=True, eight=True, offset=0.0),
        # a norm of every head of the queries, odd counts, weights around zero
        dict(name="norm_heads", kind="norm", dtype="f32", rows=6007, heads=12, d=80, residual=False, eight=False, offset=1.0),
        # training: the gradient through the norm and beside it, sums over all tokens for the weight
        dict(name="grad_train", kind="norm_grad", dtype="bf16", rows=8192, heads=1, d=4096, residual=True, offset=0.0),
        # a small model in float32 at odd sizes
        dict(name="grad_odd", kind="norm_grad", dtype="f32", rows=777, heads=1, d=5003, residual=False, offset=1.0),
        # weights after an optimizer's step, for the gradient of a product's input
        dict(name="quantize_weights", kind="quantize", dtype="bf16", m=14336, k=4096, blocks=True, transposed=True),
        # activations at odd sizes, for the gradient of the weights
        dict(name="quantize_columns", kind="quantize", dtype="f32", m=4099, k=2051, blocks=False, transposed=True),
        # the new tokens of four sequences through a projection: the weights are what is read
        dict(name="product_token", kind="product", m=4, n=14336, k=4096, blocks=True, out="bf16"),
        # a batch of running sequences and pieces of prompts: fewer tiles than compute units
        dict(name="product_batch", kind="product", m=192, n=4096, k=14336, blocks=True, out="bf16"),
        # a long prompt: the matrix cores are the bound
        dict(name="product_prompt", kind="product", m=8192, n=8192, k=8192, blocks=True, out="bf16"),
        # ragged on all sides, in float32
        dict(name="product_odd", kind="product", m=777, n=1291, k=1003, blocks=True, out="f32"),
        # the gradient of the weights: both operands with scales of rows, the tokens are summed over
        dict(name="product_gradient", kind="product", m=4096, n=6144, k=16384, blocks=False, out="f32"),
    ]


def _size(rng, lo, hi):
    """Log-uniform; half of the draws in multiples of 128, as sizes often come, the others as they fall."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if v >= 256 and rng.random() < 1 / 2:
        v = v // 128 * 128
    return max(lo, min(hi, v))


def draw(rng):
    kind = rng.choice(["norm", "norm_grad", "quantize", "product", "product"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "product":
        m, n, k = _size(rng, 1, 8192), _size(rng, 64, 16384), _size(rng, 64, 16384)
        while m * n * k > 1 << 38:
            m = (m + 1) // 2
        return dict(kind=kind, m=m, n=n, k=k, blocks=rng.random() < 0.7, out=rng.choice(["bf16", "bf16", "f32"]))
    if kind == "quantize":
        m, k = _size(rng, 1, 16384), _size(rng, 64, 16384)
        while m * k > 1 << 26:
            m = (m + 1) // 2
        return dict(kind=kind, dtype=dtype, m=m, k=k, blocks=rng.random() < 0.4, transposed=rng.random() < 0.5)
    heads = rng.choice([1, 1, 1, 4, 12, 32])
    d = _size(rng, 64, 16384) if heads == 1 else rng.choice([64, 80, 96, 128, 256])
    rows = max(1, min(_size(rng, 1, 16384), (1 << 26) // (heads * d)))
    case = dict(kind=kind, dtype=dtype, rows=rows, heads=heads, d=d, residual=rng.random() < 0.6, offset=rng.choice([0.0, 0.0, 1.0]))
    if kind == "norm":
        case["eight"] = rng.random() < 0.5
    return case


def _ceil(a, b):
    return (a + b - 1) // b


def _quantized(x, blocks, transposed):
    """(e4m3 values, scales) of x (.., K), in 32 bits."""
    x = x.float()
    if transposed:
        x = x.t()
    k = x.shape[-1]
    wide = torch.nn.functional.pad(x, (0, -k % 128)).unflatten(-1, (-1, 128))   # (.., K / 128, 128)
    top = wide.abs().amax(-1)
    if blocks:
        m = x.shape[0]
        top = torch.nn.functional.pad(top, (0, 0, 0, -m % 128)).unflatten(0, (-1, 128)).amax(1)
    scales = torch.where(top < math.inf, (top / 448.0).clamp(min=2.0 ** -126), math.nan)
    each = scales.repeat_interleave(128, 0)[:x.shape[0]] if blocks else scales
    q = torch.minimum(torch.maximum(wide / each[..., None], torch.tensor(-448.0, device=x.device)), torch.tensor(448.0, device=x.device))
    return q.flatten(-2)[..., :k].to(torch.float8_e4m3fn), scales


def _side_by_side(scales):
    """The same scales with neighbouring rows next to one another in memory."""
    return scales.t().contiguous().t()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(*shape, by=1.0, to=torch.float32):
        return (torch.randn(*shape, generator=g, device="cuda") * by).to(to)

    s = dict(case=case)
    if case["kind"] == "product":
        # rows of different sizes, a few large values among the activations
        m, n, k = case["m"], case["n"], case["k"]
        a = normal(m, k) * torch.exp(normal(m, 1)) * torch.where(torch.rand(1, k, generator=g, device="cuda") < 0.005, 20.0, 1.0)
        b = normal(n, k, by=k ** -0.5)
        s["a"], sa = _quantized(a, False, False)
        s["b"], sb = _quantized(b, case["blocks"], False)
        s["sa"], s["sb"] = _side_by_side(sa), sb if case["blocks"] else _side_by_side(sb)
        return s
    dt = _TYPES[case["dtype"]]
    if case["kind"] == "quantize":
        s["x"] = (normal(case["m"], case["k"]) * torch.exp(normal(case["m"], 1))).to(dt)
        return s
    shape = (case["rows"], case["d"]) if case["heads"] == 1 else (case["rows"], case["heads"], case["d"])
    s["x"] = normal(*shape, to=dt)
    s["weight"] = normal(case["d"], by=0.2) + (1.0 - case["offset"])
    s["residual"] = normal(*shape, by=4.0, to=dt) if case["residual"] else None
    if case["kind"] == "norm_grad":
        s["dout"] = normal(*shape, to=dt)
    return s


EPS = 1e-6


def _plain_norm(case, s):
    got = {}
    total = s["x"]
    if s["residual"] is not None:
        got["total"] = total = (s["x"].float() + s["residual"].float()).to(total.dtype)   # the norm is of the stream as it is stored
    t = total.float()
    y = t * torch.rsqrt((t * t).mean(-1, keepdim=True) + EPS) * (s["weight"] + case["offset"])
    if case["eight"]:
        got["out"], got["scales"] = _quantized(y, False, False)
    else:
        got["out"] = y.to(total.dtype)
    return got


def _plain_norm_grad(case, s):
    t, dout = s["x"].float(), s["dout"].float()
    r = torch.rsqrt((t * t).mean(-1, keepdim=True) + EPS)
    g = dout * (s["weight"] + case["offset"])
    dx = r * g - t * (r * r * r * (g * t).mean(-1, keepdim=True))
    if s["residual"] is not None:
        dx = dx + s["residual"].float()
    return dict(dx=dx.to(s["x"].dtype), dweight=(dout * t * r).flatten(0, -2).sum(0))


def _spread(q, scales, blocks):
    """The values that 8-bit ones stand for, in 32 bits."""
    if blocks:
        scales = scales.repeat_interleave(128, 0)[:q.shape[0]]
    return q.float() * scales.repeat_interleave(128, 1)[:, :q.shape[1]]


def _plain_product(case, s):
    a, b = _spread(s["a"], s["sa"], False), _spread(s["b"], s["sb"], case["blocks"])
    return torch.matmul(a, b.t()).to(_TYPES[case["out"]])


def _context(gr):
    """The program's context, made once on the stream that it works on."""
    stream = torch.cuda.current_stream().cuda_stream
    if stream not in _contexts:
        _contexts[stream] = gr.Context(stream=stream)
    return _contexts[stream]


def _own(case, s):
    from paper_1901_03771_amd import lazy as gr
    ctx = _context(gr)
    wrap = ctx.array
    if case["kind"] == "product":
        out = torch.empty(case["m"], case["n"], device="cuda", dtype=_TYPES[case["out"]])
        gr.dot_scaled(wrap(s["a"]), wrap(s["sa"]), wrap(s["b"]), wrap(s["sb"]), out=wrap(out))
        return out
    if case["kind"] == "quantize":
        m, k = (case["k"], case["m"]) if case["transposed"] else (case["m"], case["k"])
        out = torch.empty(m, k, device="cuda", dtype=torch.float8_e4m3fn)
        scales = torch.empty(_ceil(k, 128), _ceil(m, 128) if case["blocks"] else m, device="cuda").t()
        gr.quantize(wrap(s["x"]), blocks=case["blocks"], transposed=case["transposed"], out=wrap(out), scales=wrap(scales))
        return dict(out=out, scales=scales)
    x, weight = wrap(s["x"]), wrap(s["weight"])
    residual = None if s["residual"] is None else wrap(s["residual"])
    if case["kind"] == "norm_grad":
        dx, dweight = torch.empty_like(s["x"]), torch.empty_like(s["weight"])
        gr.rms_norm_grad(wrap(s["dout"]), x, weight, dtotal=residual, eps=EPS, offset=case["offset"], dx=wrap(dx), dweight=wrap(dweight))
        return dict(dx=dx, dweight=dweight)
    got, more = {}, {}
    if residual is not None:
        got["total"] = torch.empty_like(s["x"])
        more["total"] = wrap(got["total"])
    if case["eight"]:
        got["out"] = torch.empty_like(s["x"], dtype=torch.float8_e4m3fn)
        blocks = _ceil(case["d"], 128)
        if case["heads"] == 1:
            got["scales"] = torch.empty(blocks, case["rows"], device="cuda").t()
        else:
            got["scales"] = torch.empty(blocks, case["rows"], case["heads"], device="cuda").permute(1, 2, 0)
        more["scales"] = wrap(got["scales"])
    else:
        got["out"] = torch.empty_like(s["x"])
    gr.rms_norm(x, weight, residual, eps=EPS, offset=case["offset"], out=wrap(got["out"]), **more)
    return got


def run(state):
    case = state["case"]
    if own:
        return _own(case, state)
    if case["kind"] == "product":
        return _plain_product(case, state)
    if case["kind"] == "quantize":
        out, scales = _quantized(state["x"], case["blocks"], case["transposed"])
        return dict(out=out, scales=scales)
    return _plain_norm(case, state) if case["kind"] == "norm" else _plain_norm_grad(case, state)


def work(case):
    if case["kind"] == "product":
        m, n, k = case["m"], case["n"], case["k"]
        scales = _ceil(k, 128) * (m + (_ceil(n, 128) if case["blocks"] else n))
        return dict(bytes=(m + n) * k + 4 * scales + m * n * (4 if case["out"] == "f32" else 2), flops=2 * m * n * k)
    size = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "quantize":
        values = case["m"] * case["k"]
        return dict(bytes=values * (size + 1) + values / 128 / (128 if case["blocks"] else 1) * 4, flops=3 * values)
    values = case["rows"] * case["heads"] * case["d"]
    if case["kind"] == "norm_grad":
        return dict(bytes=values * size * (4 if case["residual"] else 3) + 8 * case["d"], flops=12 * values)
    out = 1 + 4 / 128 if case["eight"] else size
    return dict(bytes=values * (size * (3 if case["residual"] else 1) + out) + 4 * case["d"], flops=6 * values)


def _exact_quantized(x, blocks):
    """Values over scales, not rounded, and scales, a block at a time."""
    m, k = x.shape
    high = 128 if blocks else 1
    rows = torch.arange(m, device=x.device) // high
    scales = torch.zeros(_ceil(m, high), _ceil(k, 128), dtype=torch.float64, device=x.device)
    values = torch.empty_like(x)
    for j in range(0, k, 128):
        part = x[:, j:j + 128]
        scale = scales[:, j // 128]
        scale.index_reduce_(0, rows, part.abs().max(1)[0] / 448, "amax")
        scale.clamp_(min=2.0 ** -126)
        values[:, j:j + 128] = part / scale[rows][:, None]
    return values, scales


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "product":
        m, n, k = case["m"], case["n"], case["k"]
        total = torch.zeros(m, n, dtype=torch.float64, device="cuda")
        rows = torch.arange(n, device="cuda") // (128 if case["blocks"] else 1)
        step = 2048
        for j in range(0, k, step):
            each = torch.arange(j, min(j + step, k), device="cuda") // 128
            a = s["a"][:, j:j + step].double() * s["sa"].double()[:, each]
            b = s["b"][:, j:j + step].double() * s["sb"].double()[rows][:, each]
            total += a @ b.t().contiguous()
        return total
    if case["kind"] == "quantize":
        x = s["x"].double()
        out, scales = _exact_quantized(x.t().contiguous() if case["transposed"] else x, case["blocks"])
        return dict(out=out, scales=scales)
    d = case["d"]
    x, weight = s["x"].double().reshape(-1, d), s["weight"].double() + case["offset"]
    shape = s["x"].shape
    more = None if s["residual"] is None else s["residual"].double().reshape(-1, d)
    if case["kind"] == "norm_grad":
        dout = s["dout"].double().reshape(-1, d)
        length = torch.sqrt(torch.linalg.vector_norm(x, dim=1) ** 2 / d + EPS)[:, None]
        unit = x / length
        pull = dout * weight
        dx = (pull - unit * (pull * unit).sum(1, keepdim=True) / d) / length
        dx = dx if more is None else dx + more
        return dict(dx=dx.reshape(shape), dweight=torch.linalg.vecdot(dout, unit, dim=0))
    got = {}
    if more is not None:
        x = x + more
        got["total"] = x.reshape(shape)
        x = x.to(s["x"].dtype).double()
    y = x / torch.sqrt(torch.linalg.vector_norm(x, dim=1) ** 2 / d + EPS)[:, None] * weight
    if not case["eight"]:
        return dict(got, out=y.reshape(shape))
    out, scales = _exact_quantized(y, False)
    return dict(got, out=out.reshape(shape), scales=scales.reshape(*shape[:-1], -1))
