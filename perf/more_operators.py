"""Performance cases of the operators that make a GNN of many layers trainable and cheap to serve: root-mean-square norm with the residual's addition, forward and
backward, the same norm with its output in 8 bits, products of such 8-bit rows, and an AdamW step over all parameters with states in 32 or 8 bits.

A case is one call (`kind`) with its sizes; `dtype` is the type of the matrices (of a product: of its result, of a step: of the gradients).  Graphs of the benchmark give the sizes:
one graph of 74 nodes, power-law graphs of 56 944 nodes, community graphs of 232 965 nodes, widths 16 to 1024.

8 bits: elements of 4 exponent and 3 mantissa bits (float8_e4m3fn) with one power of two (float8_e8m0fnu) for every 32 columns of a row, or 32 elements of a tensor.  Both are returned
as tensors of those types, whose values they stand for.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZES = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-6
LR, BETA1, BETA2, ADAM_EPS, DECAY, MAX_NORM = 1e-3, 0.9, 0.999, 1e-8, 0.01, 1.0


def listed():
    return [
        # one node asked for at inference, its features and what the layer before adds to them: launches and latency are the whole time
        dict(name="rms_node", kind="rms", n=1, d=128, dtype="f32", residual=True),
        # all nodes of a community graph between two layers, half precision
        dict(name="rms_nodes_bf16", kind="rms", n=232965, d=128, dtype="bf16", residual=True),
        # the same between two layers that are served in 8 bits, wider
        dict(name="rms_fp8_nodes_bf16", kind="rms_fp8", n=232965, d=256, dtype="bf16", residual=True),
        # an odd width on the power-law graph, the first layer: nothing to add yet
        dict(name="rms_fp8_odd", kind="rms_fp8", n=56944, d=251, dtype="f32", residual=False),
        # backward, with a gradient that arrives along the residual: the widest features of the sweep, and an odd width in half precision
        dict(name="rms_grad_wide", kind="rms_grad", n=65536, d=512, dtype="f32", residual=True),
        dict(name="rms_grad_odd_bf16", kind="rms_grad", n=56944, d=251, dtype="bf16", residual=False),
        # a product of one node's row, of odd widths on the power-law graph, and of a large batch of wide rows
        dict(name="product_node", kind="product", n=1, d=512, k=512, dtype="f32"),
        dict(name="product_odd", kind="product", n=56944, d=251, k=74, dtype="f32"),
        dict(name="product_wide_bf16", kind="product", n=131072, d=1024, k=1024, dtype="bf16"),
        # the step of a 2-layer GCN; of 8 layers behind a table of all nodes' rows; of the same with states in 8 bits
        dict(name="adamw_gcn", kind="adamw", rows=0, d=64, layers=2, dtype="f32", bits=32, copies=False, clipped=True),
        dict(name="adamw_table", kind="adamw", rows=232965, d=128, layers=8, dtype="f32", bits=32, copies=False, clipped=True),
        dict(name="adamw_table_8bit", kind="adamw", rows=232965, d=128, layers=8, dtype="bf16", bits=8, copies=True, clipped=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rms", "rms_fp8", "rms_grad", "product", "product", "adamw", "adamw"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    if kind == "adamw":
        return dict(kind=kind, rows=rng.choice([0, _log_int(rng, 64, 232965)]), d=_log_int(rng, 8, 128), layers=rng.randint(1, 12), dtype=dtype,
                    bits=rng.choice([8, 32]), copies=dtype != "f32" and rng.random() < 0.5, clipped=rng.random() < 0.7)
    n = _log_int(rng, 1, 400000)
    if kind == "product":
        d = min(_log_int(rng, 16, 2048), max(16, 120000000 // n))
        return dict(kind=kind, n=n, d=d, k=min(_log_int(rng, 16, 2048), max(16, min(120000000 // n, (1 << 37) // (n * d)))), dtype=dtype)
    d = min(_log_int(rng, 8, 4096), max(8, 40000000 // n))
    return dict(kind=kind, n=n, d=d, dtype=dtype, residual=rng.random() < 0.7)


# ------------------------------------------------------------------------------------------------ inputs

def _shapes(case):
    """Parameter shapes of a model: a table, per layer a norm's weight and a square matrix, a last norm and a matrix of 44 classes."""
    d = case["d"]
    return [(case["rows"], d)] * (case["rows"] > 0) + [(d,), (d, d)] * case["layers"] + [(d,), (d, 44)]


def _counts(case):
    return [math.prod(s) for s in _shapes(case)]


def _blocks(count):
    return (count + 31) // 32


def _amounts(v, d):
    """|v| [rows, d] in blocks of 32 columns [rows, blocks, 32], zeros behind the last."""
    return torch.nn.functional.pad(v.abs(), (0, _blocks(d) * 32 - d)).reshape(v.shape[0], _blocks(d), 32)


def _exponents(v, d):
    """The smallest e >= -127 for every block with its largest amount at most 448 * 2^e; 0 for blocks of zeros."""
    fraction, exponent = torch.frexp(_amounts(v, d).amax(2))            # fraction * 2^exponent, fraction in [0.5, 1)
    return torch.where(fraction == 0, 0, (exponent - 9 + (fraction > 448 / 512)).clamp(min=-127))


def _columns(e, d):
    return e.repeat_interleave(32, 1)[:, :d]


def _nearest(v):
    """Rows in 8 bits, to the nearest: elements and powers of two."""
    d = v.shape[1]
    e = _exponents(v, d)
    return torch.ldexp(v, -_columns(e, d)).to(torch.float8_e4m3fn), torch.ldexp(torch.ones_like(e, dtype=torch.float32), e).to(torch.float8_e8m0fnu)


def _values(codes, scales):
    """float32 of rows in 8 bits."""
    return codes.float() * _columns(scales.float(), codes.shape[1])


def _aligned(codes):
    """Rows that begin at multiples of 16 bytes, as the norm leaves them."""
    n, d = codes.shape
    out = torch.zeros(n, (d + 15) // 16 * 16, dtype=codes.dtype, device=codes.device)
    out[:, :d] = codes
    return out[:, :d]


def _views(flat, sizes, shapes=None):
    parts = torch.split(flat, sizes)
    return list(parts) if shapes is None else [p.view(s) for p, s in zip(parts, shapes)]


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    normal = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")   # noqa: E731
    dtype, kind = DTYPES[case["dtype"]], case["kind"]
    if kind == "adamw":
        # flat buffers hold all parameters, gradients and states end to end, the tensors are views of them
        shapes, counts = _shapes(case), _counts(case)
        total = sum(counts)
        g = (1e-2 * normal(total) * torch.exp(normal(total))).to(dtype)
        data = dict(p=0.1 * normal(total), g=g, norm=g.double().norm().float(), step=int(seed) % 1000 + 10, shapes=shapes, counts=counts)
        if case["dtype"] != "f32" and not case["copies"]:
            data["p"] = data["p"].to(dtype)
        if case["copies"]:
            data["copy"] = data["p"].to(dtype)
        m, r = 3e-3 * normal(total), 1e-2 * torch.exp(0.5 * normal(total))
        if case["bits"] == 32:
            return dict(data, m=m, v=r * r)
        parts = [[_nearest(x[None]) for x in torch.split(s, counts)] for s in (m, r)]
        codes = [torch.cat([c[0] for c, _ in part]) for part in parts]
        scales = [torch.cat([s[0] for _, s in part]) for part in parts]
        return dict(data, m=codes[0], v=codes[1], m_scales=scales[0], v_scales=scales[1])
    n, d = case["n"], case["d"]
    if kind == "product":
        x, x_scales = _nearest(normal(n, d) * torch.exp(0.3 * normal(n, 1)))
        w, w_scales = _nearest(normal(case["k"], d) * d ** -0.5)
        return dict(x=_aligned(x), x_scales=x_scales, w=_aligned(w), w_scales=w_scales)
    data = dict(x=(1.5 * normal(n, d)).to(dtype), weight=1.0 + 0.1 * normal(d))
    if kind == "rms_grad":
        data.update(gy=normal(n, d).to(dtype), rstd=(data["x"].double().square().mean(1) + EPS).rsqrt().float())
    if case["residual"]:
        data["residual"] = (0.5 * normal(n, d)).to(dtype)        # backward: the gradient that arrives at the sum
    return data


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=case)
    if case["kind"] == "adamw":
        counts, blocks = s["counts"], [_blocks(c) for c in s["counts"]]
        s["params"], s["grads"] = _views(s["p"], counts, s["shapes"]), _views(s["g"], counts, s["shapes"])
        s["ms"], s["vs"] = _views(s["m"], counts, s["shapes"]), _views(s["v"], counts, s["shapes"])
        s["copies"] = _views(s["copy"], counts, s["shapes"]) if "copy" in s else None
        s["m_blocks"], s["v_blocks"] = (_views(s[k], blocks) if k in s else None for k in ("m_scales", "v_scales"))
    return s


# ------------------------------------------------------------------------------------------------ one pass

def _step_outputs(s):
    return {k: s[k] for k in ("p", "m", "v", "m_scales", "v_scales", "copy") if k in s}


def _run_own(s):
    from paper_1906_03707_amd import binding
    case = s["case"]
    kind = case["kind"]
    if kind == "rms":
        return binding.rms_norm(s["x"], s["weight"], eps=EPS, residual=s.get("residual"))
    if kind == "rms_fp8":
        return binding.rms_norm_fp8(s["x"], s["weight"], eps=EPS, residual=s.get("residual"))
    if kind == "rms_grad":
        return binding.rms_norm_grad(s["gy"], s["x"], s["rstd"], s["weight"], g_h=s.get("residual"))
    if kind == "product":
        return binding.fp8_product(s["x"], s["x_scales"], s["w"], s["w_scales"], dtype=DTYPES[case["dtype"]])
    s["step"] += 1
    binding.adamw(s["params"], s["grads"], s["ms"], s["vs"], s["step"], lr=LR, betas=(BETA1, BETA2), eps=ADAM_EPS, weight_decay=DECAY,
                  norm=s["norm"] if case["clipped"] else None, max_norm=MAX_NORM if case["clipped"] else None,
                  copies=s["copies"], m_scales=s["m_blocks"], v_scales=s["v_blocks"])
    return _step_outputs(s)


def _mixed(x):
    """32 bits that depend on all bits of the whole numbers x (of which the low 32 bits count)."""
    x = x & 0xFFFFFFFF
    x = (x ^ (x >> 15)) * 0x6A09E667 & 0xFFFFFFFF
    x = (x ^ (x >> 13)) * 0xBB67AE85 & 0xFFFFFFFF
    return x ^ (x >> 16)


def _thresholds(count, step):
    """16 random bits for the first and for the second moment of every element; the seed is 0."""
    key = _mixed(torch.tensor((0 + step * 0x9E3779B1) & 0xFFFFFFFF, device="cuda"))
    x = _mixed(torch.arange(count, device="cuda") * 0x9E3779B1 + key)
    return x & 0xFFFF, x >> 16


def _dithered(v, random, keep):
    """A tensor's elements in 8 bits, up where the part that is cut off, in 2^-16 of a step, and the random bits with a half carry over; keep: what is not zero does not become it."""
    count = v.numel()
    e = _exponents(v[None], count)
    small = torch.ldexp(v.abs(), -_columns(e, count)[0]) * 2.0 ** -120       # float32's exponent is 120 above e4m3's
    codes = (small.view(torch.int32) + (random * 16 + 8).int()) >> 20
    codes = torch.where((v != 0) & keep, codes.clamp(min=1), codes) | (torch.signbit(v).int() << 7)
    return codes.to(torch.uint8).view(torch.float8_e4m3fn), torch.ldexp(torch.ones_like(e, dtype=torch.float32), e)[0].to(torch.float8_e8m0fnu)


def _step_plain(s):
    case = s["case"]
    s["step"] += 1
    t, counts = s["step"], s["counts"]
    g = s["g"].float()
    if case["clipped"]:
        g = (g.double() * (MAX_NORM / s["norm"].double()).clamp(max=1.0)).float()
    m, v = s["m"], s["v"]
    if case["bits"] == 8:
        m, v = (torch.cat([_values(c[None], b[None])[0] for c, b in zip(torch.split(s[k], counts), s[k + "_blocks"])]) for k in ("m", "v"))
    m = BETA1 * m + (1 - BETA1) * g
    if case["bits"] == 8:
        root = torch.sqrt(BETA2 * (v * v) + (1 - BETA2) * (g * g))
    else:
        v = BETA2 * v + (1 - BETA2) * (g * g)
        root = v.sqrt()
    p = s["p"].float() * (1 - LR * DECAY) - LR / (1 - BETA1 ** t) * m / (root / math.sqrt(1 - BETA2 ** t) + ADAM_EPS)
    s["p"].copy_(p)
    if case["copies"]:
        s["copy"].copy_(p)
    if case["bits"] == 32:
        s["m"].copy_(m)
        s["v"].copy_(v)
        return _step_outputs(s)
    random = _thresholds(max(counts), t)
    for key, moment, bits in (("m", m, random[0]), ("v", root, random[1])):
        parts = [_dithered(x, bits[:x.numel()], key == "v") for x in torch.split(moment, counts)]
        s[key].copy_(torch.cat([c for c, _ in parts]))
        s[key + "_scales"].copy_(torch.cat([e for _, e in parts]))
    return _step_outputs(s)


def _run_plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "adamw":
        return _step_plain(s)
    if kind == "product":
        return (_values(s["x"], s["x_scales"]) @ _values(s["w"], s["w_scales"]).t()).to(DTYPES[case["dtype"]])
    if kind == "rms_grad":
        rstd, gy = s["rstd"][:, None], s["gy"].float()
        xh = s["x"].float() * rstd
        u = gy * s["weight"]
        gx = rstd * (u - xh * (u * xh).mean(1, keepdim=True))
        if case["residual"]:
            gx = gx + s["residual"].float()
        return gx.to(s["x"].dtype), (gy * xh).sum(0)
    h = (s["x"].float() + s["residual"].float()).to(s["x"].dtype) if case["residual"] else s["x"]
    rstd = (h.float().square().mean(1) + EPS).rsqrt()
    y = h.float() * rstd[:, None] * s["weight"]
    return (y.to(h.dtype), h, rstd) if kind == "rms" else (*_nearest(y), h)


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------------------------------------ cost and exact results

def work(case):
    kind, size = case["kind"], SIZES[case["dtype"]]
    if kind == "adamw":
        count, blocks = sum(_counts(case)), sum(_blocks(c) for c in _counts(case))
        p = 4 if case["copies"] else size
        states = 16 * count if case["bits"] == 32 else 4 * count + 4 * blocks
        return dict(bytes=count * (2 * p + size + size * case["copies"]) + states, flops=15 * count)
    n, d, residual = case["n"], case["d"], case["residual"] if kind != "product" else False
    if kind == "product":
        k = case["k"]
        return dict(bytes=(n + k) * (d + _blocks(d)) + n * k * size, flops=2 * n * d * k)
    if kind == "rms_grad":
        return dict(bytes=(3 + residual) * n * d * size + 4 * n + 8 * d, flops=(10 + residual) * n * d)
    out = n * d * size + 4 * n if kind == "rms" else n * (d + _blocks(d))
    return dict(bytes=(1 + 2 * residual) * n * d * size + out + 4 * d, flops=(4 + residual) * n * d)


def _exact_8bit(v, random=None, keep=False):
    """Elements and powers of two of the rows of v in 64 bits, to the nearest (ties to even) or with the thresholds `random`."""
    d = v.shape[1]
    a = torch.nn.functional.pad(v.abs(), (0, -d % 32)).unflatten(1, (-1, 32)).amax(2)
    scale = torch.where(a == 0, 1.0, torch.exp2(torch.ceil(torch.log2(a / 448)).clamp(min=-127)))
    y = v / scale.repeat_interleave(32, 1)[:, :d]
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    if random is None:
        return torch.round(y / step) * step, scale
    q = torch.floor(y.abs() / step + (random + 0.5) / 65536) * step
    if keep:
        q = torch.where(y != 0, q.clamp(min=2.0 ** -9), q)
    return torch.copysign(q, y), scale


def _exact_step(case, s):
    counts, t = s["counts"], s["step"] + 1
    g, p = s["g"].double(), s["p"].double()
    if case["clipped"]:
        g = g * min(1.0, MAX_NORM / s["norm"].item())
    if case["bits"] == 8:
        scales = [torch.split(s[k], [_blocks(c) for c in counts]) for k in ("m_scales", "v_scales")]
        m, v = (torch.cat([c.double() * b.double().repeat_interleave(32)[:c.numel()] for c, b in zip(torch.split(s[k], counts), of)]) for k, of in zip("mv", scales))
        v = v.square()
    else:
        m, v = s["m"].double(), s["v"].double()
    m, v = torch.lerp(g, m, BETA1), torch.lerp(g.square(), v, BETA2)
    update = (m / -math.expm1(t * math.log(BETA1))) / ((v / -math.expm1(t * math.log(BETA2))).sqrt() + ADAM_EPS)
    p = p - LR * (update + DECAY * p)
    out = dict(p=p, copy=p) if case["copies"] else dict(p=p)
    if case["bits"] == 32:
        return dict(out, m=m, v=v)
    random = _thresholds(max(counts), t)
    for key, moment, bits in (("m", m, random[0]), ("v", v.sqrt(), random[1])):
        parts = [_exact_8bit(x[None], bits[:x.numel()], key == "v") for x in torch.split(moment, counts)]
        out[key], out[key + "_scales"] = (torch.cat([part[k][0] for part in parts]) for k in range(2))
    return out


def exact(case, seed):
    s, kind = _inputs(case, seed), case["kind"]
    if kind == "adamw":
        return _exact_step(case, s)
    if kind == "product":
        x, w = (s[k].double() * torch.repeat_interleave(s[k + "_scales"].double(), 32, 1)[:, :case["d"]] for k in "xw")
        return torch.matmul(x, w.t().contiguous())
    w, d = s["weight"].double(), case["d"]
    if kind == "rms_grad":
        # xh = h / dev; the derivative takes out the part of w g along xh
        h, g = s["x"].double(), s["gy"].double()
        dev = torch.sqrt(torch.linalg.vector_norm(h, dim=1).square() / d + EPS)[:, None]
        xh = h / dev
        gx = (g * w - ((g * xh) @ w)[:, None] / d * xh) / dev
        if case["residual"]:
            gx = gx + s["residual"].double()
        return gx, (torch.ones(1, case["n"], device="cuda", dtype=torch.float64) @ (g * xh))[0]
    h = s["x"].double()
    if case["residual"]:
        h = (s["x"].double() + s["residual"].double()).to(s["x"].dtype).double()     # the sum is what is normed: as it is kept
    dev = torch.sqrt(torch.linalg.vector_norm(h, dim=1).square() / d + EPS)
    y = torch.addcmul(torch.zeros_like(h), h / dev[:, None], w)
    return (y, h, 1.0 / dev) if kind == "rms" else (*_exact_8bit(y), h)
