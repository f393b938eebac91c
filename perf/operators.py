"""Performance cases of the operators that feed and steady the training of a GNN whose nodes carry ids or categories: the lookup of
table rows and its gradient, layer norm forward and backward, and the global norm of all gradients with clipping.

A case is one call (`kind`) with its sizes; `dtype` is the type of the matrices.  Graphs of the benchmark give the sizes: batches of 5000
graphs of 74 nodes, power-law graphs of 56 944 nodes, community graphs of 232 965 nodes, widths 16 to 512.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZES = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-5


def listed():
    return [
        # one small graph at inference: 74 nodes looked up by their degree; launches and latency are the whole time
        dict(name="embed_graph", kind="embed", n=74, rows=74, d=64, dtype="f32", ids="skew", padded=0.0),
        # a batch of 5000 such graphs: many lookups of few rows, so the output is what has to be moved
        dict(name="embed_batch", kind="embed", n=370000, rows=74, d=64, dtype="f32", ids="skew", padded=0.0),
        # sampled neighbours of a community graph, short samples padded: rows of a table that exceeds every L2, half precision
        dict(name="embed_sampled_bf16", kind="embed", n=524288, rows=232965, d=128, dtype="bf16", ids="even", padded=0.1),
        # the gradient for one mini-batch with an odd width: few tokens against a table of thousands of rows
        dict(name="embed_grad_ragged_f16", kind="embed_grad", n=777, rows=4096, d=37, dtype="f16", ids="skew", padded=0.05),
        # the gradient for the batch of graphs: thousands of tokens for each of a few rows
        dict(name="embed_grad_batch", kind="embed_grad", n=370000, rows=74, d=64, dtype="f32", ids="skew", padded=0.0),
        # the gradient for the sampled neighbours: tokens spread over a large table
        dict(name="embed_grad_sampled", kind="embed_grad", n=524288, rows=232965, d=128, dtype="f32", ids="even", padded=0.1),
        # layer norm: one small graph, then all nodes of a community graph in half precision
        dict(name="norm_graph", kind="norm", n=74, d=64, dtype="f32"),
        dict(name="norm_nodes_bf16", kind="norm", n=232965, d=128, dtype="bf16"),
        # its backward pass: the widest features of the sweep, and an odd width in half precision on the power-law graph
        dict(name="norm_grad_wide", kind="norm_grad", n=65536, d=512, dtype="f32"),
        dict(name="norm_grad_odd_bf16", kind="norm_grad", n=56944, d=251, dtype="bf16"),
        # clipping: the weights of a 2-layer GCN with 16 hidden units, and GraphSAGE-LSTM layers behind a table of all nodes' rows
        dict(name="clip_gcn", kind="clip", rows=0, d=64, hidden=16, layers=2, cells=False, dtype="f32", max_norm=0.05),
        dict(name="clip_table", kind="clip", rows=232965, d=128, hidden=64, layers=2, cells=True, dtype="f32", max_norm=1.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["embed", "embed_grad", "embed_grad", "norm", "norm_grad", "norm_grad", "clip"])
    dtype = rng.choice(["f32", "f32", "bf16", "f16"])
    if kind == "clip":
        return dict(kind=kind, rows=rng.choice([0, _log_int(rng, 64, 232965)]), d=_log_int(rng, 8, 128), hidden=8 * _log_int(rng, 1, 16), layers=rng.randint(1, 9),
                    cells=rng.random() < 0.5, dtype=dtype, max_norm=round(math.exp(rng.uniform(math.log(0.01), math.log(30.0))), 3))
    n = _log_int(rng, 1, 400000)
    d = min(_log_int(rng, 8, 1024), max(8, 30000000 // n))
    if kind in ("norm", "norm_grad"):
        return dict(kind=kind, n=n, d=d, dtype=dtype)
    rows = _log_int(rng, 16, min(240000, 30000000 // d))
    return dict(kind=kind, n=n, rows=rows, d=d, dtype=dtype, ids=rng.choice(["skew", "even"]), padded=rng.choice([0.0, 0.0, 0.1, 0.6]))


# ------------------------------------------------------------------------------------------------ inputs

def _shapes(case):
    """Parameter shapes of a model: a table, layer norms, and per layer its weights (and an LSTM cell where `cells`)."""
    d, hid = case["d"], case["hidden"]
    shapes = [(case["rows"], d)] * (case["rows"] > 0)
    widths = [d] + [hid] * (case["layers"] - 1)
    for w in widths:
        shapes += [(w,), (w,)]
        shapes += [(4 * hid, w), (4 * hid, hid), (4 * hid,), (hid + w, hid)] if case["cells"] else [(w, hid)]
    return shapes


def _views(flat, shapes):
    return [part.view(shape) for part, shape in zip(torch.split(flat, [math.prod(s) for s in shapes]), shapes)]


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    normal = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")   # noqa: E731
    dtype, kind = DTYPES[case["dtype"]], case["kind"]
    if kind == "clip":
        # one buffer holds all gradients end to end, as data-parallel training keeps them; parameters are views of it
        shapes = _shapes(case)
        count = sum(math.prod(s) for s in shapes)
        flat = (1e-2 * normal(count)).to(dtype)
        out = torch.empty_like(flat)
        return dict(grads=_views(flat, shapes), out_flat=out, out=_views(out, shapes))
    n, d = case["n"], case["d"]
    if kind in ("embed", "embed_grad"):
        u = torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)
        rows = case["rows"]
        # skew: the number of a row grows exponentially, as frequencies by rank fall off; even: every row alike
        ids = ((rows + 1.0) ** u - 1.0 if case["ids"] == "skew" else rows * u).long().clamp_(0, rows - 1)
        if case["ids"] == "skew":
            ids = torch.randperm(rows, generator=gen, device="cuda")[ids]
        ids = torch.where(torch.rand(n, generator=gen, device="cuda") < case["padded"], -1, ids)
        data = dict(ids=ids, scale=math.sqrt(d))
        if kind == "embed":
            return dict(data, table=(normal(rows, d) * d ** -0.5).to(dtype))
        return dict(data, gy=normal(n, d).to(dtype))
    x = (1.5 * normal(n, d) + 0.5 * normal(n, 1)).to(dtype)
    data = dict(x=x, weight=1.0 + 0.1 * normal(d), bias=0.1 * normal(d))
    if kind == "norm_grad":
        mean = x.double().mean(1)
        data.update(gy=normal(n, d).to(dtype), mean=mean.float(),
                    rstd=((x.double() - mean[:, None]).square().mean(1) + EPS).rsqrt().float())
    return data


def prepare(case, seed):
    return dict(_inputs(case, seed), case=case)


# ------------------------------------------------------------------------------------------------ one pass

def _run_own(s):
    from paper_1906_03707_amd import binding
    case = s["case"]
    kind = case["kind"]
    if kind == "embed":
        return binding.embedding(s["table"], s["ids"], scale=s["scale"], padding=-1)
    if kind == "embed_grad":
        return binding.embedding_grad(s["gy"], s["ids"], case["rows"], scale=s["scale"], padding=-1)
    if kind == "norm":
        return binding.layer_norm(s["x"], s["weight"], s["bias"], eps=EPS)
    if kind == "norm_grad":
        return binding.layer_norm_grad(s["gy"], s["x"], s["mean"], s["rstd"], s["weight"])
    norm = binding.clip_gradients(s["grads"], case["max_norm"], out=s["out"])
    return norm, s["out_flat"]


def _run_plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "embed":
        rows = s["table"][s["ids"].clamp(min=0)].float() * s["scale"]
        return torch.where(s["ids"][:, None] >= 0, rows, 0.0).to(s["table"].dtype)
    if kind == "embed_grad":
        # one row more than the table has takes the padded tokens' gradients
        rows = case["rows"]
        total = torch.zeros(rows + 1, case["d"], device="cuda")
        total.index_add_(0, torch.where(s["ids"] >= 0, s["ids"], rows), s["gy"].float())
        return (total[:rows] * s["scale"]).to(s["gy"].dtype)
    if kind == "norm":
        x = s["x"].float()
        mean = x.mean(1)
        x = x - mean[:, None]
        rstd = (x.square().mean(1) + EPS).rsqrt()
        return (x * rstd[:, None] * s["weight"] + s["bias"]).to(s["x"].dtype), mean, rstd
    if kind == "norm_grad":
        rstd, gy = s["rstd"][:, None], s["gy"].float()
        xh = (s["x"].float() - s["mean"][:, None]) * rstd
        u = gy * s["weight"]
        gx = rstd * (u - u.mean(1, keepdim=True) - xh * (u * xh).mean(1, keepdim=True))
        return gx.to(s["x"].dtype), (gy * xh).sum(0), gy.sum(0)
    norm = torch.stack([g.float().square().sum() for g in s["grads"]]).sum().sqrt()
    scale = (case["max_norm"] / norm).clamp(max=1.0)
    return norm, torch.cat([(g.float() * scale).reshape(-1) for g in s["grads"]]).to(s["out_flat"].dtype)


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------------------------------------ cost and exact results

def work(case):
    kind, size, d = case["kind"], SIZES[case["dtype"]], case["d"]
    if kind == "clip":
        count = sum(math.prod(s) for s in _shapes(case))
        return dict(bytes=2 * count * size + 4, flops=3 * count)
    n = case["n"]
    if kind in ("embed", "embed_grad"):
        kept, rows = round(n * (1 - case["padded"])), case["rows"]
        named = min(kept, rows)
        if case["ids"] == "even":
            named = rows * -math.expm1(-kept / rows)       # distinct rows that so many even draws name
        if kind == "embed":
            return dict(bytes=8 * n + int(named) * d * size + n * d * size, flops=n * d)
        return dict(bytes=8 * n + kept * d * size + rows * d * size, flops=n * d)
    if kind == "norm":
        return dict(bytes=2 * n * d * size + 8 * n + 8 * d, flops=8 * n * d)
    return dict(bytes=3 * n * d * size + 8 * n + 12 * d, flops=15 * n * d)


def exact(case, seed):
    s, kind = _inputs(case, seed), case["kind"]
    if kind == "clip":
        flat = torch.cat([g.reshape(-1) for g in s["grads"]]).double()
        norm = torch.linalg.vector_norm(flat)
        return norm, flat * min(1.0, case["max_norm"] / norm.item())
    if kind == "embed":
        table = torch.cat([s["table"].double(), torch.zeros(1, case["d"], device="cuda", dtype=torch.float64)])
        return s["scale"] * torch.index_select(table, 0, s["ids"] % (case["rows"] + 1))   # -1: the row of zeros at the end
    if kind == "embed_grad":
        kept = s["ids"] >= 0
        total = torch.zeros(case["rows"], case["d"], device="cuda", dtype=torch.float64)
        return total.index_put((s["ids"][kept],), s["gy"][kept].double() * s["scale"], accumulate=True)
    x, w = s["x"].double(), s["weight"].double()
    var, mean = torch.var_mean(x, 1, correction=0)
    if kind == "norm":
        dev = torch.sqrt(var + EPS)
        return torch.addcmul(s["bias"].double(), (x - mean[:, None]) / dev[:, None], w), mean, 1.0 / dev
    # xh = (x - m) / dev; its derivative takes out the parts of w g along the ones and along xh
    dev = torch.sqrt(var + EPS)[:, None]
    xh, g = (x - mean[:, None]) / dev, s["gy"].double()
    along = torch.stack([torch.mv(g, w), (g * xh) @ w], 1) / case["d"]
    gx = (g * w - along[:, :1] - along[:, 1:] * xh) / dev
    ones = torch.ones(1, case["n"], device="cuda", dtype=torch.float64)
    return gx, (ones @ (g * xh))[0], (ones @ g)[0]
