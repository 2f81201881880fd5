"""The operators in front of attention over packed event rows, one case per use: the embedding of the events' ids, layer
normalisation of the rows, and the linear maps that differ from group to group (event types, experts).

    embedding       y[r] = scale * table[ids[r]]  (an id outside the table: a zero row);
                    d table[v] = scale * sum of d y[r] over the r with ids[r] = v
    layer norm      y = (x - mean) * rstd * weight + bias over the last axis, rstd = 1 / sqrt(var + eps);  gradients of x, weight, bias
    grouped linear  y[r] = x[r] @ w[g] for the rows r = offsets[g] .. offsets[g + 1] - 1 of group g;
                    d x[r] = d y[r] @ w[g]^T,  d w[g] = x_g^T @ d y_g

    listed()            the named cases
    draw(rng)           one more case of the same ranges
    prepare(case, seed) inputs on the GPU
    run(state)          one pass: the plain form in 32 bits, or with `own` the library's entry point
    work(case)          bytes and flops the pass cannot do without
    exact(case, seed)   the outputs in 64 bits
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
SKEW = 4.0  # ids: floor(V u^SKEW) with u uniform, a few ids in a large part of the rows as in logged events
PADDING = 1 / 64  # rows whose id is -1
EPS = 1e-5


def _embedding(name, op, n, V, D, dtype="bf16", ids="int32", scale=1.0):
    return dict(name=name, op=op, n=n, V=V, D=D, dtype=dtype, ids=ids, scale=scale)


def _norm(name, op, n, D, dtype="bf16", affine=True):
    return dict(name=name, op=op, n=n, D=D, dtype=dtype, affine=affine)


def _grouped(name, op, n, G, K, N, dtype="bf16"):
    return dict(name=name, op=op, n=n, G=G, K=K, N=N, dtype=dtype)


def listed():
    return [
        # One serving request: the events of a user, rows of four heads of 64.  Launch and host time count.
        _embedding("embedding_request", "embedding_fwd", 640, 50_000, 256),
        # A ranking batch (256 histories of 64 to 1024 events), 64-bit ids.
        _embedding("embedding_batch", "embedding_fwd", 139_264, 1_000_000, 256, ids="int64", scale=16.0),
        # The gradient of the same batch for a table of frequent items.
        _embedding("embedding_grad_batch", "embedding_bwd", 139_264, 200_000, 256, ids="int64", scale=16.0),
        # The large jagged batch (1024 log-normal histories, rows of eight heads of 128).
        _embedding("embedding_grad_large", "embedding_bwd", 1_144_603, 1_000_000, 1024),
        # Norm(E_seed): the seeds of one layer, in single precision.
        _norm("norm_seeds", "norm_fwd", 32, 256, "fp32"),
        # Rows in front of the attention of a ranking batch: serving ...
        _norm("norm_batch", "norm_fwd", 139_264, 256),
        # ... a backward pass at an odd width in single precision ...
        _norm("norm_grad_odd", "norm_bwd", 9_973, 203, "fp32"),
        # ... and the backward pass of the large batch.
        _norm("norm_grad_large", "norm_bwd", 1_144_603, 1024),
        # q, k and v of one request's events, by event type.
        _grouped("grouped_request", "grouped_fwd", 384, 8, 256, 768),
        # A training step's gradients of the same maps.
        _grouped("grouped_grad_batch", "grouped_bwd", 139_264, 8, 256, 768),
        # Sixteen experts of a wide layer.
        _grouped("grouped_large", "grouped_fwd", 262_144, 16, 1024, 4096),
        # Small odd sizes in single precision, both gradients.
        _grouped("grouped_grad_fp32", "grouped_bwd", 9_973, 5, 200, 328, "fp32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["embedding_fwd", "embedding_bwd", "norm_fwd", "norm_bwd", "grouped_fwd", "grouped_bwd"])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    if op.startswith("embedding"):
        c = _embedding("", op, _log_int(rng, 1, 1_144_603), _log_int(rng, 100, 1_000_000), _log_int(rng, 8, 1024), dtype,
                       rng.choice(["int32", "int64"]), rng.choice([1.0, 0.5, 16.0, 11.3]))
        c["D"] = rng.choice([c["D"], (c["D"] + 7) // 8 * 8, (c["D"] + 7) // 8 * 8])
        largest = {"bytes": 4.6e9, "flops": math.inf}
    elif op.startswith("norm"):
        c = _norm("", op, _log_int(rng, 1, 1_144_603), _log_int(rng, 8, 8192), dtype, rng.random() < 0.8)
        c["D"] = rng.choice([c["D"], (c["D"] + 7) // 8 * 8, (c["D"] + 7) // 8 * 8])
        largest = {"bytes": 7.0e9, "flops": math.inf}
    else:
        width = lambda: (_log_int(rng, 8, 4096) + 7) // 8 * 8
        c = _grouped("", op, _log_int(rng, 1, 262_144), _log_int(rng, 1, 64), width(), width(), dtype)
        if dtype == "fp32" and rng.random() < 0.5:
            c["K"] += 4
        largest = {"bytes": 2.5e9, "flops": 2.1e12 if dtype == "bf16" else 4e11}
    while c["n"] > 1 and any(work(c)[k] > largest[k] for k in largest):
        c["n"] //= 2
    return {k: v for k, v in c.items() if k != "name"}


# ---- sizes ----

def _distinct(n, V):
    """Expected number of table rows that n ids name."""
    edges = (np.arange(V + 1) / V) ** (1 / SKEW)
    return float(-np.expm1(n * (1 - PADDING) * np.log1p(-np.minimum(np.diff(edges), 1 - 1e-12))).sum())


def _sizes(case, seed=None):
    """Rows of every group, the largest about n / 4 for many groups; of four groups or more one is empty.  The seed orders them."""
    G, n = case["G"], case["n"]
    full = G - 1 if G >= 4 else G
    share = 1.0 / np.sqrt(np.arange(1, full + 1))
    edges = np.rint(np.concatenate([[0.0], np.cumsum(share) / share.sum()]) * n).astype(np.int64)
    sizes = np.concatenate([np.diff(edges), np.zeros(G - full, dtype=np.int64)])
    return sizes if seed is None else np.random.default_rng(seed).permutation(sizes)


def work(case):
    e = 4 if case["dtype"] == "fp32" else 2
    n = case["n"]
    if case["op"].startswith("embedding"):
        D, ids = case["D"], n * (8 if case["ids"] == "int64" else 4)
        if case["op"] == "embedding_fwd":
            return {"bytes": ids + (n + _distinct(n, case["V"])) * D * e, "flops": n * D}
        return {"bytes": ids + (n + case["V"]) * D * e, "flops": n * D}
    if case["op"].startswith("norm"):
        D = case["D"]
        if case["op"] == "norm_fwd":
            return {"bytes": 2 * n * D * e + 8 * n, "flops": 8 * n * D}
        return {"bytes": 3 * n * D * e + 8 * n, "flops": 14 * n * D}
    K, N = case["K"], case["N"]
    w = case["G"] * K * N
    if case["op"] == "grouped_fwd":
        return {"bytes": (n * K + w + n * N) * e, "flops": 2 * n * K * N}
    return {"bytes": (2 * n * K + 2 * w + n * N) * e, "flops": 4 * n * K * N}


# ---- inputs ----

def _normal(gen, shape, sigma, dtype):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, sigma, generator=gen)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dtype, op, n = DTYPES[case["dtype"]], case["op"], case["n"]
    s = dict(op=op)
    if op.startswith("embedding"):
        V, D = case["V"], case["D"]
        u = torch.rand(n, dtype=torch.float64, device="cuda", generator=gen)
        ids = (u ** SKEW * V).long().clamp_(max=V - 1) * 1_000_003 % V  # the frequent ones spread over the table
        ids[torch.rand(n, device="cuda", generator=gen) < PADDING] = -1
        s.update(ids=ids.to(torch.int64 if case["ids"] == "int64" else torch.int32), scale=case["scale"], V=V)
        rows = V if op == "embedding_fwd" else n
        s["table" if op == "embedding_fwd" else "d_out"] = _normal(gen, (rows, D), 1.0, dtype)
        return s
    if op.startswith("norm"):
        D = case["D"]
        x = _normal(gen, (n, D), 1.0, dtype)
        x += _normal(gen, (n, 1), 0.5, dtype)
        s.update(x=x, weight=_normal(gen, (D,), 0.2, dtype) + 1 if case["affine"] else None, bias=_normal(gen, (D,), 0.2, dtype) if case["affine"] else None)
        if op == "norm_bwd":
            x = x.double()
            mean = x.mean(1)
            rstd = (x.var(1, correction=0) + EPS).rsqrt()
            s.update(dy=_normal(gen, (n, D), 1.0, dtype), mean=mean.float(), rstd=rstd.float())
        return s
    G, K, N = case["G"], case["K"], case["N"]
    sizes = _sizes(case, seed)
    offsets = torch.from_numpy(np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)).cuda()
    s.update(x=_normal(gen, (n, K), 1.0, dtype), w=_normal(gen, (G, K, N), K ** -0.5, dtype), offsets=offsets, sizes=sizes.tolist())
    if op == "grouped_bwd":
        s["dy"] = _normal(gen, (n, N), 1.0, dtype)
    return s


# ---- one pass ----

def run(s):
    if own:
        return _own(s)
    return {"embedding_fwd": _embedding_fwd, "embedding_bwd": _embedding_bwd, "norm_fwd": _norm_fwd, "norm_bwd": _norm_bwd,
            "grouped_fwd": _grouped_fwd, "grouped_bwd": _grouped_bwd}[s["op"]](s)


def _own(s):
    from paper_2602_10016_amd import binding as kb
    op = s["op"]
    if op == "embedding_fwd":
        return {"y": kb.embedding_fwd(s["table"], s["ids"], s["scale"])}
    if op == "embedding_bwd":
        return {"d_table": kb.embedding_bwd(s["d_out"], s["ids"], s["V"], s["scale"])}
    if op == "norm_fwd":
        return dict(zip(("y", "mean", "rstd"), kb.layer_norm_fwd(s["x"], s["weight"], s["bias"], EPS)))
    if op == "norm_bwd":
        dx, dw, db = kb.layer_norm_bwd(s["x"], s["weight"], s["dy"], s["mean"], s["rstd"])
        return {"dx": dx} if s["weight"] is None else {"dx": dx, "dw": dw, "db": db}
    if op == "grouped_fwd":
        return {"y": kb.grouped_linear_fwd(s["x"], s["w"], s["offsets"])}
    return dict(zip(("dx", "dw"), kb.grouped_linear_bwd(s["x"], s["w"], s["dy"], s["offsets"])))


def _embedding_fwd(s):
    ids, table = s["ids"].long(), s["table"]
    rows = table[ids.clamp(min=0)].float() * s["scale"]
    return {"y": torch.where((ids >= 0)[:, None], rows, 0.0).to(table.dtype)}


def _embedding_bwd(s):
    ids, d_out = s["ids"].long(), s["d_out"]
    rows = torch.where((ids >= 0)[:, None], d_out.float(), 0.0)
    sums = torch.zeros(s["V"], d_out.shape[1], dtype=torch.float32, device="cuda").index_add_(0, ids.clamp(min=0), rows)
    return {"d_table": (sums * s["scale"]).to(d_out.dtype)}


def _norm_fwd(s):
    x = s["x"].float()
    mean = x.mean(1)
    x = x - mean[:, None]
    rstd = ((x * x).mean(1) + EPS).rsqrt()
    y = x * rstd[:, None]
    if s["weight"] is not None:
        y = y * s["weight"].float() + s["bias"].float()
    return {"y": y.to(s["x"].dtype), "mean": mean, "rstd": rstd}


def _norm_bwd(s):
    dtype, rstd, dy = s["x"].dtype, s["rstd"][:, None], s["dy"].float()
    x = (s["x"].float() - s["mean"][:, None]) * rstd
    g = dy if s["weight"] is None else dy * s["weight"].float()
    dx = (rstd * (g - g.mean(1, keepdim=True) - x * (g * x).mean(1, keepdim=True))).to(dtype)
    if s["weight"] is None:
        return {"dx": dx}
    return {"dx": dx, "dw": (dy * x).sum(0).to(dtype), "db": dy.sum(0).to(dtype)}


def _grouped_fwd(s):
    w = s["w"].float()
    return {"y": torch.cat([x @ w_g for x, w_g in zip(s["x"].float().split(s["sizes"]), w)]).to(s["x"].dtype)}


def _grouped_bwd(s):
    w, dtype = s["w"].float(), s["x"].dtype
    x, dy = s["x"].float().split(s["sizes"]), s["dy"].float().split(s["sizes"])
    dx = torch.cat([g @ w_g.T for g, w_g in zip(dy, w)])
    dw = torch.stack([x_g.T @ g for x_g, g in zip(x, dy)])
    return {"dx": dx.to(dtype), "dw": dw.to(dtype)}


# ---- 64 bits ----

def exact(case, seed):
    s = prepare(case, seed)
    op = s["op"]
    if op == "embedding_fwd":
        y = s["table"].index_select(0, s["ids"].long().abs()).double().mul_(s["scale"])
        return {"y": y.masked_fill_((s["ids"] < 0)[:, None], 0.0)}
    if op == "embedding_bwd":
        # rows in the order of their ids, running sums along them, differences at the ends of equal ids
        V, D = case["V"], case["D"]
        order = torch.argsort(s["ids"])
        ends = torch.searchsorted(s["ids"][order].long(), torch.arange(-1, V, device="cuda"), right=True)
        out = torch.empty(V, D, dtype=torch.float64, device="cuda")
        for c in range(0, D, 64):
            part = s["d_out"][:, c:c + 64].double()[order]
            sums = torch.cat([torch.zeros_like(part[:1]), part.cumsum(0)])[ends]
            out[:, c:c + 64] = sums.diff(dim=0) * s["scale"]
        return {"d_table": out}
    if op.startswith("norm"):
        x = s["x"].double()
        var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
        rstd = 1 / torch.sqrt(var + EPS)
        affine = s["weight"] is not None
        if op == "norm_fwd":
            y = (x - mean) * rstd
            return {"y": torch.addcmul(s["bias"].double(), y, s["weight"].double()) if affine else y, "mean": mean[:, 0], "rstd": rstd[:, 0]}
        dy = s["dy"].double()
        h = (x - mean).mul_(rstd)
        g = dy * s["weight"].double() if affine else dy
        along = torch.linalg.vecdot(g, h)[:, None] / case["D"]
        dx = (g - g.sum(1, keepdim=True) / case["D"] - h * along) * rstd
        return {"dx": dx, "dw": torch.linalg.vecdot(dy, h, dim=0), "db": dy.sum(0)} if affine else {"dx": dx}
    x, w, offsets = s["x"].double(), s["w"].double(), s["offsets"].tolist()
    if op == "grouped_fwd":
        y = torch.empty(case["n"], case["N"], dtype=torch.float64, device="cuda")
        for g in range(case["G"]):
            torch.mm(x[offsets[g]:offsets[g + 1]], w[g], out=y[offsets[g]:offsets[g + 1]])
        return {"y": y}
    dy, dx, dw = s["dy"].double(), torch.empty_like(x), torch.empty_like(w)
    for g in range(case["G"]):
        rows = slice(offsets[g], offsets[g + 1])
        torch.mm(dy[rows], w[g].t().contiguous(), out=dx[rows])
        torch.mm(x[rows].t().contiguous(), dy[rows], out=dw[g])
    return {"dx": dx, "dw": dw}
