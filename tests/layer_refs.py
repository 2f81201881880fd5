"""The operators in front of attention in 64 bits by plain numpy, each with a bound on how far a correct implementation with fp32 sums
may be: u = 2^-24 per fp32 rounding (n + 1 roundings for a sum of n rounded products, in any order), v = half a step of the output
type.  A bound is a sum of those times the magnitudes that they act on, first order; 1 % and a few smallest numbers are added for the rest."""
import numpy as np
import torch

U = 2.0 ** -24
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
DTYPES = [torch.bfloat16, torch.float32]


def up(x):
    return None if x is None else x.detach().cpu().double().numpy()


def check(what, got, ref, bound, dtype):
    """|got - ref| <= bound + half a step of the output type, for every value; not a number where ref is none."""
    got = up(got)
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    limit = 1.01 * (bound + HALF_STEP[dtype] * (np.abs(ref) + bound)) + 1e-37
    bad = ~(np.abs(got - ref) <= limit)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size}, worst {np.nanmax(np.abs(got - ref) / limit):.2f} of the bound"


def embedding_fwd(table, ids, scale):
    """One product: one fp32 rounding before the output's."""
    table, ids = up(table), ids.cpu().numpy().astype(np.int64)
    ok = (ids >= 0) & (ids < len(table))
    y = np.zeros(ids.shape + table.shape[1:])
    y[ok] = table[ids[ok]] * float(np.float32(scale))
    return y, U * np.abs(y)


def embedding_bwd(d_out, ids, rows, scale):
    d_out, ids, scale = up(d_out), ids.cpu().numpy().astype(np.int64).ravel(), float(np.float32(scale))
    d_out = d_out.reshape(len(ids), -1) if len(ids) else d_out.reshape(0, d_out.shape[-1])
    ok = (ids >= 0) & (ids < rows)
    total, size, count = np.zeros((rows, d_out.shape[1])), np.zeros((rows, d_out.shape[1])), np.zeros(rows)
    np.add.at(total, ids[ok], d_out[ok])
    np.add.at(size, ids[ok], np.abs(d_out[ok]))
    np.add.at(count, ids[ok], 1)
    return total * scale, (count[:, None] + 1) * U * size * abs(scale)


def norm_fwd(x, weight, bias, eps):
    """((y, bound), (mean, bound), (rstd, bound))"""
    x, weight, bias = up(x), up(weight), up(bias)
    D = x.shape[-1]
    m = x.mean(-1, keepdims=True)
    c = x - m
    var = (c * c).mean(-1, keepdims=True)
    r = 1 / np.sqrt(var + float(np.float32(eps)))
    dm = (D + 1) * U * np.abs(x).mean(-1, keepdims=True)
    dc = dm + U * np.abs(c)
    dvar = 2 * (dc * np.abs(c)).mean(-1, keepdims=True) + (dc * dc).mean(-1, keepdims=True) + (D + 2) * U * var
    dr = r * (0.5 * dvar / (var + float(np.float32(eps))) + 3 * U)
    w, b = (1 if weight is None else weight), (0 if bias is None else bias)
    y = c * r * w + b
    dy = np.abs(w) * (dc * r + np.abs(c) * dr + 2 * U * np.abs(c * r)) + U * (np.abs(y) + np.abs(b))
    return (y, dy), (m[..., 0], dm[..., 0]), (r[..., 0], dr[..., 0])


def norm_bwd(x, weight, dy, mean, rstd):
    """Of the given statistics.  ((dx, bound), (dw, bound), (db, bound))"""
    x, weight, dy, m, r = up(x), up(weight), up(dy), up(mean)[..., None], up(rstd)[..., None]
    D = x.shape[-1]
    x, dy, m, r = x.reshape(-1, D), dy.reshape(-1, D), m.reshape(-1, 1), r.reshape(-1, 1)
    R = len(x)
    h, g = (x - m) * r, dy * (1 if weight is None else weight)
    mg, mgh = g.mean(1, keepdims=True), (g * h).mean(1, keepdims=True)
    dx = r * (g - mg - h * mgh)
    along = (D + 2) * U * np.abs(g).mean(1, keepdims=True) + np.abs(h) * (D + 5) * U * np.abs(g * h).mean(1, keepdims=True)
    bx = r * (along + 6 * U * (np.abs(g) + np.abs(mg) + np.abs(h * mgh)))
    dw, db = (dy * h).sum(0), dy.sum(0)
    return (dx, bx), (dw, (R + 4) * U * np.abs(dy * h).sum(0)), (db, (R + 1) * U * np.abs(dy).sum(0))


def grouped_fwd(x, w, offsets):
    x, w, offsets = up(x), up(w), offsets.tolist()
    K = x.shape[1]
    y, size = np.zeros((len(x), w.shape[2])), np.zeros((len(x), w.shape[2]))
    for g in range(len(w)):
        r = slice(offsets[g], offsets[g + 1])
        y[r], size[r] = x[r] @ w[g], np.abs(x[r]) @ np.abs(w[g])
    return y, (K + 1) * U * size


def grouped_bwd(x, w, dy, offsets):
    x, w, dy, offsets = up(x), up(w), up(dy), offsets.tolist()
    dx, bx, dw, bw = np.zeros_like(x), np.zeros_like(x), np.zeros_like(w), np.zeros_like(w)
    for g in range(len(w)):
        r = slice(offsets[g], offsets[g + 1])
        dx[r], bx[r] = dy[r] @ w[g].T, (w.shape[2] + 1) * U * (np.abs(dy[r]) @ np.abs(w[g].T))
        dw[g], bw[g] = x[r].T @ dy[r], (offsets[g + 1] - offsets[g] + 1) * U * (np.abs(x[r].T) @ np.abs(dy[r]))
    return (dx, bx), (dw, bw)


def normal(shape, dtype, seed, sigma=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, device="cuda", generator=gen) * sigma).to(dtype)


def guarded(shape, dtype):
    """A tensor of NaN between two rims of NaN; the second result: the rims."""
    n, rim = int(np.prod(shape)), 128
    buf = torch.full((n + 2 * rim,), float("nan"), dtype=dtype, device="cuda")
    return buf[rim:rim + n].view(shape), (buf[:rim], buf[rim + n:])


def untouched(rims):
    return all(bool(r.isnan().all()) for r in rims)
