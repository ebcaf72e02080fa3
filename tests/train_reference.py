"""64-bit definitions of the calls around the layers (embedding, layer norm, attention
within documents, gradient norm), and the bounds of their kernels' roundings.

u below is fp32's half step, H bf16's.  A sum of n fp32 terms in any order is off by at
most (n - 1) u times the sum of the terms' magnitudes."""
import math

import torch

U = torch.finfo(torch.float32).eps / 2
H = torch.finfo(torch.bfloat16).eps / 2
D = 128


def f64(t):
    return t.double()


def rounding(dtype):
    return H if dtype is torch.bfloat16 else U


# ------------------------------------------------------------------ embedding
def embedding(ids, table, scale, off):
    ids = ids.long() - off
    here = (ids >= 0) & (ids < table.shape[0])
    rows = f64(table)[ids.clamp(0, table.shape[0] - 1)] * scale
    return torch.where(here[:, None], rows, 0.0)


def embedding_bwd(ids, dy, vocab, scale, off):
    """The gradient, and a bound of an fp32 sum in any order, the scaling and the rounding."""
    ids = ids.long() - off
    here = (ids >= 0) & (ids < vocab)
    at = torch.where(here, ids, vocab)
    grad = torch.zeros((vocab + 1, dy.shape[1]), dtype=torch.float64, device=dy.device)
    size, count = torch.zeros_like(grad), torch.zeros_like(grad[:, :1])
    grad.index_add_(0, at, f64(dy))
    size.index_add_(0, at, f64(dy).abs())
    count.index_add_(0, at, torch.ones_like(count[:1]).expand(len(ids), 1))
    return grad[:vocab] * scale, ((count + 2) * U * size * abs(scale))[:vocab]


# ------------------------------------------------------------------ layer norm
# A lane adds at most 32 values, then at most ten levels join lanes and waves; the
# centred squares take two operations more, the root and the division three.
ROW_SUM = 32 + 10


def norm_stats(x):
    """Mean and centred squares of rows, with the bounds of both."""
    x = f64(x)
    mean = x.mean(1)
    e_mean = (ROW_SUM + 2) * U * x.abs().mean(1)
    dev = x - mean[:, None]
    m2 = (dev ** 2).sum(1)
    # each difference is off by e_mean and a rounding
    e_dev = e_mean[:, None] + U * (dev.abs() + x.abs())
    e_m2 = (ROW_SUM + 2) * U * m2 + (2 * dev.abs() * e_dev + e_dev ** 2).sum(1)
    return mean, m2, e_mean, e_m2


def norm(x, w, b, eps, mean, m2, e_mean, e_m2, total):
    """y, rstd and their bounds from statistics of rows of `total` values."""
    x = f64(x)
    var = m2 / total + eps
    rstd = var ** -0.5
    rel = 0.5 * (e_m2 / total) / var + 5 * U
    xh = (x - mean[:, None]) * rstd[:, None]
    e_xh = rstd[:, None] * (e_mean[:, None] + U * (x - mean[:, None]).abs()) + \
        xh.abs() * (rel[:, None] + U)
    w = torch.ones_like(x[0]) if w is None else f64(w)
    b = torch.zeros_like(x[0]) if b is None else f64(b)
    y = xh * w + b
    e_y = e_xh * w.abs() + 2 * U * ((xh * w).abs() + y.abs())
    return y, rstd, e_y + H * (y.abs() + e_y), 1.01 * rel * rstd


def norm_bwd(x, w, mean, rstd, dy, d_res, sums=None, total=None):
    """dx (before its rounding), dw, db and their bounds, from the forward's mean and rstd
    as they are; sums: the row sums of the other devices."""
    x, dy, mean, rstd = f64(x), f64(dy), f64(mean)[:, None], f64(rstd)[:, None]
    w = torch.ones_like(x[0]) if w is None else f64(w)
    total = total or x.shape[1]
    xh = (x - mean) * rstd
    e_xh = 3 * U * xh.abs()
    g = dy * w
    c1, c2 = g.sum(1, keepdim=True), (g * xh).sum(1, keepdim=True)
    a1, a2 = g.abs().sum(1, keepdim=True), (g * xh).abs().sum(1, keepdim=True)
    n = ROW_SUM
    own = torch.cat((c1, c2), 1)
    e_own = torch.cat(((n + 2) * U * a1, (n + 6) * U * a2), 1)
    e1, e2 = e_own[:, :1], e_own[:, 1:]
    for s in sums or []:
        s = f64(s)
        c1, c2 = c1 + s[:, :1], c2 + s[:, 1:]
    k = len(sums or [])
    e1 = (e1 + k * U * (c1.abs() + a1)) / total
    e2 = (e2 + k * U * (c2.abs() + a2)) / total
    c1, c2 = c1 / total, c2 / total
    inner = g - c1 - xh * c2
    size = g.abs() + c1.abs() + (xh * c2).abs()
    e_in = e1 + xh.abs() * e2 + e_xh * c2.abs() + 6 * U * size
    dx = rstd * inner
    e_dx = rstd * e_in + 2 * U * rstd * size
    if d_res is not None:
        dx = dx + f64(d_res)
        e_dx = e_dx + 2 * U * dx.abs()
    rows = x.shape[0]
    dw, db = (dy * xh).sum(0), dy.sum(0)
    e_dw = (rows + 5) * U * (dy * xh).abs().sum(0)
    e_db = (rows + 1) * U * dy.abs().sum(0)
    return dict(dx=dx, e_dx=e_dx, dw=dw, e_dw=e_dw, db=db, e_db=e_db, own=own, e_own=e_own)


# ------------------------------------------------------------------ attention
# exp2 and rcp of the hardware are off by 2^-22 at most, relative to their result;
# tanh by 3 u of 1.
EXP = 2.0 ** -22


def _pairs(n, prefix, device):
    i = torch.arange(n, device=device)
    sees = (i[None, :] <= i[:, None]) | (i < prefix)[None, :]
    return sees, (i[:, None] - i[None, :]).abs().double()


def _score(q, k, cap, slope, far):
    """Scores, d score / d raw, and the bound of the scores' roundings."""
    raw = q @ k.T.contiguous() / math.sqrt(D)
    e = (D + 2) * U * (q.abs() @ k.abs().T.contiguous()) / math.sqrt(D)
    x, dx = raw, torch.ones_like(raw)
    if cap:
        t = torch.tanh(raw / cap)
        x, dx = cap * t, 1 - t * t
        e = dx * e + 6 * U * cap
    if slope:
        x = x - slope * far
    return x, dx, e + 3 * U * x.abs()


def attention(qkv, kv, group, cu, prefix=None, slopes=None, cap=0.0, out=None, lse=None,
              d_out=None):
    """Forward: (out, lse, bound of out, bound of lse); with d_out, out and lse (the
    forward's, as they are): (d_qkv, its bound).  Rows outside the documents are NaN."""
    t = qkv.shape[0]
    x = f64(qkv).reshape(t, kv, group + 2, D)
    nan = dict(dtype=torch.float64, device=qkv.device)
    back = d_out is not None
    if back:
        res, bound = torch.full(x.shape, float("nan"), **nan), torch.zeros(x.shape, **nan)
    else:
        res = torch.full((t, kv * group, D), float("nan"), **nan)
        bound = torch.zeros(res.shape, **nan)
        z = torch.full((kv * group, t), float("nan"), **nan)
        e_z = torch.zeros(z.shape, **nan)
    for d in range(len(cu) - 1):
        a, n = cu[d], cu[d + 1] - cu[d]
        if n == 0:
            continue
        rows = slice(a, a + n)
        sees, far = _pairs(n, min(max(prefix[d], 0), n) if prefix else 0, qkv.device)
        for u in range(kv):
            k, v = x[rows, u, group], x[rows, u, group + 1]
            if back:
                dk, dv, e_dk, e_dv = (torch.zeros_like(k) for _ in range(4))
            for m in range(group):
                h = u * group + m
                q = x[rows, u, m]
                s, slope, e = _score(q, k, cap, slopes[h] if slopes else 0.0, far)
                s = torch.where(sees, s, -math.inf)
                if not back:
                    lz = torch.logsumexp(s, 1)
                    w = torch.exp(s - lz[:, None])
                    # the weights' errors, their rounding to bf16, the sums' errors
                    rel = torch.where(sees, e, 0.0)
                    rel = rel + (rel * w).sum(1, keepdim=True) + 2 * EXP + (n + 8) * U
                    o = w @ v
                    e_o = (w * (rel + H)) @ v.abs() * (1 + 2 * H)
                    res[rows, h] = o
                    bound[rows, h] = e_o + H * (o.abs() + e_o)
                    z[h, rows] = lz
                    e_z[h, rows] = (torch.where(sees, e, 0.0) * w).sum(1) + 3 * EXP + \
                        (n + 8) * U + 4 * U * lz.abs()
                    continue
                lz = f64(lse[h, rows])[:, None]
                p = torch.exp(s - lz)
                rel = torch.where(sees, e, 0.0) + 2 * EXP + 4 * U * lz.abs()
                do, o = f64(d_out)[rows].reshape(n, -1, D)[:, h], f64(out)[rows].reshape(
                    n, -1, D)[:, h]
                dp = do @ v.T.contiguous()
                delta = (do * o).sum(1, keepdim=True)
                e_d = (D + 2) * U * (do.abs() @ v.abs().T.contiguous() +
                                     (do * o).abs().sum(1, keepdim=True))
                diff = dp - delta
                ds = p * diff * slope
                e_slope = 12 * U if cap else 0.0
                e_ds = p * slope * (e_d + diff.abs() * (rel + 3 * U)) + p * diff.abs() * e_slope
                e_ds = e_ds + H * (ds.abs() + e_ds)
                sc = 1 / math.sqrt(D)
                dq = ds @ k * sc
                e_dq = (e_ds + n * U * ds.abs()) @ k.abs() * sc * (1 + H)
                res[rows, u, m] = dq
                bound[rows, u, m] = e_dq + 2 * U * dq.abs() + H * (dq.abs() + e_dq)
                e_p = p * (rel + H * (1 + rel))
                many = n * group * U
                dk += ds.T.contiguous() @ q * sc
                e_dk += (e_ds + many * ds.abs()).T.contiguous() @ q.abs() * sc * (1 + H)
                dv += p.T.contiguous() @ do
                e_dv += (e_p + many * p).T.contiguous() @ do.abs() * (1 + H)
            if back:
                for c, (g_, e_) in enumerate(((dk, e_dk), (dv, e_dv))):
                    res[rows, u, group + c] = g_
                    bound[rows, u, group + c] = e_ + 2 * U * g_.abs() + H * (g_.abs() + e_)
    if back:
        return res.reshape(t, -1), bound.reshape(t, -1)
    return res.reshape(t, -1), z, bound.reshape(t, -1), e_z


# ------------------------------------------------------------------ gradients
def grad_factor(total, scale, max_norm):
    norm = scale * math.sqrt(total)
    return norm, scale * (1.0 if norm <= max_norm else max_norm / norm)


def check(got, want, bound, what):
    err = (f64(got) - want).abs()
    bad = ~(err <= bound)
    assert not bad.any(), (what, int(bad.sum()), float((err - bound).nan_to_num(1e30).max()),
                           bad.nonzero()[:3].tolist())
