"""64-bit definitions of the position, cache and cached-attention operators on
the CPU, written from their formulas, and error bounds counted in roundings."""
import math

import torch

D = 128
HALF_BF16 = 2.0 ** -8          # half a step, relative to the value
EPS32 = 2.0 ** -24             # the same for float32


def f64(t):
    return t.detach().to("cpu", torch.float64)


# ------------------------------------------------------------------ norms and rotation
class Rope:
    """Parameters on the CPU (float64 copies of what the call gets)."""

    def __init__(self, qw=None, kw=None, eps=1e-6, inv_freq=None, rot=0, inter=False, norm=True):
        self.qw = torch.ones(D, dtype=torch.float64) if qw is None else f64(qw)
        self.kw = torch.ones(D, dtype=torch.float64) if kw is None else f64(kw)
        self.eps, self.rot, self.inter, self.norm = float(torch.tensor(eps).float()), rot, inter, norm
        self.inv_freq = None if inv_freq is None else f64(inv_freq)

    def pairs(self):
        i = torch.arange(self.rot // 2)
        return (2 * i, 2 * i + 1) if self.inter else (i, i + self.rot // 2)


def heads(block, kv, group):
    return f64(block).reshape(-1, kv, group + 2, D)


def _turn(p, y, angle, sign):
    if not p.rot:
        return y.clone()
    a, b = p.pairs()
    c, s = torch.cos(angle), sign * torch.sin(angle)
    out = y.clone()
    out[..., a] = y[..., a] * c - y[..., b] * s
    out[..., b] = y[..., a] * s + y[..., b] * c
    return out


def _angles(p, positions):
    if not p.rot:
        return None
    return (positions.double()[:, None] * p.inv_freq)[:, None, None, :]


def _weights(p, group):
    return torch.cat((p.qw.expand(group, D), p.kw.expand(1, D)))     # [group + 1, D]


def norm_rope(p, x, group, positions):
    """x [t, kv, group + 2, D] -> (y, bound): queries and keys, values as they are.
    Roundings: the result's, and fp32's in u = w x r and the turn, at most 2^6 of
    them of values no larger than the head's largest |u|."""
    qk = x[:, :, :group + 1]
    u = qk
    if p.norm:
        r = torch.rsqrt((qk ** 2).mean(-1, keepdim=True) + p.eps)
        u = qk * r * _weights(p, group)
    y = _turn(p, u, _angles(p, positions), 1.0)
    bound = HALF_BF16 * y.abs() + 64 * EPS32 * u.abs().amax(-1, keepdim=True)
    v = x[:, :, group + 1:]
    return torch.cat((y, v), 2), torch.cat((bound, torch.zeros_like(v)), 2)


def norm_rope_bwd(p, x, dy, group, positions):
    """(dx, bound, dqw, dkw, sum |terms| of each)."""
    qk, g = x[:, :, :group + 1], dy[:, :, :group + 1]
    turned = _turn(p, g, _angles(p, positions), -1.0)
    w = _weights(p, group)
    dx, amp = turned, turned.abs().amax(-1, keepdim=True)
    dws = None
    if p.norm:
        r = torch.rsqrt((qk ** 2).mean(-1, keepdim=True) + p.eps)
        xh = qk * r
        terms = turned * xh
        dws = (terms[:, :, :group].sum((0, 1, 2)), terms[:, :, group].sum((0, 1)),
               terms[:, :, :group].abs().sum((0, 1, 2)), terms[:, :, group].abs().sum((0, 1)))
        gw = turned * w
        mean = (gw * xh).mean(-1, keepdim=True)
        dx = r * (gw - xh * mean)
        amp = r * (gw.abs().amax(-1, keepdim=True) + xh.abs().amax(-1, keepdim=True) *
                   (gw * xh).abs().mean(-1, keepdim=True))
    bound = HALF_BF16 * dx.abs() + 64 * EPS32 * amp
    v = dy[:, :, group + 1:]
    return (torch.cat((dx, v), 2), torch.cat((bound, torch.zeros_like(v)), 2), dws)


# ------------------------------------------------------------------ attention
def attention(pool, table, ctx, cu, q, kv, group, page, mask=None, tokens=None, wide=True):
    """Cached attention in 64 bits -> (out, lse, out bound, lse bound); rows that no
    sequence owns are NaN in `out`.  Empty or invalid places are not seen.

    Bounds: the score sums 128 products in fp32 (128 EPS32 of scale * sum |q k| each
    way, so twice that of a weight); a weight is rounded to bf16 where the tile is
    wide, to 16 bits else; sums over n keys take n EPS32; the output one rounding."""
    n_pages = pool.shape[0]
    tokens = q.shape[0] if tokens is None else tokens
    out = torch.full((tokens, kv * group, D), math.nan, dtype=torch.float64)
    ob = torch.zeros_like(out)
    lse = torch.full((kv * group, tokens), math.nan, dtype=torch.float64)
    lb = torch.zeros_like(lse)
    pool, qd = f64(pool), f64(q)
    table = table.cpu()
    for s in range(len(ctx)):
        a, b = cu[s], cu[s + 1]
        n, keys = b - a, ctx[s] + b - a
        if n <= 0:
            continue
        place = torch.arange(keys)
        col = place // page
        inside = col < table.shape[1]
        pg = torch.where(inside, table[s][col.clamp(max=table.shape[1] - 1)].long(), -1)
        there = (pg >= 0) & (pg < n_pages)
        sees = torch.zeros((n, keys), dtype=torch.bool)
        for j in range(n):
            sees[j, :ctx[s]] = True
            for i in range(n):
                if mask is None:
                    sees[j, ctx[s] + i] = i <= j
                elif i < 64 * mask.shape[1]:
                    sees[j, ctx[s] + i] = bool((int(mask[a + j, i // 64]) >> (i % 64)) & 1)
        sees &= there
        pg = pg.clamp(0, n_pages - 1)
        for h in range(kv):
            k, v = pool[pg, 0, h, place % page], pool[pg, 1, h, place % page]
            for m in range(group):
                hq = h * group + m
                qr = qd[a:b, hq * D:(hq + 1) * D]
                k0, v0 = torch.where(sees.any(0)[:, None], k, 0), torch.where(sees.any(0)[:, None], v, 0)
                score = qr @ k0.T / math.sqrt(D)
                size = (qr.abs() @ k0.abs().T / math.sqrt(D)).masked_fill(~sees, 0).nan_to_num(0)
                score = torch.where(sees, score, -math.inf)
                z = torch.logsumexp(score, -1)
                w = torch.exp(score - torch.where(z > -math.inf, z, 0.0)[:, None])
                # rows do not see the infinities and NaN of places masked for them
                o = torch.stack([w[j][sees[j]] @ v[sees[j]] for j in range(n)])
                amp = torch.stack([w[j][sees[j]] @ v[sees[j]].abs() for j in range(n)])
                top = size.amax(-1) if keys else torch.zeros(n, dtype=torch.float64)
                ds = 2 * 128 * EPS32 * top + (keys + 64) * EPS32
                rw = HALF_BF16 if wide else 2.0 ** -15
                out[a:b, hq] = o
                ob[a:b, hq] = HALF_BF16 * o.abs() + (rw + 2 * ds)[:, None] * amp if rw is not None else 0
                lse[hq, a:b] = z
                lb[hq, a:b] = ds + 8 * EPS32 * (1 + z.abs().nan_to_num(0, 0, 0))
    return out.reshape(tokens, -1), lse, ob.reshape(tokens, -1), lb


# ------------------------------------------------------------------ pages, one at a time
class Pool:
    """Tables and counts as lists, changed one sequence and one page at a time."""

    def __init__(self, n_pages, page, refs, table):
        self.n, self.page, self.refs = n_pages, page, list(refs)
        self.table = [list(r) for r in table]

    def ok(self, e):
        return 0 <= e < self.n

    def release(self, keep):
        for row, k in zip(self.table, keep):
            if k >= 0:
                for i in range(-(-k // self.page), len(row)):
                    if self.ok(row[i]):
                        self.refs[row[i]] -= 1
                    row[i] = -1

    def fork(self, ctx, parents, children):
        done, n = [], len(self.table)
        for f, (p, c) in enumerate(zip(parents, children)):
            bad = not (0 <= p < n and 0 <= c < n) or c in parents or c in children[:f]
            bad = bad or any(self.ok(e) for e in self.table[c])
            done.append(int(bad))
            if bad:
                continue
            for i in range(len(self.table[c])):
                e = self.table[p][i] if i < -(-ctx[p] // self.page) else -1
                self.table[c][i] = e if self.ok(e) else -1
                if self.ok(e):
                    self.refs[e] += 1
        return done

    def reserve(self, ctx, cu):
        free = [i for i, r in enumerate(self.refs) if r == 0]
        start, given, dry = list(self.refs), 0, False
        missing, src, dst, rows = [], [], [], []
        for s, row in enumerate(self.table):
            new = cu[s + 1] - cu[s]
            lo, hi = ctx[s] // self.page, -(-(ctx[s] + new) // self.page)
            want = [i for i in range(lo, min(hi, len(row)))
                    if not self.ok(row[i]) or start[row[i]] > 1] if new > 0 else []
            over = max(0, hi - len(row)) if new > 0 else 0
            src.append(-1), dst.append(-1), rows.append(0)
            dry = dry or (bool(want) and not over and given + len(want) > len(free))
            if over or (want and dry):
                missing.append(len(want) + over)
                continue
            missing.append(0)
            for i in want:
                old, row[i] = row[i], free[given]
                given += 1
                self.refs[row[i]] += 1
                if self.ok(old):
                    self.refs[old] -= 1
                    if i == lo and ctx[s] % self.page:
                        src[-1], dst[-1], rows[-1] = old, row[i], ctx[s] % self.page
        return missing, src, dst, rows
