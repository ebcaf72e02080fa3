"""Performance cases of what a device needs around its layers to train them on
packed documents: the embedding of the tokens and its gradient, the layer norms
(with the residual sum, and over rows whose columns lie on several devices), the
attention within documents, and the norm and clipping of the gradients.

A pass is one call of an operator, or the forward and backward call that a
training step makes, on one device's share.  With `own` false the same outputs
come from elementary torch operations.  Head dimension 128 everywhere, as in the
layer; a QKV row holds for each key/value head its `group` query heads, the key
and the value ([q .. q | k | v], 128 columns each).
"""
import math
import random

import torch

own = False

DEV = "cuda"
BF = torch.bfloat16
D = 128                                    # head dimension of every configuration
SCALE = 1.0 / math.sqrt(D)
EPS = 1e-5


# ------------------------------------------------------------------ the cases
def _embed(kind, tokens, vocab, shards, cols, out="bf16", skew=True):
    return dict(kind="embed_" + kind, tokens=tokens, vocab=vocab, shards=shards, cols=cols,
                out=out, skew=skew)


def _norm(kind, tokens, cols, shards=1, stream="bf16", add=True, affine=True):
    return dict(kind="norm_" + kind, tokens=tokens, cols=cols, shards=shards, stream=stream,
                add=add, affine=affine)


def _clip(kind, shards, out="f32", **kw):
    return dict(kind="clip_" + kind, shards=shards, out=out, **kw)


def _attend(kind, docs, lens, kv, group, pad=0, cap=0.0, slopes=False, prefix=False, at=1):
    return dict(kind="attend_" + kind, docs=docs, len_lo=lens[0], len_hi=lens[1], kv=kv,
                group=group, pad=pad, cap=cap, slopes=slopes, prefix=prefix, at=at)


def listed():
    cases = dict(
        # the smallest training call: a tiny model's step, launch latency
        embed_step_small=_embed("step", 256, 1000, 1, 512),
        # a vocabulary over four devices: rows of other devices are zeros of this
        # one's partial sum
        embed_fwd_h4096=_embed("fwd", 8192, 50000, 4, 4096, out="f32"),
        # the widest layer's table, an eighth of the vocabulary: the gradient's rows
        # of tokens that occur hundreds of times, once, or not at all
        embed_bwd_h20480=_embed("bwd", 4096, 50000, 8, 20480),
        # the next token's norm of a small layer, latency
        norm_fwd_token=_norm("fwd", 1, 512),
        # the widest layer: the residual sum with the norm, and both gradients
        norm_step_h20480=_norm("step", 4096, 20480),
        # a quarter of every row, statistics of four devices, a 32-bit residual
        # stream, a ragged number of tokens
        norm_step_shards=_norm("step", 5003, 1024, 4, stream="f32"),
        # the gradients of the widest layer's share, one norm over eight devices
        clip_layer_h20480=_clip("layer", 8, h=20480, d1=8, d2=1, layers=1),
        # hundreds of tensors of all sizes, 16- and 32-bit, into one 16-bit buffer
        clip_many=_clip("many", 1, out="bf16", count=300, hi=200000, at=5),
        # the smallest attention call: one short document of two heads
        attend_fwd_small=_attend("fwd", 1, (300, 300), 2, 1),
        # a batch of packed documents of 20 to 1400 tokens at the widest layer's heads
        attend_step_packed=_attend("step", 12, (20, 1400), 20, 1, pad=37),
        # shared key/value heads, capped scores, long documents
        attend_step_capped=_attend("step", 3, (1500, 4096), 2, 8, cap=50.0, at=3),
        # prompts seen whole by their answers, a bias by distance
        attend_bwd_prefix=_attend("bwd", 9, (100, 1500), 4, 3, slopes=True, prefix=True, at=4),
    )
    return [dict(c, name=n) for n, c in cases.items()]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    form = rng.choice(("embed", "norm", "clip", "attend", "attend"))
    if form == "embed":
        cols = 8 * _log(rng, 8, 2560)
        vocab, shards = _log(rng, 300, 60000), rng.choice((1, 1, 2, 4, 8))
        while vocab // shards * cols > 120_000_000:
            shards *= 2
        tokens = _log(rng, 1, min(40000, 4096 * 20480 // cols))
        return _embed(rng.choice(("fwd", "bwd", "step")), tokens, vocab, shards, cols,
                      out=rng.choice(("bf16", "f32")), skew=rng.random() < 0.8)
    if form == "norm":
        cols = 8 * _log(rng, 8, 2560)
        tokens = _log(rng, 1, min(40000, 4096 * 20480 // cols))
        return _norm(rng.choice(("fwd", "step")), tokens, cols, rng.choice((1, 1, 1, 2, 4, 8)),
                     stream=rng.choice(("bf16", "f32")) if cols * tokens < 4e7 else "bf16",
                     add=rng.random() < 0.8, affine=rng.random() < 0.85)
    if form == "clip":
        out = rng.choice(("f32", "bf16"))
        if rng.random() < 0.4:
            d1, d2 = rng.choice(((1, 1), (2, 2), (2, 4), (8, 1)))
            return _clip("layer", d1 * d2, out, h=128 * d1 * d2 * rng.randrange(1, 9), d1=d1, d2=d2,
                         layers=rng.choice((1, 2, 3)))
        return _clip("many", rng.choice((1, 3, 8)), out, count=_log(rng, 1, 400),
                     hi=_log(rng, 10, 400000), at=rng.randrange(1, 1 << 30))
    kv, group = rng.choice(((1, 1), (2, 1), (5, 1), (12, 1), (20, 1), (1, 8), (2, 4), (4, 5),
                            (2, 7), (1, 16), (8, 2), (1, 3)))
    total = _log(rng, 4, int(math.sqrt(8192 * 8192 * 10 / (kv * group))))
    docs = _log(rng, 1, min(200, total))
    hi = max(1, min(total // docs, 8192))
    return _attend(rng.choice(("fwd", "bwd", "step")), docs, (rng.choice((0, 1, hi)), hi), kv,
                   group, pad=rng.choice((0, 0, 5, 130)), cap=rng.choice((0.0, 0.0, 30.0, 50.0)),
                   slopes=rng.random() < 0.4, prefix=rng.random() < 0.4,
                   at=rng.randrange(1, 1 << 30))


# ------------------------------------------------------------------ sizes
def _docs(case):
    """Lengths and prefixes of the documents."""
    r = random.Random(case["at"])
    lens = [r.randint(case["len_lo"], case["len_hi"]) for _ in range(case["docs"])]
    lens[0] = max(1, lens[0])
    return lens, [r.randint(0, n) if case["prefix"] else 0 for n in lens]


def _shard(case):
    """Rows of the vocabulary on this device (the first shard: the frequent tokens)."""
    return -(-case["vocab"] // case["shards"])


def _grads(case):
    """(rows, cols, bits) of every gradient."""
    if case["kind"] == "clip_layer":
        h, d1, d2 = case["h"], case["d1"], case["d2"]
        one = [(h // d2, 3 * h // d1), (h // d1, h // d2), (h // d2, 4 * h // d1),
               (4 * h // d1, h // d2)]
        one = [(r, c, 32) for r, c in one] + [(1, c, 32) for _, c in one]
        return one * case["layers"]
    r = random.Random(case["at"])
    out = []
    for _ in range(case["count"]):
        n = _log(r, 1, case["hi"])
        out.append((1, n, r.choice((16, 32))))
    return out


def work(case):
    kind = case["kind"]
    if kind.startswith("embed"):
        t, c, v = case["tokens"], case["cols"], _shard(case)
        wide = 4 if case["out"] == "f32" else 2
        fwd, bwd = t * c * (2 + wide) + 4 * t, t * c * 2 + v * c * 4 + 4 * t
        return {"bytes": (0 if kind == "embed_bwd" else fwd) + (0 if kind == "embed_fwd" else bwd),
                "flops": t * c * (1 if kind == "embed_fwd" else 2)}
    if kind.startswith("norm"):
        n, s = case["tokens"] * case["cols"], 4 if case["stream"] == "f32" else 2
        fwd = n * (s + 2 + (2 + s if case["add"] else 0))
        # the sum, the norm's gradient and the residual's are read, one gradient is written
        bwd = n * (3 * s + 2 + (2 if s == 4 else 0))
        return {"bytes": fwd + (bwd if kind == "norm_step" else 0) + 16 * case["tokens"],
                "flops": n * (8 if kind == "norm_fwd" else 22)}
    if kind.startswith("clip"):
        wide = 4 if case["out"] == "f32" else 2
        return {"bytes": sum(r * c * (b // 8 + wide) for r, c, b in _grads(case)),
                "flops": sum(3 * r * c for r, c, _ in _grads(case))}
    lens, prefix = _docs(case)
    kv, group, t = case["kv"], case["group"], sum(lens)
    pairs = sum(n * (n + 1) // 2 + p * (p - 1) // 2 for n, p in zip(lens, prefix))
    blk, rows = 2 * t * kv * (group + 2) * D, 2 * t * kv * group * D
    lse = 4 * t * kv * group
    moved = {"attend_fwd": blk + rows + lse, "attend_bwd": 2 * blk + 2 * rows + lse,
             "attend_step": 3 * blk + 3 * rows + 2 * lse}
    prods = {"attend_fwd": 4, "attend_bwd": 10, "attend_step": 14}
    return {"bytes": moved[kind], "flops": prods[kind] * D * pairs * kv * group}


# ------------------------------------------------------------------ inputs
class _Gen:
    def __init__(self, seed):
        self.g = torch.Generator(device=DEV).manual_seed(seed * 1000003 + 29)

    def normal(self, shape, std=1.0, dtype=BF):
        return torch.randn(shape, generator=self.g, device=DEV, dtype=dtype) * std

    def uniform(self, shape, dtype=torch.float32):
        return torch.rand(shape, generator=self.g, device=DEV, dtype=dtype)


def _wide(name):
    return torch.float32 if name == "f32" else BF


def _prepare_embed(case, seed):
    g = _Gen(seed)
    t, c, v = case["tokens"], case["cols"], _shard(case)
    u = g.uniform((t,), torch.float64)
    # token frequencies fall with the rank, as in text
    ids = torch.exp(u * math.log(case["vocab"] + 1)) - 1 if case["skew"] else u * case["vocab"]
    st = dict(case=case, ids=ids.to(torch.int32).clamp(0, case["vocab"] - 1), scale=math.sqrt(c))
    if case["kind"] != "embed_bwd":
        st["table"] = g.normal((v, c), 0.02)
        st["out"] = torch.empty((t, c), dtype=_wide(case["out"]), device=DEV)
    if case["kind"] != "embed_fwd":
        st["dy"] = g.normal((t, c), 0.01)
        st["dtable"] = torch.empty((v, c), device=DEV)
        if own:
            import paper_2301_08658_amd as atp
            st["ws"] = torch.empty(atp.atp_embedding_workspace_bytes(t, v, c), dtype=torch.uint8,
                                   device=DEV)
    return st


def _prepare_norm(case, seed):
    g = _Gen(seed)
    t, c, n = case["tokens"], case["cols"], case["shards"]
    dt = _wide(case["stream"])
    st = dict(case=case, own=n // 2)                 # this device's place in its group

    def shard():
        x = g.normal((t, c), 2.0, dt) + 0.5
        return x, g.normal((t, c)) if case["add"] else None
    st["x"], st["add"] = shard()
    st["w"] = (1.0 + g.normal((c,), 0.1, torch.float32)).to(BF) if case["affine"] else None
    st["b"] = g.normal((c,), 0.1) if case["affine"] else None
    st["x_out"] = torch.empty_like(st["x"]) if case["add"] else None
    st["y"] = torch.empty((t, c), dtype=BF, device=DEV)
    st["mean"], st["rstd"] = torch.empty((t,), device=DEV), torch.empty((t,), device=DEV)
    # the statistics of the other devices' columns: mean and centred squares, and the
    # backward's two sums
    st["stats"] = [torch.stack((0.5 + 2.2 * g.normal((t,), c ** -0.5, torch.float32),
                                4.9 * c * (1.0 + g.normal((t,), 0.02, torch.float32))), 1)
                   for _ in range(n)]
    if case["kind"] == "norm_step":
        st["dy"], st["d_res"] = g.normal((t, c), 0.1), g.normal((t, c), 0.1, dt)
        st["dx"] = torch.empty_like(st["x"])
        st["d_add"] = torch.empty((t, c), dtype=BF, device=DEV) if dt != BF else None
        st["dw"], st["db"] = torch.empty((c,), device=DEV), torch.empty((c,), device=DEV)
        st["sums"] = [g.normal((t, 2), 0.1 * c ** 0.5, torch.float32) for _ in range(n)]
    if own:
        import paper_2301_08658_amd as atp
        st["norm"] = atp.layer_norm(st["w"], st["b"], EPS)
        st["ws"] = torch.empty(atp.atp_layer_norm_workspace_bytes(t, c), dtype=torch.uint8,
                               device=DEV)
    return st


def _prepare_clip(case, seed):
    g = _Gen(seed)
    shapes = _grads(case)
    src = [g.normal((r, c), 0.01, torch.float32 if b == 32 else BF) for r, c, b in shapes]
    # the clipped gradients go into one buffer, each at a multiple of 8 values
    at = [0]
    for r, c, _ in shapes:
        at.append(at[-1] + -(-r * c // 8) * 8)
    flat = torch.zeros((at[-1],), dtype=_wide(case["out"]), device=DEV)
    dst = [flat[a:a + r * c].view(r, c) for a, (r, c, _) in zip(at, shapes)]
    sums = [(1.0 + g.uniform((1,), torch.float64)) * 30.0 for _ in range(case["shards"])]
    st = dict(case=case, src=src, flat=flat, dst=dst, sums=sums, own=case["shards"] // 2,
              norm=torch.empty((2,), device=DEV))
    if own:
        import paper_2301_08658_amd as atp
        st["grads"] = atp.grad_list(src, dst)
        st["ws"] = torch.empty(atp.atp_grad_workspace_bytes(st["grads"]), dtype=torch.uint8,
                               device=DEV)
    return st


def _prepare_attend(case, seed):
    g = _Gen(seed)
    lens, prefix = _docs(case)
    kv, group = case["kv"], case["group"]
    n = sum(lens)
    t = n + case["pad"]
    starts = [0]
    for k in lens:
        starts.append(starts[-1] + k)
    st = dict(case=case, tokens=t, rows=n,
              cu=torch.tensor(starts, dtype=torch.int32, device=DEV),
              prefix=torch.tensor(prefix, dtype=torch.int32, device=DEV) if case["prefix"] else None,
              slopes=None, qkv=g.normal((t, kv * (group + 2) * D)),
              out=torch.zeros((t, kv * group * D), dtype=BF, device=DEV),
              lse=torch.zeros((kv * group, t), device=DEV))
    if case["slopes"]:
        h = torch.arange(1, kv * group + 1, dtype=torch.float32, device=DEV)
        st["slopes"] = torch.exp2(-8.0 * h / (kv * group))
    if case["kind"] != "attend_fwd":
        st["d_out"] = g.normal((t, kv * group * D), 0.1)
        st["d_qkv"] = torch.zeros_like(st["qkv"])
    if case["kind"] == "attend_bwd":
        _plain_attend_fwd(st)                       # the forward's outputs are inputs here
    if own:
        import paper_2301_08658_amd as atp
        st["docs"] = atp.attention_docs(st["cu"], prefix=st["prefix"], slopes=st["slopes"],
                                        cap=case["cap"])
        st["ws"] = torch.empty(atp.atp_attention_docs_workspace_bytes(t, kv, group),
                               dtype=torch.uint8, device=DEV)
    return st


def prepare(case, seed):
    form = case["kind"].split("_")[0]
    return {"embed": _prepare_embed, "norm": _prepare_norm, "clip": _prepare_clip,
            "attend": _prepare_attend}[form](case, seed)


# ------------------------------------------------------------------ the plain forms
def _plain_embed(st):
    case, v, out = st["case"], _shard(st["case"]), []
    ids = st["ids"].long()
    here = ids < v                                   # this device holds the first shard
    if case["kind"] != "embed_bwd":
        rows = st["table"][torch.where(here, ids, 0)].float() * st["scale"]
        out.append(torch.where(here[:, None], rows, 0.0).to(_wide(case["out"])))
    if case["kind"] != "embed_fwd":
        grad = torch.zeros((v + 1, case["cols"]), device=DEV)
        grad.index_add_(0, torch.where(here, ids, v), st["dy"].float() * st["scale"])
        out.append(grad[:v])
    return out


def _plain_norm(st):
    case, n, c = st["case"], st["case"]["shards"], st["case"]["cols"]
    x = st["x"]
    if case["add"]:
        x = (x.float() + st["add"].float()).to(x.dtype)
    out = [x] if case["add"] else []
    xf = x.float()
    mean = xf.mean(1)
    m2 = (xf - mean[:, None]).square().sum(1)
    if n > 1:
        stats = torch.stack([torch.stack((mean, m2), 1) if j == st["own"] else s
                             for j, s in enumerate(st["stats"])])
        mean = stats[:, :, 0].mean(0)
        m2 = stats[:, :, 1].sum(0) + c * (stats[:, :, 0] - mean).square().sum(0)
    rstd = torch.rsqrt(m2 / (n * c) + EPS)
    xh = (xf - mean[:, None]) * rstd[:, None]
    w = st["w"].float() if case["affine"] else 1.0
    y = xh * w + (st["b"].float() if case["affine"] else 0.0)
    out += [y.to(BF), mean, rstd]
    if case["kind"] == "norm_fwd":
        return out
    dy = st["dy"].float()
    g = dy * w
    sums = torch.stack((g.sum(1), (g * xh).sum(1)), 1)
    if n > 1:
        sums = torch.stack([sums if j == st["own"] else s
                            for j, s in enumerate(st["sums"])]).sum(0)
    sums = sums / (n * c)
    dx = rstd[:, None] * (g - sums[:, :1] - xh * sums[:, 1:]) + st["d_res"].float()
    out.append(dx.to(x.dtype))
    if case["stream"] == "f32":
        out.append(dx.to(BF))
    return out + [(dy * xh).sum(0), dy.sum(0)]


def _plain_clip(st):
    total = torch.stack([s.float().square().sum(dtype=torch.float64) for s in st["src"]]).sum()
    parts = [total if j == st["own"] else s[0] for j, s in enumerate(st["sums"])]
    norm = torch.sqrt(torch.stack(parts).sum()) * 0.5
    factor = 0.5 * torch.where(norm > 1.0, 1.0 / norm, 1.0)
    torch._foreach_copy_(st["dst"], [s.float() * factor.float() for s in st["src"]])
    return [st["flat"], torch.stack((norm, factor)).float()]


def _visible(st):
    """Which keys each row sees, and the distances."""
    n = st["rows"]
    i = torch.arange(n, device=DEV)
    doc = torch.searchsorted(st["cu"][1:].contiguous(), i.to(torch.int32), right=True)
    sees = i[None, :] <= i[:, None]
    if st["prefix"] is not None:
        ends = st["cu"][:-1] + st["prefix"]
        sees = sees | (i < ends[doc])[None, :]
    return sees & (doc[None, :] == doc[:, None]), (i[:, None] - i[None, :]).abs().float()


def _heads(st, x, first, count):
    """Heads [first, first + count) of every key/value head's run, [kv, count * rows, D]."""
    kv, n = st["case"]["kv"], st["rows"]
    x = x[:n].view(n, kv, -1, D)[:, :, first:first + count]
    return x.permute(1, 2, 0, 3).reshape(kv, count * n, D).float()


def _plain_scores(st):
    """Scores of all pairs, [kv, group * rows, rows], and tanh of the capped ones."""
    case, n = st["case"], st["rows"]
    kv, group = case["kv"], case["group"]
    q, k = _heads(st, st["qkv"], 0, group), _heads(st, st["qkv"], group, 1)
    s = torch.matmul(q, k.transpose(1, 2).contiguous()) * SCALE
    t = None
    if case["cap"]:
        t = torch.tanh(s / case["cap"])
        s = t * case["cap"]
    sees, far = _visible(st)
    s = s.view(kv, group, n, n)
    if st["slopes"] is not None:
        s = s - st["slopes"].view(kv, group, 1, 1) * far
    return s.masked_fill(~sees, -math.inf).view(kv, group * n, n), t


def _rows_of(st, x, count):
    """[kv, count * rows, D] back to [rows, kv, count, D]."""
    return x.view(st["case"]["kv"], count, st["rows"], D).permute(2, 0, 1, 3)


def _plain_attend_fwd(st):
    case, n = st["case"], st["rows"]
    kv, group = case["kv"], case["group"]
    s, _ = _plain_scores(st)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - top)
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, _heads(st, st["qkv"], group + 1, 1)) / total
    st["out"][:n] = _rows_of(st, o, group).reshape(n, -1).to(BF)
    st["lse"][:, :n] = (top + torch.log(total)).view(kv * group, n)
    return [st["out"], st["lse"]]


def _plain_attend_bwd(st):
    case, n = st["case"], st["rows"]
    kv, group = case["kv"], case["group"]
    s, t = _plain_scores(st)
    lse = st["lse"][:, :n].reshape(kv, group * n, 1)
    p = torch.exp(s - lse)
    do, o = _heads(st, st["d_out"], 0, group), _heads(st, st["out"], 0, group)
    v = _heads(st, st["qkv"], group + 1, 1)
    ds = p * (torch.matmul(do, v.transpose(1, 2).contiguous()) - (do * o).sum(-1, keepdim=True))
    if t is not None:
        ds = ds * (1.0 - t * t)
    ds = ds * SCALE
    q, k = _heads(st, st["qkv"], 0, group), _heads(st, st["qkv"], group, 1)
    grads = [_rows_of(st, torch.matmul(ds, k), group),
             _rows_of(st, torch.matmul(ds.transpose(1, 2).contiguous(), q), 1),
             _rows_of(st, torch.matmul(p.transpose(1, 2).contiguous(), do), 1)]
    st["d_qkv"][:n] = torch.cat(grads, 2).reshape(n, -1).to(BF)
    return [st["d_qkv"]]


def _plain_attend(st):
    kind = st["case"]["kind"]
    return ([] if kind == "attend_bwd" else _plain_attend_fwd(st)) + \
        ([] if kind == "attend_fwd" else _plain_attend_bwd(st))


def _run_plain(st):
    form = st["case"]["kind"].split("_")[0]
    return {"embed": _plain_embed, "norm": _plain_norm, "clip": _plain_clip,
            "attend": _plain_attend}[form](st)


# ------------------------------------------------------------------ the framework's calls
def _own_embed(st, atp):
    case, out = st["case"], []
    t = case["tokens"]
    if case["kind"] != "embed_bwd":
        atp.atp_embedding_fwd(t, st["ids"], st["table"], st["out"], scale=st["scale"])
        out.append(st["out"])
    if case["kind"] != "embed_fwd":
        atp.atp_embedding_bwd(t, st["ids"], st["dy"], st["dtable"], st["ws"], scale=st["scale"])
        out.append(st["dtable"])
    return out


def _own_norm(st, atp):
    case, t, me = st["case"], st["case"]["tokens"], st["own"]
    x, add, x_out, stats = st["x"], st["add"], st["x_out"], None
    if case["shards"] > 1:
        # the sum and this device's statistics, then the norm from everyone's
        atp.atp_layer_norm_stats(t, x, st["stats"][me], add=add, x_out=x_out)
        x, add, x_out, stats = (x_out if case["add"] else x), None, None, st["stats"]
    atp.atp_layer_norm_fwd(t, st["norm"], x, st["y"], st["mean"], st["rstd"], add=add,
                           x_out=x_out, stats=stats)
    x = st["x_out"] if case["add"] else st["x"]
    out = ([x] if case["add"] else []) + [st["y"], st["mean"], st["rstd"]]
    if case["kind"] == "norm_fwd":
        return out
    sums = None
    if case["shards"] > 1:
        sums = st["sums"]
        atp.atp_layer_norm_bwd_sums(t, st["norm"], x, st["mean"], st["rstd"], st["dy"], sums[me])
    atp.atp_layer_norm_bwd(t, st["norm"], x, st["mean"], st["rstd"], st["dy"], st["dx"],
                           d_res=st["d_res"], d_add=st["d_add"], sums=sums, dweight=st["dw"],
                           dbias=st["db"], workspace=st["ws"])
    return out + [st["dx"]] + ([st["d_add"]] if st["d_add"] is not None else []) + \
        [st["dw"], st["db"]]


def _own_clip(st, atp):
    atp.atp_grad_sq_sum(st["grads"], st["sums"][st["own"]], st["ws"])
    atp.atp_grad_clip(st["grads"], st["sums"], st["norm"], max_norm=1.0, scale=0.5)
    return [st["flat"], st["norm"]]


def _own_attend(st, atp):
    case = st["case"]
    args = (st["tokens"], case["kv"], case["group"], st["docs"], st["qkv"], st["out"], st["lse"])
    out = []
    if case["kind"] != "attend_bwd":
        atp.atp_attention_docs_fwd(*args)
        out += [st["out"], st["lse"]]
    if case["kind"] != "attend_fwd":
        atp.atp_attention_docs_bwd(*args, st["d_out"], st["d_qkv"], st["ws"])
        out.append(st["d_qkv"])
    return out


def _run_own(st):
    import paper_2301_08658_amd as atp
    form = st["case"]["kind"].split("_")[0]
    return {"embed": _own_embed, "norm": _own_norm, "clip": _own_clip,
            "attend": _own_attend}[form](st, atp)


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------ 64-bit definitions
def _exact_embed(case, st):
    v, out = _shard(case), []
    ids = st["ids"].tolist()
    mine = [t for t, i in enumerate(ids) if i < v]
    at = torch.tensor(mine, dtype=torch.long, device=DEV)
    row = torch.tensor([ids[t] for t in mine], dtype=torch.long, device=DEV)
    if case["kind"] != "embed_bwd":
        y = torch.zeros((case["tokens"], case["cols"]), dtype=torch.float64, device=DEV)
        y[at] = st["table"].double()[row] * st["scale"]
        out.append(y)
    if case["kind"] != "embed_fwd":
        dy = st["dy"].double()
        order = sorted(range(len(mine)), key=lambda k: ids[mine[k]])
        grad = torch.zeros((v, case["cols"]), dtype=torch.float64, device=DEV)
        k = 0
        while k < len(order):                        # one run of equal tokens after the other
            e = k
            while e < len(order) and ids[mine[order[e]]] == ids[mine[order[k]]]:
                e += 1
            rows = torch.tensor([mine[j] for j in order[k:e]], device=DEV)
            grad[ids[mine[order[k]]]] = dy[rows].sum(0) * st["scale"]
            k = e
        out.append(grad)
    return out


def _exact_norm(case, st):
    n, c, me = case["shards"], case["cols"], st["own"]
    x = st["x"].double()
    if case["add"]:
        x = (x + st["add"].double()).to(st["x"].dtype).double()
    out = [x.clone()] if case["add"] else []
    # moments of the whole rows: the sums of x and x^2 about zero
    first, second = x.sum(1), (x * x).sum(1)
    for j, s in enumerate(st["stats"]):
        if n > 1 and j != me:
            m, q = s[:, 0].double(), s[:, 1].double()
            first, second = first + c * m, second + q + c * m * m
    mean = first / (n * c)
    var = second / (n * c) - mean ** 2
    dev = torch.sqrt(var + EPS)
    xh = (x - mean.unsqueeze(1)) / dev.unsqueeze(1)
    gamma = st["w"].double() if case["affine"] else torch.ones(c, dtype=torch.float64, device=DEV)
    beta = st["b"].double() if case["affine"] else torch.zeros(c, dtype=torch.float64, device=DEV)
    out += [gamma * xh + beta, mean, 1.0 / dev]
    if case["kind"] == "norm_fwd":
        return out
    dy = st["dy"].double()
    a, b = dy @ gamma, (dy * xh) @ gamma
    for j, s in enumerate(st["sums"]):
        if n > 1 and j != me:
            a, b = a + s[:, 0].double(), b + s[:, 1].double()
    dx = (gamma * dy - (a / (n * c)).unsqueeze(1) - xh * (b / (n * c)).unsqueeze(1))
    dx = dx / dev.unsqueeze(1) + st["d_res"].double()
    out += [dx] if case["stream"] == "bf16" else [dx, dx]
    return out + [torch.einsum("tc,tc->c", dy, xh), dy.sum(0)]


def _exact_clip(case, st):
    total = sum(float((s.double() ** 2).sum()) for s in st["src"])
    total += sum(float(s) for j, s in enumerate(st["sums"]) if j != st["own"])
    norm = 0.5 * math.sqrt(total)
    factor = 0.5 * min(1.0, 1.0 / norm)
    flat = torch.zeros(st["flat"].shape, dtype=torch.float64, device=DEV)
    at = 0
    for s in st["src"]:
        flat[at:at + s.numel()] = s.double().reshape(-1) * factor
        at += -(-s.numel() // 8) * 8
    return [flat, torch.tensor([norm, factor], dtype=torch.float64, device=DEV)]


def _exact_attend(case, st):
    """Softmax within one document and one head at a time; gradients by the chain rule
    through the normalised weights."""
    lens, prefix = _docs(case)
    kv, group, t = case["kv"], case["group"], st["tokens"]
    x = st["qkv"].double().view(t, kv, group + 2, D)
    out = torch.zeros((t, kv, group, D), dtype=torch.float64, device=DEV)
    lse = torch.zeros((kv * group, t), dtype=torch.float64, device=DEV)
    dx = torch.zeros_like(x)
    back = case["kind"] != "attend_fwd"
    a = 0
    for n, pre in zip(lens, prefix):
        rows = slice(a, a + n)
        idx = torch.arange(n, device=DEV)
        hidden = torch.ones((n, n), dtype=torch.bool, device=DEV).triu(1)
        hidden[:, :pre] = False
        for h in range(kv * group if n else 0):
            u, m = divmod(h, group)
            q, k, v = x[rows, u, m], x[rows, u, group], x[rows, u, group + 1]
            z = (q @ k.T.contiguous()) / math.sqrt(D)
            slope = 1.0
            if case["cap"]:
                th = torch.tanh(z / case["cap"])
                z, slope = case["cap"] * th, 1.0 - th ** 2
            if st["slopes"] is not None:
                z = z - st["slopes"][h].double() * (idx[:, None] - idx[None, :]).abs()
            z[hidden] = -math.inf
            lse[h, rows] = torch.logsumexp(z, 1)
            w = torch.softmax(z, 1)
            out[rows, u, m] = w @ v
            if back:
                do = st["d_out"][rows, h * D:(h + 1) * D].double()
                dw = do @ v.T.contiguous()
                dz = w * (dw - (w * dw).sum(1, keepdim=True)) * slope / math.sqrt(D)
                dx[rows, u, m] = dz @ k
                dx[rows, u, group] += dz.T.contiguous() @ q
                dx[rows, u, group + 1] += w.T.contiguous() @ do
        a += n
    fwd = [out.reshape(t, -1), lse] if case["kind"] != "attend_bwd" else []
    return fwd + ([dx.reshape(t, -1)] if back else [])


def exact(case, seed):
    if case["kind"].startswith("attend"):
        pairs = sum(n * n for n in _docs(case)[0]) * case["kv"] * case["group"]
        if pairs > 2e9:                              # 64-bit products: seconds
            return None
    st = prepare(case, seed)
    form = case["kind"].split("_")[0]
    return {"embed": _exact_embed, "norm": _exact_norm, "clip": _exact_clip,
            "attend": _exact_attend}[form](case, st)
