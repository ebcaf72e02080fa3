"""Performance cases of the serving and position operators around the attention
core: the norms of queries and keys with the position rotation, the paged
key/value cache, and the attention that reads it.

A pass is one call of an operator (or the short run of calls that a serving or
training step makes) on one device's run of heads.  With `own` false the same
outputs come from elementary torch operations.  Head dimension 128 everywhere,
as in the layer; a QKV row holds for each key/value head its `group` query
heads, the key and the value ([q .. q | k | v], 128 columns each).
"""
import math
import random

import torch

own = False

DEV = "cuda"
BF = torch.bfloat16
D = 128                                    # head dimension of every configuration
SCALE = 1.0 / math.sqrt(D)
EPS = 1e-6


# ------------------------------------------------------------------ the cases
def _norm(kind, batch, seq, kv, group, rot=D, interleaved=False, norm=True, weights=True,
          far=0, theta=10000.0):
    return dict(kind=kind, batch=batch, seq=seq, kv=kv, group=group, rot=rot,
                interleaved=interleaved, norm=norm, weights=weights, far=far, theta=theta)


def _cached(kind, seqs, ctx, new, kv, group, page, lens=1, tree=False, **kw):
    return dict(kind=kind, seqs=seqs, ctx_lo=ctx[0], ctx_hi=ctx[1], new_lo=new[0], new_hi=new[1],
                kv=kv, group=group, page=page, lens=lens, tree=tree, **kw)


def _rope(rot=D, interleaved=False, norm=True, weights=True, theta=10000.0):
    return dict(rot=rot, interleaved=interleaved, norm=norm, weights=weights, theta=theta)


def listed():
    cases = dict(
        # the smallest training call: two heads of a small layer, launch latency
        norm_fwd_h512=_norm("norm_fwd", 1, 256, 2, 1),
        # the widest layer's share (20 heads) at the paper's batch of 4 x 2048
        # tokens, forward and backward
        norm_step_h20480=_norm("norm_step", 4, 2048, 20, 1),
        # shared heads, a partial rotation of neighbouring pairs, far positions,
        # a ragged number of tokens: a long-context fine-tuning step's backward
        norm_bwd_odd=_norm("norm_bwd", 3, 1667, 5, 7, rot=48, interleaved=True, far=900000,
                           theta=500000.0),
        # a decode step writes one token of every sequence into the cache
        append_decode=_cached("append", 48, (10, 600), (1, 1), 20, 1, 64, **_rope()),
        # a ragged batch of prompts enters the cache
        append_prompts=_cached("append", 9, (0, 700), (1, 1500), 4, 8, 16,
                               **_rope(rot=64, interleaved=True)),
        # parallel sampling: every prompt is forked into 16 samples, which get
        # their next page (a copy of the prompt's last, partly filled one)
        pages_samples=_cached("samples", 6, (300, 2900), (1, 1), 10, 1, 64, samples=16),
        # a verified draft: the drafted rows are written and the accepted path
        # moved behind the context
        pages_accept=_cached("accept", 40, (20, 1500), (24, 63), 8, 4, 32, tree=True, **_rope()),
        # the smallest attention call: one sequence's next token
        attend_decode_small=_cached("attend", 1, (300, 300), (1, 1), 2, 1, 16),
        # a decode step of a large batch, ragged contexts
        attend_decode_batch=_cached("attend", 64, (200, 8000), (1, 1), 20, 1, 64),
        # verification of a tree of drafted tokens, shared key/value heads
        attend_tree=_cached("attend", 24, (500, 12000), (17, 64), 4, 5, 64, tree=True),
        # one token over a long context
        attend_long=_cached("attend", 1, (131000, 131000), (1, 1), 2, 8, 128),
        # prompts that enter in chunks: causal rows over what is cached already
        attend_chunk=_cached("attend", 4, (0, 6000), (500, 1024), 10, 1, 64),
    )
    return [dict(c, name=n) for n, c in cases.items()]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_rope(rng):
    return _rope(rot=rng.choice((0, 16, 32, 48, 64, 96, 120, 128)),
                 interleaved=rng.random() < 0.5, norm=rng.random() < 0.85,
                 weights=rng.random() < 0.8, theta=rng.choice((10000.0, 500000.0)))


def _draw_heads(rng):
    return rng.choice(((1, 1), (2, 1), (3, 1), (5, 1), (12, 1), (20, 1), (1, 8), (2, 4), (4, 5),
                       (2, 7), (1, 16), (8, 2), (1, 3)))


def draw(rng):
    kind = rng.choice(("norm_fwd", "norm_bwd", "norm_step", "append", "samples", "accept",
                       "attend", "attend", "attend"))
    kv, group = _draw_heads(rng)
    lens = rng.randrange(1, 1 << 30)
    page = rng.choice((16, 32, 64, 128, 256))
    rope = _draw_rope(rng)
    if kind.startswith("norm"):
        cols = kv * (group + 2)
        tokens = _log(rng, 1, min(40000, 8192 * 60 // cols))
        batch = rng.choice((1, 2, 3, 4)) if tokens > 16 else 1
        return _norm(kind, batch, max(1, tokens // batch), kv, group,
                     far=rng.choice((0, 0, 5000, 1000000)), **rope)
    if kind == "append":
        seqs = _log(rng, 1, 100)
        hi = _log(rng, 1, max(2, 12000 // seqs))
        return _cached("append", seqs, (0, _log(rng, 1, 500)), (rng.choice((0, 1, hi)), hi), kv,
                       group, page, lens, **rope)
    if kind == "samples":
        return _cached("samples", _log(rng, 1, 12), (1, _log(rng, 2, 2000)),
                       (0, _log(rng, 1, 200)), kv, group, page, lens,
                       samples=rng.choice((1, 2, 4, 7, 16)))
    if kind == "accept":
        return _cached("accept", _log(rng, 1, 60), (0, _log(rng, 1, 1200)),
                       (1, _log(rng, 1, 120)), kv, group, page, lens, tree=True, **rope)
    # attention: the cached tokens of the batch stay below the largest listed case's
    form = rng.choice(("decode", "decode", "tree", "chunk"))
    budget = 64 * 4100 * 20 // kv
    seqs = _log(rng, 1, 100) if form == "decode" else _log(rng, 1, 24)
    hi = _log(rng, 1, min(140000, budget // seqs))
    if form == "decode":
        new = (1, 1)
    elif form == "tree":
        new = (rng.choice((0, 1, 8)), _log(rng, 8, 128))
    else:
        new = (1, _log(rng, 2, 1500))
        hi = min(hi, 8000)
    return _cached("attend", seqs, (rng.choice((0, hi // 2, hi)), hi), new, kv, group, page, lens,
                   tree=form == "tree")


# ------------------------------------------------------------------ sizes
def _lens(case):
    """Cached and new tokens of every sequence (parents alone for "samples")."""
    r = random.Random(case["lens"])
    n = case["seqs"]
    ctx = [r.randint(case["ctx_lo"], case["ctx_hi"]) for _ in range(n)]
    new = [r.randint(case["new_lo"], case["new_hi"]) for _ in range(n)]
    return ctx, [max(1, new[0])] + new[1:]


def _up(a, b):
    return -(-a // b)


def work(case):
    kv, group = case["kv"], case["group"]
    head = 2 * D                                  # bytes of one head's row
    if case["kind"].startswith("norm"):
        t = case["batch"] * case["seq"]
        blk = t * kv * (group + 2) * head
        qk = t * kv * (group + 1) * head
        moved = {"norm_fwd": 2 * blk, "norm_bwd": qk + 2 * blk, "norm_step": qk + 4 * blk}
        flops = {"norm_fwd": 8, "norm_bwd": 16, "norm_step": 24}
        return {"bytes": moved[case["kind"]], "flops": flops[case["kind"]] * qk // 2}
    ctx, new = _lens(case)
    page, t = case["page"], sum(new)
    blk = t * kv * (group + 2) * head
    if case["kind"] == "append":
        return {"bytes": 2 * blk, "flops": 8 * t * kv * (group + 1) * D}
    if case["kind"] == "samples":
        n = case["samples"]
        copies = sum(n * (c % page) for c, a in zip(ctx, new) if a > 0) * 2 * kv * head
        tables = sum(_up(c + a, page) * 4 * n for c, a in zip(ctx, new))
        return {"bytes": 2 * copies + 3 * tables, "flops": 0}
    if case["kind"] == "accept":
        path = sum(max(1, a // 5) for a in new) * 2 * kv * head
        return {"bytes": 2 * blk + 2 * path, "flops": 8 * t * kv * (group + 1) * D}
    keys = sum(c + a for c, a in zip(ctx, new) if a > 0)
    drafted = 8 if case["tree"] else 1 << 30      # ancestors that a drafted token sees
    pairs = sum(a * c + sum(min(i + 1, drafted) for i in range(a)) for c, a in zip(ctx, new))
    return {"bytes": keys * kv * 2 * head + t * kv * group * (2 * head + 4),
            "flops": pairs * kv * group * 4 * D}


# ------------------------------------------------------------------ inputs
class _Gen:
    def __init__(self, seed):
        self.g = torch.Generator(device=DEV).manual_seed(seed * 1000003 + 17)

    def normal(self, shape, std=1.0, dtype=BF):
        return torch.randn(shape, generator=self.g, device=DEV, dtype=dtype) * std

    def ints(self, lo, hi, shape):
        return torch.randint(lo, hi, shape, generator=self.g, device=DEV, dtype=torch.int32)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _starts(v):
    out = [0]
    for n in v:
        out.append(out[-1] + n)
    return out


def _rope_inputs(case, g):
    """Norm weights around one and the inverse frequencies theta^(-2i / rot)."""
    rot = case["rot"]
    p = dict(qw=None, kw=None, inv_freq=None)
    if case["norm"] and case["weights"]:
        p["qw"] = (1.0 + g.normal((D,), 0.1, torch.float32)).to(BF)
        p["kw"] = (1.0 + g.normal((D,), 0.1, torch.float32)).to(BF)
    if rot:
        i = torch.arange(0, rot, 2, dtype=torch.float64, device=DEV)
        p["inv_freq"] = torch.pow(torch.tensor(case["theta"], dtype=torch.float64, device=DEV),
                                  -i / rot).float()
    if own:
        import paper_2301_08658_amd as atp
        p["own"] = atp.qk_norm_rope(q_weight=p["qw"], k_weight=p["kw"], eps=EPS,
                                    inv_freq=p["inv_freq"], rotary_dims=rot,
                                    interleaved=case["interleaved"], norm=case["norm"])
    return p


def _prepare_norm(case, seed):
    g = _Gen(seed)
    t, cols = case["batch"] * case["seq"], case["kv"] * (case["group"] + 2) * D
    st = dict(case=case, rope=_rope_inputs(case, g), qkv=g.normal((t, cols)),
              out=torch.empty((t, cols), dtype=BF, device=DEV), positions=None)
    if case["far"]:
        start = g.ints(0, case["far"], (case["batch"], 1))
        st["positions"] = (start + torch.arange(case["seq"], device=DEV,
                                                dtype=torch.int32)).reshape(-1).contiguous()
    if case["kind"] != "norm_fwd":
        st["d_out"] = g.normal((t, cols))
        st["d_qkv"] = torch.empty((t, cols), dtype=BF, device=DEV)
        st["dqw"] = torch.empty((D,), device=DEV) if case["norm"] else None
        st["dkw"] = torch.empty((D,), device=DEV) if case["norm"] else None
        if own:
            import paper_2301_08658_amd as atp
            st["ws"] = torch.empty(atp.atp_qk_norm_rope_workspace_bytes(t), dtype=torch.uint8,
                                   device=DEV)
    return st


def _tables(case, g, ctx, new, extra=0):
    """Scattered pages for every sequence's cached and new tokens; `extra` free pages."""
    page = case["page"]
    need = [_up(c + a, page) for c, a in zip(ctx, new)]
    n_pages = sum(need) + max(2, sum(need) // 8) + extra
    order = torch.randperm(n_pages, generator=g.g, device=DEV).to(torch.int32)
    width = max(1, max(need))
    at = _starts(need)
    table = torch.full((len(need), width), -1, dtype=torch.int32, device=DEV)
    for s, n in enumerate(need):
        table[s, :n] = order[at[s]:at[s + 1]]
    return table, n_pages


def _pool(case, g, n_pages):
    return g.normal((n_pages, 2, case["kv"], case["page"], D))


def _tree(case, new, seed):
    """Parents of drafted tokens, as ancestor bits and depths."""
    r = random.Random(seed)
    words = _up(max(1, max(new)), 64)
    bits, depth, paths = [], [], []
    for n in new:
        anc, dep, par = [], [], []
        for j in range(n):
            p = r.randint(max(0, j - 8), j - 1) if j else -1
            par.append(p)
            anc.append((anc[p] if p >= 0 else 0) | (1 << j))
            dep.append(dep[p] + 1 if p >= 0 else 0)
        bits += anc
        depth += dep
        path, j = [], (r.randrange(max(1, n - 8), n) if n > 1 else n - 1)
        while j >= 0:                              # the accepted path, root first
            path.insert(0, j)
            j = par[j]
        paths.append(path)
    signed = [[(w >> (64 * k)) & ((1 << 64) - 1) for k in range(words)] for w in bits]
    signed = [[v - (1 << 64) if v >> 63 else v for v in row] for row in signed]
    mask = torch.tensor(signed, dtype=torch.int64, device=DEV).reshape(len(bits), words)
    return mask, depth, paths


def _prepare_cached(case, seed):
    g = _Gen(seed)
    ctx, new = _lens(case)
    kv, group, t = case["kv"], case["group"], sum(new)
    st = dict(case=case, ctx=ctx, new=new, at=_starts(new))
    if case["kind"] == "samples":
        n = case["samples"]
        kids = case["seqs"] * n
        extra = n * sum(_up(c % case["page"] + a, case["page"]) for c, a in zip(ctx, new))
        table, n_pages = _tables(case, g, ctx, [0] * len(ctx), extra)
        width = max(_up(c + a, case["page"]) for c, a in zip(ctx, new))
        full = torch.full((case["seqs"] + kids, width), -1, dtype=torch.int32, device=DEV)
        full[:case["seqs"], :table.shape[1]] = table
        st["parents"] = _ints([p for p in range(case["seqs"]) for _ in range(n)])
        st["children"] = _ints(list(range(case["seqs"], case["seqs"] + kids)))
        st["keep"] = _ints([-1] * case["seqs"] + [0] * kids)
        st["ctx"] = ctx + [c for c in ctx for _ in range(n)]
        st["new"] = [0] * len(ctx) + [a for a in new for _ in range(n)]
        st["at"] = _starts(st["new"])
        st["table"] = full
        refs = torch.zeros((n_pages,), dtype=torch.int32, device=DEV)
        refs.index_fill_(0, table[table >= 0].long(), 1)
        st["refs"] = refs
        rows = case["seqs"] + kids
        for k in ("missing", "src", "dst", "rows"):
            st[k] = torch.empty((rows,), dtype=torch.int32, device=DEV)
        st["done"] = torch.empty((kids,), dtype=torch.int32, device=DEV)
    else:
        st["table"], n_pages = _tables(case, g, ctx, new)
    st["pool"] = _pool(case, g, n_pages)
    st["d_ctx"], st["d_at"] = _ints(st["ctx"]), _ints(st["at"])
    if case["tree"]:
        st["mask"], depth, st["paths"] = _tree(case, new, seed)
        st["positions"] = _ints([c + depth[st["at"][s] + j] for s, c in enumerate(ctx)
                                 for j in range(new[s])])
    else:
        st["mask"], st["positions"] = None, None
    if case["kind"] in ("append", "accept"):
        st["rope"] = _rope_inputs(case, g)
        st["qkv"] = g.normal((t, kv * (group + 2) * D))
        st["q"] = torch.empty((t, kv * group * D), dtype=BF, device=DEV)
    if case["kind"] == "accept":
        st["d_keep_at"] = _ints(_starts([len(p) for p in st["paths"]]))
        st["d_keep"] = _ints([j for p in st["paths"] for j in p])
        st["moved"] = torch.empty((case["seqs"],), dtype=torch.int32, device=DEV)
    if case["kind"] == "attend":
        st["q"] = g.normal((t, kv * group * D))
        st["out"] = torch.empty((t, kv * group * D), dtype=BF, device=DEV)
        st["lse"] = torch.empty((kv * group, t), device=DEV)
    if own:
        import paper_2301_08658_amd as atp
        st["cache"] = atp.kv_cache(st["pool"])
        st["batch"] = atp.kv_batch(st["table"], st["d_ctx"], st["d_at"])
        if case["kind"] == "samples":
            st["ws"] = torch.empty(atp.atp_cache_workspace_bytes(n_pages, st["table"].shape[0]),
                                   dtype=torch.uint8, device=DEV)
        if case["kind"] == "attend":
            st["ws"] = torch.empty(
                atp.atp_attention_cache_workspace_bytes(kv, group, max(1, max(new))),
                dtype=torch.uint8, device=DEV)
    return st


def prepare(case, seed):
    f = _prepare_norm if case["kind"].startswith("norm") else _prepare_cached
    return f(case, seed)


# ------------------------------------------------------------------ the plain forms
def _positions(st):
    if st["positions"] is not None:
        return st["positions"]
    c = st["case"]
    if "seq" in c:
        return torch.arange(c["seq"], device=DEV).repeat(c["batch"])
    owner, local = _owners(st)
    return st["d_ctx"].long()[owner] + local


def _owners(st):
    """Sequence of every new token and its index among the sequence's new ones."""
    t = st["at"][-1]
    new = st["d_at"][1:].long() - st["d_at"][:-1].long()
    owner = torch.repeat_interleave(torch.arange(len(st["ctx"]), device=DEV), new, output_size=t)
    return owner, torch.arange(t, device=DEV) - st["d_at"].long()[owner]


def _angles(case, inv_freq, positions):
    a = positions.double()[:, None] * inv_freq.double()[None, :]     # far positions: 64 bits
    return torch.cos(a).float()[:, None, None, :], torch.sin(a).float()[:, None, None, :]


def _rotate(case, x, cos, sin):
    rot, half = case["rot"], case["rot"] // 2
    if case["interleaved"]:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        r = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = x[..., :half], x[..., half:rot]
        r = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((r, x[..., rot:]), -1)


def _split(case, block):
    """Queries [t, kv, group, D] and keys [t, kv, 1, D] of QKV rows in 32 bits; values as given."""
    g = case["group"]
    x = block.view(block.shape[0], case["kv"], g + 2, D)
    return x[:, :, :g].float(), x[:, :, g:g + 1].float(), x[:, :, g + 1:]


def _plain_norm_rope(case, rope, block, positions):
    q, k, v = _split(case, block)
    if case["norm"]:
        q = q * torch.rsqrt((q * q).mean(-1, keepdim=True) + EPS)
        k = k * torch.rsqrt((k * k).mean(-1, keepdim=True) + EPS)
        if rope["qw"] is not None:
            q, k = q * rope["qw"].float(), k * rope["kw"].float()
    if case["rot"]:
        cos, sin = _angles(case, rope["inv_freq"], positions)
        q, k = _rotate(case, q, cos, sin), _rotate(case, k, cos, sin)
    return q.to(BF), k.to(BF), v


def _plain_fwd(st):
    case = st["case"]
    q, k, v = _plain_norm_rope(case, st["rope"], st["qkv"], _positions(st))
    return torch.cat((q, k, v), 2).reshape(st["qkv"].shape)


def _plain_bwd(st):
    case, rope = st["case"], st["rope"]
    xs, dys = _split(case, st["qkv"])[:2], _split(case, st["d_out"])
    grads, dws = [], []
    for x, dy, w in zip(xs, dys, (rope["qw"], rope["kw"])):
        if case["rot"]:
            cos, sin = _angles(case, rope["inv_freq"], _positions(st))
            dy = _rotate(case, dy, cos, -sin)
        if case["norm"]:
            r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
            xh = x * r
            dws.append((dy * xh).sum((0, 1, 2), dtype=torch.float64).float())
            u = dy * w.float() if w is not None else dy
            dy = r * (u - xh * (u * xh).mean(-1, keepdim=True))
        grads.append(dy.to(BF))
    return [torch.cat((*grads, dys[2]), 2).reshape(st["qkv"].shape), *dws]


def _slots(st, index):
    """Page and slot of token `index` of each new token's sequence."""
    owner, _ = _owners(st)
    page = st["case"]["page"]
    return st["table"].long()[owner, index // page], index % page


def _plain_append(st):
    case = st["case"]
    q, k, v = _plain_norm_rope(case, st["rope"], st["qkv"], _positions(st))
    owner, local = _owners(st)
    page, slot = _slots(st, st["d_ctx"].long()[owner] + local)
    st["pool"][page, 0, :, slot] = k[:, :, 0]
    st["pool"][page, 1, :, slot] = v[:, :, 0]
    return q.reshape(st["q"].shape)


def _plain_accept(st):
    q = _plain_append(st)
    pool, table, page = st["pool"], st["table"].long(), st["case"]["page"]
    counts = st["d_keep_at"][1:].long() - st["d_keep_at"][:-1].long()
    n = sum(len(p) for p in st["paths"])
    owner = torch.repeat_interleave(torch.arange(len(st["ctx"]), device=DEV), counts,
                                    output_size=n)
    rank = torch.arange(n, device=DEV) - st["d_keep_at"].long()[owner]
    base = st["d_ctx"].long()[owner]
    src, dst = base + st["d_keep"].long(), base + rank
    rows = pool[table[owner, src // page], :, :, src % page]
    pool[table[owner, dst // page], :, :, dst % page] = rows
    return [q, pool, counts.int()]


def _plain_samples(st):
    case = st["case"]
    page, table, refs = case["page"], st["table"], st["refs"]
    col = torch.arange(table.shape[1], device=DEV)
    # the last samples' pages are given back
    keep = st["keep"].long()[:, None]
    drop = (keep >= 0) & (col * page >= keep) & (table >= 0)
    refs.index_add_(0, table.clamp(min=0).long().reshape(-1), -drop.int().reshape(-1))
    table.masked_fill_(drop, -1)
    # every child shares its parent's pages
    held = table[st["parents"].long()]
    rows = torch.where(col * page < st["d_ctx"].long()[st["parents"].long()][:, None], held, -1)
    refs.index_add_(0, rows.clamp(min=0).long().reshape(-1), (rows >= 0).int().reshape(-1))
    table[st["children"].long()] = rows
    # the pages that the new tokens go to: free ones, or copies of shared ones
    ctx = st["d_ctx"].long()[:, None]
    new = (st["d_at"][1:].long() - st["d_at"][:-1].long())[:, None]
    written = (new > 0) & ((col + 1) * page > ctx) & (col * page < ctx + new)
    shared = (table >= 0) & (refs[table.clamp(min=0).long()] > 1)
    want = written & ((table < 0) | shared)
    free = torch.argsort((refs != 0).int(), stable=True)
    rank = (torch.cumsum(want.reshape(-1).int(), 0) - 1).clamp(min=0).reshape(want.shape)
    got = free[rank].int()
    first = want & shared & (col * page < ctx) & ((col + 1) * page > ctx)
    copy = first.any(1)
    src = torch.where(copy, torch.where(first, table, 0).sum(1), -1).int()
    dst = torch.where(copy, torch.where(first, got, 0).sum(1), -1).int()
    count = torch.where(copy, ctx[:, 0] % page, 0).int()
    refs.index_add_(0, table.clamp(min=0).long().reshape(-1), -(want & shared).int().reshape(-1))
    refs.index_add_(0, got.long().reshape(-1), want.int().reshape(-1))
    table.copy_(torch.where(want, got, table))
    # the rows of the copied pages
    pool = st["pool"]
    still = table[0, 0].long()                       # a prompt's page: never a destination
    a = torch.where(copy, src.long(), still)
    b = torch.where(copy, dst.long(), still)
    take = (torch.arange(page, device=DEV) < count[:, None])[:, None, None, :, None]
    pool[b] = torch.where(take, pool[a], pool[b])
    done = torch.zeros_like(st["children"])
    return [table, refs, done, torch.zeros_like(count), src, dst, count, pool]


def _visible(st, s, keys):
    """Which of `keys` cached tokens each new token of sequence s sees."""
    ctx, new, a = st["ctx"][s], st["new"][s], st["at"][s]
    k = torch.arange(keys, device=DEV) - ctx
    if st["mask"] is None:
        return k[None, :] <= torch.arange(new, device=DEV)[:, None]
    j = k.clamp(min=0)
    bits = (st["mask"][a:a + new][:, j // 64] >> (j % 64)) & 1
    return (k < 0)[None, :] | (bits != 0)


def _plain_attend(st):
    case = st["case"]
    kv, group, page = case["kv"], case["group"], case["page"]
    outs, lses = [], []
    for s, (c, n) in enumerate(zip(st["ctx"], st["new"])):
        if n == 0:
            continue
        a, keys = st["at"][s], c + n
        pages = st["table"][s, :_up(keys, page)].long()
        kvp = st["pool"][pages].permute(1, 2, 0, 3, 4).reshape(2, kv, -1, D)[:, :, :keys].float()
        q = st["q"][a:a + n].view(n, kv, group, D).permute(1, 0, 2, 3).float()
        score = torch.matmul(q.reshape(kv, n * group, D), kvp[0].transpose(1, 2)) * SCALE
        score = score.view(kv, n, group, keys)
        score = score.masked_fill(~_visible(st, s, keys)[None, :, None], -math.inf)
        top = score.amax(-1, keepdim=True).clamp(min=-3e38)
        p = torch.exp(score - top)
        total = p.sum(-1, keepdim=True)
        o = torch.matmul(p.view(kv, n * group, keys), kvp[1]).view(kv, n, group, D)
        o = torch.where(total > 0, o / total.clamp(min=1e-38), 0.0)
        outs.append(o.permute(1, 0, 2, 3).reshape(n, kv * group * D).to(BF))
        lse = (top + torch.log(total))[..., 0]
        lses.append(lse.permute(0, 2, 1).reshape(kv * group, n))
    if not outs:
        return [st["out"], st["lse"]]
    return [torch.cat(outs), torch.cat(lses, 1)]


def _run_plain(st):
    kind = st["case"]["kind"]
    if kind == "norm_fwd":
        return [_plain_fwd(st)]
    if kind == "norm_bwd":
        return _plain_bwd(st)
    if kind == "norm_step":
        return [_plain_fwd(st)] + _plain_bwd(st)
    if kind == "append":
        return [_plain_append(st), st["pool"]]
    return {"accept": _plain_accept, "samples": _plain_samples,
            "attend": _plain_attend}[kind](st)


# ------------------------------------------------------------------ the framework's calls
def _own_append(st):
    import paper_2301_08658_amd as atp
    atp.atp_qk_norm_rope_cache(st["cache"], st["batch"], st["at"][-1], st["case"]["group"],
                               st["rope"]["own"], st["qkv"], st["q"], positions=st["positions"])


def _run_own(st):
    import paper_2301_08658_amd as atp
    case = st["case"]
    kind, group = case["kind"], case["group"]
    if kind.startswith("norm"):
        out = []
        args = (case["batch"], case["seq"], case["kv"], group, st["rope"]["own"], st["qkv"])
        if kind != "norm_bwd":
            atp.atp_qk_norm_rope_fwd(*args, st["out"], positions=st["positions"])
            out.append(st["out"])
        if kind != "norm_fwd":
            atp.atp_qk_norm_rope_bwd(*args, st["d_out"], st["d_qkv"], dq_weight=st["dqw"],
                                     dk_weight=st["dkw"], workspace=st["ws"],
                                     positions=st["positions"])
            out += [st["d_qkv"]] + ([st["dqw"], st["dkw"]] if case["norm"] else [])
        return out
    if kind == "append":
        _own_append(st)
        return [st["q"], st["pool"]]
    if kind == "accept":
        _own_append(st)
        atp.atp_cache_compact(st["cache"], st["batch"], st["d_keep_at"], st["d_keep"],
                              st["moved"])
        return [st["q"], st["pool"], st["moved"]]
    if kind == "samples":
        n_pages, page = st["refs"].shape[0], case["page"]
        atp.atp_cache_release(page, st["refs"], st["batch"], st["keep"])
        atp.atp_cache_fork(page, st["refs"], st["batch"], st["parents"], st["children"],
                           st["done"])
        atp.atp_cache_reserve(page, st["refs"], st["batch"], st["missing"], st["src"], st["dst"],
                              st["rows"], st["ws"])
        atp.atp_cache_copy_pages(st["cache"], st["src"], st["dst"], st["rows"])
        return [st["table"], st["refs"], st["done"], st["missing"], st["src"], st["dst"],
                st["rows"], st["pool"]]
    atp.atp_attention_cache_fwd(st["cache"], st["batch"], st["at"][-1], group,
                                max(1, max(st["new"])), st["q"], st["out"], lse=st["lse"],
                                tree_mask=st["mask"], workspace=st["ws"])
    return [st["out"], st["lse"]]


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------ 64-bit definitions
def _exact_heads(case, rope, block, positions):
    """y = R(angle) (w * x / rms(x)) head by head, pair by pair, in 64 bits; also the pieces."""
    t, kv, g, rot = block.shape[0], case["kv"], case["group"], case["rot"]
    x = block.double().reshape(t, kv, g + 2, D)
    w = torch.ones((g + 2, D), dtype=torch.float64, device=DEV)
    rms = torch.ones((t, kv, g + 2, 1), dtype=torch.float64, device=DEV)
    if case["norm"]:
        if rope["qw"] is not None:
            w[:g], w[g] = rope["qw"].double(), rope["kw"].double()
        rms[:, :, :g + 1] = torch.sqrt((x[:, :, :g + 1] ** 2).sum(-1, keepdim=True) / D + EPS)
    turn = torch.zeros((t, rot // 2), dtype=torch.float64, device=DEV)
    if rot:
        turn = positions.double().reshape(-1, 1) * rope["inv_freq"].double()
    i = torch.arange(rot // 2, device=DEV)
    first, second = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + rot // 2)
    return x, w, rms, turn[:, None, None, :], first, second


def _exact_turn(y, turn, first, second, heads, sign):
    a, b = y[:, :, :heads, first].clone(), y[:, :, :heads, second].clone()
    c, s = torch.cos(turn), sign * torch.sin(turn)
    out = y.clone()
    # assigned through a view of the turned heads
    view = out[:, :, :heads]
    view[..., first] = a * c - b * s
    view[..., second] = a * s + b * c
    return out


def _exact_norm_rope(case, rope, block, positions):
    x, w, rms, turn, first, second = _exact_heads(case, rope, block, positions)
    return _exact_turn(x / rms * w, turn, first, second, case["group"] + 1, 1.0)


def _exact_norm(case, st):
    rope, g = st["rope"], case["group"]
    pos = st["positions"]
    if pos is None:
        pos = torch.tensor([i % case["seq"] for i in range(case["batch"] * case["seq"])],
                           device=DEV)
    shape = st["qkv"].shape
    out = []
    if case["kind"] != "norm_bwd":
        out.append(_exact_norm_rope(case, rope, st["qkv"], pos).reshape(shape))
    if case["kind"] != "norm_fwd":
        x, w, rms, turn, first, second = _exact_heads(case, rope, st["qkv"], pos)
        dy = st["d_out"].double().reshape(x.shape)
        u = _exact_turn(dy, turn, first, second, g + 1, -1.0)
        xh = x / rms
        dx = u * w
        if case["norm"]:
            dx = (dx - xh * (dx * xh).sum(-1, keepdim=True) / D) / rms
        dx[:, :, g + 1] = dy[:, :, g + 1]
        out.append(dx.reshape(shape))
        if case["norm"]:
            out += [(u * xh)[:, :, :g].sum((0, 1, 2)), (u * xh)[:, :, g].sum((0, 1))]
    return out


def _exact_append(case, st):
    g, page = case["group"], case["page"]
    rows = [(s, c + j) for s, (c, n) in enumerate(zip(st["ctx"], st["new"])) for j in range(n)]
    if not rows:
        return [st["q"].double(), st["pool"].double()]
    pos = st["positions"]
    if pos is None:
        pos = torch.tensor([p for _, p in rows], device=DEV)
    y = _exact_norm_rope(case, st["rope"], st["qkv"], pos)
    table = st["table"].tolist()
    page_of = torch.tensor([table[s][p // page] for s, p in rows], device=DEV)
    slot = torch.tensor([p % page for _, p in rows], device=DEV)
    pool = st["pool"].double()
    pool[page_of, 0, :, slot] = y[:, :, g]
    pool[page_of, 1, :, slot] = y[:, :, g + 1]
    return [y[:, :, :g].reshape(st["q"].shape), pool]


def _exact_accept(case, st):
    q, pool = _exact_append(case, st)
    page, table = case["page"], st["table"].tolist()
    before = pool.clone()
    for s, (c, path) in enumerate(zip(st["ctx"], st["paths"])):
        for i, j in enumerate(path):
            to, fr = c + i, c + j
            pool[table[s][to // page], :, :, to % page] = \
                before[table[s][fr // page], :, :, fr % page]
    return [q, pool, torch.tensor([len(p) for p in st["paths"]], dtype=torch.int32, device=DEV)]


def _exact_samples(case, st):
    """The page bookkeeping one sequence and one page at a time."""
    page = case["page"]
    table, refs, pool = st["table"].tolist(), st["refs"].tolist(), st["pool"].double()
    for p, c in zip(st["parents"].tolist(), st["children"].tolist()):
        for i in range(_up(st["ctx"][p], page)):
            table[c][i] = table[p][i]
            refs[table[p][i]] += 1
    free = iter([i for i, r in enumerate(refs) if r == 0])
    start = list(refs)
    src, dst, rows = [], [], []
    for s, (c, n) in enumerate(zip(st["ctx"], st["new"])):
        src.append(-1)
        dst.append(-1)
        rows.append(0)
        if n == 0:
            continue
        for i in range(c // page, _up(c + n, page)):
            old = table[s][i]
            if old >= 0 and start[old] <= 1:
                continue
            table[s][i] = next(free)
            refs[table[s][i]] += 1
            if old >= 0:
                refs[old] -= 1
                if c % page:
                    src[s], dst[s], rows[s] = old, table[s][i], c % page
    for a, b, r in zip(src, dst, rows):
        if r:
            pool[b, :, :, :r] = pool[a, :, :, :r]
    zeros = [0] * len(src)
    return [_ints(table), _ints(refs), _ints([0] * len(st["children"])), _ints(zeros), _ints(src),
            _ints(dst), _ints(rows), pool]


def _exact_attend(case, st):
    """Softmax over the visible tokens, a block of keys at a time, head by head."""
    kv, group, page = case["kv"], case["group"], case["page"]
    out = torch.zeros((st["at"][-1], kv * group, D), dtype=torch.float64, device=DEV)
    lse = torch.empty((kv * group, st["at"][-1]), dtype=torch.float64, device=DEV)
    for s, (c, n) in enumerate(zip(st["ctx"], st["new"])):
        if n == 0:
            continue
        a, idx = st["at"][s], torch.arange(c + n, device=DEV)
        pg, slot = st["table"][s].long()[idx // page], idx % page
        sees = torch.zeros((n, c + n), dtype=torch.bool, device=DEV)
        sees[:, :c] = True
        if st["mask"] is None:
            sees[:, c:] = torch.ones((n, n), device=DEV).tril() > 0
        else:
            words = st["mask"][a:a + n].tolist()
            sees[:, c:] = torch.tensor([[(w[j // 64] >> (j % 64)) & 1 == 1 for j in range(n)]
                                        for w in words], device=DEV)
        for h in range(kv):
            k, v = st["pool"][pg, 0, h, slot].double(), st["pool"][pg, 1, h, slot].double()
            for m in range(group):
                hq = h * group + m
                q = st["q"][a:a + n, hq * D:(hq + 1) * D].double()
                logit = (q @ k.t().contiguous()) / math.sqrt(D)
                logit = torch.where(sees, logit, -math.inf)
                z = torch.logsumexp(logit, -1)
                lse[hq, a:a + n] = z
                w = torch.exp(logit - torch.where(z > -math.inf, z, 0.0)[:, None])
                out[a:a + n, hq] = w @ v
    return [out.reshape(st["q"].shape), lse]


def exact(case, seed):
    if case["kind"] == "attend":
        ctx, new = _lens(case)
        pairs = sum(a * (c + a) for c, a in zip(ctx, new)) * case["kv"] * case["group"]
        if pairs > 3e9:                            # 64-bit products: seconds
            return None
    st = prepare(case, seed)
    if case["kind"].startswith("norm"):
        return _exact_norm(case, st)
    return {"append": _exact_append, "accept": _exact_accept, "samples": _exact_samples,
            "attend": _exact_attend}[case["kind"]](case, st)
