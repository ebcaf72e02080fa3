"""The position, cache and cached-attention calls together, as a program runs them:
a prompt in chunks, samples forked from it, a drafted tree verified and its path
kept, captured decode steps; and the norms around the attention core in training."""
import math

import pytest
import torch

import cache_reference as C
import paper_2301_08658_amd as atp

pytestmark = pytest.mark.gpu
DEV, BF, D = "cuda:0", torch.bfloat16, 128
I32 = dict(dtype=torch.int32, device=DEV)


def ints(v):
    return torch.tensor(v, **I32)


def rope(seed=1):
    g = torch.Generator().manual_seed(seed)
    qw = (1 + 0.1 * torch.randn(D, generator=g)).to(BF).to(DEV)
    kw = (1 + 0.1 * torch.randn(D, generator=g)).to(BF).to(DEV)
    inv = (10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)).float().to(DEV)
    return atp.qk_norm_rope(qw, kw, 1e-6, inv, D), C.Rope(qw, kw, 1e-6, inv, D)


class Server:
    """One layer's cache and a batch of sequences, stepped by the calls."""

    def __init__(self, kv, group, page, n_pages, seqs, cols, seed=1):
        self.kv, self.group, self.page, self.seqs = kv, group, page, seqs
        self.pool = torch.full((n_pages, 2, kv, page, D), math.nan, dtype=BF, device=DEV)
        self.cache = atp.kv_cache(self.pool)
        self.table = torch.full((seqs, cols), -1, **I32)
        self.refs = torch.zeros((n_pages,), **I32)
        self.ctx = torch.zeros((seqs,), **I32)
        self.cu = torch.zeros((seqs + 1,), **I32)
        self.batch = atp.kv_batch(self.table, self.ctx, self.cu)
        self.ws = torch.empty(atp.atp_cache_workspace_bytes(n_pages, seqs), dtype=torch.uint8,
                              device=DEV)
        self.lists = [torch.empty((seqs,), **I32) for _ in range(4)]
        self.gpu, self.ref = rope(seed)

    def lengths(self, new):
        self.cu.copy_(ints([sum(new[:i]) for i in range(self.seqs + 1)]))

    def pages(self):
        atp.atp_cache_reserve(self.page, self.refs, self.batch, *self.lists, self.ws)
        atp.atp_cache_copy_pages(self.cache, *self.lists[1:])

    def attend(self, x, max_new, positions=None, mask=None):
        t = x.shape[0]
        q = torch.empty((t, self.kv * self.group * D), dtype=BF, device=DEV)
        out = torch.full_like(q, 9.0)
        ws = torch.empty(atp.atp_attention_cache_workspace_bytes(self.kv, self.group, max_new),
                         dtype=torch.uint8, device=DEV)
        atp.atp_qk_norm_rope_cache(self.cache, self.batch, t, self.group, self.gpu, x, q, positions)
        atp.atp_attention_cache_fwd(self.cache, self.batch, t, self.group, max_new, q, out,
                                    tree_mask=mask, workspace=ws)
        return out

    def step(self, x, new, positions=None, mask=None, grow=True):
        self.lengths(new)
        self.pages()
        assert not self.lists[0].any()
        out = self.attend(x, max(new), positions, mask)
        if grow:
            self.ctx += ints(new)
        return out


def whole(srv, x):
    """Causal attention of one sequence's rows from nothing, in 64 bits, from the
    queries, keys and values rounded once to bf16 -> (out, bound)."""
    t, kv, group = x.shape[0], srv.kv, srv.group
    y, _ = C.norm_rope(srv.ref, C.heads(x, kv, group), group, torch.arange(t))
    y = y.float().to(BF).double()
    out, bound = [], []
    for h in range(kv):
        k, v = y[:, h, group], y[:, h, group + 1]
        for m in range(group):
            s = y[:, h, m] @ k.T / math.sqrt(D)
            s = s.masked_fill(~torch.ones(t, t).tril().bool(), -math.inf)
            w = torch.softmax(s, -1)
            out.append(w @ v)
            size = (y[:, h, m].abs() @ k.abs().T).amax(-1, keepdim=True) / math.sqrt(D)
            # the GPU's bf16 queries and keys may round the other way at a tie of
            # fp32 and 64-bit values: one more half step of a few of 128 products,
            # bounded by a half step of the score's largest product sum / 8
            ds = size * (2 * 128 * C.EPS32 + C.HALF_BF16 / 8)
            bound.append(C.HALF_BF16 * out[-1].abs() + (C.HALF_BF16 + 2 * ds) * (w @ v.abs()))
    return torch.cat(out, 1), torch.cat(bound, 1)


def close(got, want, bound):
    err = (C.f64(got) - want).abs()
    assert (err <= bound).all(), float((err - bound).max())


@pytest.mark.parametrize("group,page", [(1, 16), (4, 64)])
def test_prompt_samples_tree_and_decode(group, page):
    """A prompt enters in two chunks beside another sequence; it is forked into two
    samples; each gets its own next tokens (the shared last page is copied); a tree is
    drafted on one, its path kept, and the next token attends over it: every output
    is that of plain causal attention over the tokens that the sequence then has."""
    kv, seqs = 2, 4
    srv = Server(kv, group, page, 24 if page == 64 else 60, seqs, 12)
    w = kv * (group + 2) * D
    g = torch.Generator().manual_seed(5)
    rows = lambda n: torch.randn((n, w), generator=g).to(BF).to(DEV)      # noqa: E731
    prompt, other = rows(90), rows(21)
    a = srv.step(torch.cat((prompt[:50], other)), [50, 21, 0, 0])
    b = srv.step(prompt[50:], [40, 0, 0, 0])
    want, bound = whole(srv, prompt)
    close(torch.cat((a[:50], b)), want, bound)
    w2, b2 = whole(srv, other)
    close(a[50:], w2, b2)

    done = torch.empty((2,), **I32)
    atp.atp_cache_fork(page, srv.refs, srv.batch, ints([0, 0]), ints([2, 3]), done)
    assert not done.any()
    srv.ctx[2:] = 90
    before = srv.pool[srv.table[0, :6].clamp(min=0).long()].clone()
    x = rows(6)                                 # 1 and 2 tokens: each its own
    out = srv.step(x, [0, 3, 1, 2])
    after = srv.pool[srv.table[0, :6].clamp(min=0).long()]
    assert torch.equal(before.view(torch.int16), after.view(torch.int16))   # the prompt's pages
    hist = [prompt, torch.cat((other, x[:3])), torch.cat((prompt, x[3:4])),
            torch.cat((prompt, x[4:]))]
    for s, (lo, hi) in enumerate(((0, 0), (0, 3), (3, 4), (4, 6))):
        if hi > lo:
            want, bound = whole(srv, hist[s])
            close(out[lo:hi], want[lo - hi:], bound[lo - hi:])

    # a tree of 6 drafts on sequence 2: 0 - 1 - 4, 0 - 2 - 5, 3; and one token on 3
    parents = [-1, 0, 0, -1, 1, 2]
    anc = []
    for j, p in enumerate(parents):
        anc.append((anc[p] if p >= 0 else 0) | 1 << j)
    depth = [bin(v).count("1") - 1 for v in anc]
    mask = torch.tensor(anc + [1], dtype=torch.int64, device=DEV).reshape(-1, 1)
    base = srv.ctx.tolist()
    x = rows(7)
    out = srv.step(x, [0, 0, 6, 1], ints([base[2] + d for d in depth] + [base[3]]), mask,
                   grow=False)
    for j in range(6):
        path = [i for i in range(6) if anc[j] >> i & 1]
        want, bound = whole(srv, torch.cat((hist[2], x[path])))
        close(out[j:j + 1], want[-1:], bound[-1:])
    moved = torch.empty((seqs,), **I32)
    atp.atp_cache_compact(srv.cache, srv.batch, ints([0, 0, 0, 3, 4]), ints([0, 2, 5, 0]), moved)
    assert moved.tolist() == [0, 0, 3, 1]
    hist[2], hist[3] = torch.cat((hist[2], x[[0, 2, 5]])), torch.cat((hist[3], x[6:]))
    srv.ctx += moved
    keep = srv.ctx.clone()
    keep[:2] = -1
    atp.atp_cache_release(page, srv.refs, srv.batch, keep)
    x = rows(2)
    out = srv.step(x, [0, 0, 1, 1])
    for s in (2, 3):
        want, bound = whole(srv, torch.cat((hist[s], x[s - 2:s - 1])))
        close(out[s - 2:s - 1], want[-1:], bound[-1:])
    atp.atp_cache_release(page, srv.refs, srv.batch, ints([0] * seqs))
    assert not srv.refs.any() and (srv.table == -1).all()


def test_agrees_with_the_attention_core():
    """A whole prompt at once is the training path's result (norms into the block,
    then the attention core), up to both paths' bounds: the same bf16 queries and
    keys, weights of either path rounded to bf16."""
    kv, t = 2, 200
    srv = Server(kv, 1, 64, 8, 1, 4)
    x = torch.randn((t, kv * 3 * D), generator=torch.Generator().manual_seed(6)).to(BF).to(DEV)
    got = srv.step(x, [t])
    m = atp.mesh(1, 1, 0, 0)
    y = torch.empty_like(x)
    atp.atp_qk_norm_rope_fwd(1, t, kv, 1, srv.gpu, x, y)
    out = torch.empty((t, kv * D), dtype=BF, device=DEV)
    lse = torch.empty((kv, t), device=DEV)
    atp.atp_attention_fwd(m, atp.ATP_BLOCK_COL, 1, t, kv * D, kv, y, out, lse)
    want, bound = whole(srv, x)
    close(out, want, bound)
    close(got, C.f64(out), 2 * bound)


def test_captured_steps_grow():
    """One captured decode step (pages, cache, attention; all lengths on the device)
    replayed while the sequences grow, with eager work between, against the same
    steps run eagerly; two graphs share their workspaces."""
    kv, group, page, seqs, steps = 2, 2, 16, 3, 40
    w = kv * (group + 2) * D
    x = torch.randn((steps, seqs, w), generator=torch.Generator().manual_seed(7)).to(BF).to(DEV)
    runs = []
    for captured in (False, True):
        srv = Server(kv, group, page, 30, seqs, 8)
        srv.ctx.copy_(ints([5, 0, 30]))
        srv.lengths([1] * seqs)
        for s in range(seqs):                     # the tokens cached before
            srv.table[s, :2] = ints([3 * s, 3 * s + 1])
            srv.refs[3 * s:3 * s + 2] += 1
        srv.pool.copy_(torch.randn(srv.pool.shape, generator=torch.Generator().manual_seed(8)))
        cur = torch.empty((seqs, w), dtype=BF, device=DEV)
        q = torch.empty((seqs, kv * group * D), dtype=BF, device=DEV)
        out = torch.empty_like(q)
        ws = torch.empty(atp.atp_attention_cache_workspace_bytes(kv, group, 1), dtype=torch.uint8,
                         device=DEV)

        def step():
            srv.pages()
            atp.atp_qk_norm_rope_cache(srv.cache, srv.batch, seqs, group, srv.gpu, cur, q)
            atp.atp_attention_cache_fwd(srv.cache, srv.batch, seqs, group, 1, q, out, workspace=ws)

        graphs = []
        if captured:
            torch.cuda.synchronize()
            for _ in range(2):
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph):
                    step()
                graphs.append(graph)
        outs = []
        for i in range(steps):
            cur.copy_(x[i])
            if captured:
                graphs[i % 2].replay()
            else:
                step()
            outs.append(out.clone())
            srv.ctx += 1
            if i % 7 == 0:
                torch.cuda.synchronize()
                (torch.ones((1000,), device=DEV) * 2).sum().item()
        runs.append((torch.stack(outs), srv.table.clone(), srv.refs.clone(), srv.pool.clone()))
    for a, b in zip(*runs):
        assert torch.equal(a.view(torch.int16) if a.dtype == BF else a,
                           b.view(torch.int16) if b.dtype == BF else b)


def test_training_gradient_through_the_attention_core():
    """d/dx of <attention(norm_rope(x)), d_out>: the calls' chain against central
    differences of the whole function in 64 bits along the chain's own gradient.  Each
    of the chain's five bf16 roundings (y, out, d_out's use, d_y, dx) and the core's
    two of the weights is at most 2^-8 of its value; along the gradient their sum is at
    most 7 x 2^-8 of sum |dx dir|."""
    kv, t = 2, 60
    gpu, ref = rope(3)
    g = torch.Generator().manual_seed(9)
    x = torch.randn((t, kv * 3 * D), generator=g).to(BF).to(DEV)
    d_out = torch.randn((t, kv * D), generator=g).to(BF).to(DEV)
    m, mode, h = atp.mesh(1, 1, 0, 0), atp.ATP_BLOCK_COL, kv * D
    y, dy, dx = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    out, lse = torch.empty_like(d_out), torch.empty((kv, t), device=DEV)
    delta = torch.empty((kv * t,), device=DEV)
    dqw, dkw = torch.empty(D, device=DEV), torch.empty(D, device=DEV)
    ws = torch.empty(atp.atp_qk_norm_rope_workspace_bytes(t), dtype=torch.uint8, device=DEV)

    def chain():
        atp.atp_qk_norm_rope_fwd(1, t, kv, 1, gpu, x, y)
        atp.atp_attention_fwd(m, mode, 1, t, h, kv, y, out, lse)
        atp.atp_attention_bwd(m, mode, 1, t, h, kv, y, out, lse, d_out, dy, delta)
        atp.atp_qk_norm_rope_bwd(1, t, kv, 1, gpu, x, dy, dx, dqw, dkw, ws)

    chain()

    def f(xd, p):
        z, _ = C.norm_rope(p, xd, 1, torch.arange(t))
        total = 0.0
        for i in range(kv):
            s = z[:, i, 0] @ z[:, i, 1].T / math.sqrt(D)
            s = s.masked_fill(~torch.ones(t, t).tril().bool(), -math.inf)
            total += float((torch.softmax(s, -1) @ z[:, i, 2] *
                            C.f64(d_out)[:, i * D:(i + 1) * D]).sum())
        return total

    xd, got = C.heads(x, kv, 1), C.heads(dx, kv, 1)
    direction = got / got.norm()
    e = 1e-4
    diff = (f(xd + e * direction, ref) - f(xd - e * direction, ref)) / (2 * e)
    assert abs(float((got * direction).sum()) - diff) <= 7 * 2 ** -8 * float(
        (got * direction).abs().sum())
    for name, dw in (("qw", dqw), ("kw", dkw)):
        w = getattr(ref, name)
        d = C.f64(dw) / C.f64(dw).norm()
        vals = []
        for sign in (1, -1):
            setattr(ref, name, w + sign * e * d)
            vals.append(f(xd, ref))
        setattr(ref, name, w)
        diff = (vals[0] - vals[1]) / (2 * e)
        assert abs(float((C.f64(dw) * d).sum()) - diff) <= 7 * 2 ** -8 * float(
            (C.f64(dw) * d).abs().sum())

    # captured: the same bits on every replay
    want = [v.clone() for v in (y, out, dx, dqw, dkw)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain()
    for _ in range(3):
        for v in (y, out, dx, dqw, dkw):
            v.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        for v, r in zip((y, out, dx, dqw, dkw), want):
            assert torch.equal(v, r)


def test_profile_names_the_new_kernels():
    atp.atp_profile_enable(1)
    try:
        srv = Server(1, 1, 16, 4, 1, 2)
        x = torch.randn((3, 3 * D), device=DEV).to(BF)
        srv.step(x, [3])
        y = torch.empty_like(x)
        atp.atp_qk_norm_rope_fwd(1, 3, 1, 1, srv.gpu, x, y)
        stats = atp.atp_profile_collect()
    finally:
        atp.atp_profile_enable(0)
    names = {s["name"] if isinstance(s, dict) else s.name for s in stats}
    names = {n.decode() if isinstance(n, bytes) else n for n in names}
    assert {"cache_reserve", "cache_copy_pages", "qk_norm_rope_cache", "attention_cache",
            "qk_norm_rope_fwd"} <= names
