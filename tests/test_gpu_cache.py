"""Pages of the cache on the GPU: reserving, forking, releasing, copying and
compacting, against bookkeeping one page at a time."""
import random

import pytest
import torch

import cache_reference as C
import paper_2301_08658_amd as atp

pytestmark = pytest.mark.gpu
DEV, BF, D = "cuda:0", torch.bfloat16, 128


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV).reshape(-1)


class Both:
    """The calls and the reference side by side."""

    def __init__(self, n_pages, page, seqs, cols, held=(), refs=None, pad=0):
        table = [[-1] * cols for _ in range(seqs)]
        for s, pages in held:
            table[s][:len(pages)] = pages
        if refs is None:
            refs = [0] * n_pages
            for row in table:
                for e in row:
                    if 0 <= e < n_pages:
                        refs[e] += 1
        self.ref = C.Pool(n_pages, page, refs, table)
        self.page, self.seqs = page, seqs
        self.table = torch.full((seqs, cols + pad), 77, dtype=torch.int32, device=DEV)[:, :cols]
        self.table.copy_(torch.tensor(table, dtype=torch.int32))
        self.refs = ints(refs)
        self.ws = torch.empty(atp.atp_cache_workspace_bytes(n_pages, seqs), dtype=torch.uint8,
                              device=DEV)

    def batch(self, ctx, new):
        cu = [0]
        for n in new:
            cu.append(cu[-1] + n)
        return atp.kv_batch(self.table, ints(ctx), ints(cu)), cu

    def same(self):
        assert self.table.tolist() == self.ref.table
        assert self.refs.tolist() == self.ref.refs

    def reserve(self, ctx, new):
        b, cu = self.batch(ctx, new)
        out = [ints([9] * self.seqs) for _ in range(4)]
        atp.atp_cache_reserve(self.page, self.refs, b, *out, self.ws)
        want = self.ref.reserve(ctx, cu)
        assert [o.tolist() for o in out] == [list(w) for w in want]
        self.same()
        return want

    def fork(self, ctx, parents, children):
        b, _ = self.batch(ctx, [0] * self.seqs)
        done = ints([9] * len(parents))
        atp.atp_cache_fork(self.page, self.refs, b, ints(parents), ints(children), done)
        assert done.tolist() == self.ref.fork(ctx, parents, children)
        self.same()

    def release(self, keep):
        atp.atp_cache_release(self.page, self.refs, atp.kv_batch(self.table), ints(keep))
        self.ref.release(keep)
        self.same()


def test_reserve_from_nothing():
    """One token, whole pages, none, prompts longer than a lane looks at."""
    for seqs, new in ((1, [1]), (5, [16, 17, 0, 1, 700]), (3, [0, 0, 0])):
        b = Both(80, 16, seqs, 50, pad=6)
        b.reserve([0] * seqs, new)
        b.reserve(new, [1] * seqs)


def test_reserve_copies_shared_pages():
    """A page that others hold is replaced; only one that holds cached tokens of the
    sequence is copied.  All holders writing at once give the old page back."""
    b = Both(40, 16, 6, 6)
    b.reserve([0] * 6, [37, 32, 0, 0, 0, 5])
    ctx = [37, 32, 0, 0, 0, 5]
    b.fork(ctx, [0, 0, 1], [2, 3, 4])
    ctx[2], ctx[3], ctx[4] = 37, 37, 32
    m, src, dst, rows = b.reserve(ctx, [0, 1, 2, 70, 1, 0])
    # sequence 3 would need a seventh column: it gets nothing
    assert rows == [0, 0, 5, 0, 0, 0] and [bool(x) for x in m] == [0, 0, 0, 1, 0, 0]
    b.reserve(ctx, [1, 0, 0, 1, 0, 20])
    b.release([-1, 20, 16, 17, 0, -1])
    # truncated into a page that is still shared: written only after a copy
    b.fork([37, 20, 16, 17, 0, 25], [0], [4])
    b.reserve([30, 20, 16, 17, 33, 25], [3, 0, 0, 0, 3, 0])


def test_reserve_all_write_at_once():
    b = Both(12, 16, 3, 2)
    b.reserve([0, 0, 0], [7, 0, 0])
    b.fork([7, 0, 0], [0, 0], [1, 2])
    before = b.table[0, 0].item()
    b.reserve([7, 7, 7], [1, 1, 1])
    assert b.refs.tolist()[before] == 0


def test_reserve_beyond_the_pool_and_the_table():
    """All or nothing, in order; a sequence that its table cannot hold takes nothing
    from those behind it."""
    b = Both(5, 16, 5, 3)
    m = b.reserve([0] * 5, [16, 64, 33, 32, 1])[0]
    assert m == [0, 4, 0, 2, 1]
    m = b.reserve([16, 0, 33, 0, 0], [0, 0, 0, 0, 1])[0]
    assert m == [0, 0, 0, 0, 0]
    assert b.reserve([16, 0, 33, 0, 1], [1, 0, 0, 0, 0])[0] == [1, 0, 0, 0, 0]


def test_reserve_ignores_invalid_entries():
    b = Both(10, 16, 2, 4, held=[(0, [3, 11, -7]), (1, [2])])
    b.reserve([16, 16], [30, 1])


def test_many_sequences_and_pages():
    """More sequences than the reserving workgroup has lanes; a pool whose free
    pages lie behind many used ones."""
    rng = random.Random(3)
    n_pages, seqs = 20000, 2500
    refs = [1 if rng.random() < 0.7 or i < 9000 else 0 for i in range(n_pages)]
    b = Both(n_pages, 32, seqs, 9, refs=refs)
    new = [rng.choice((0, 1, 31, 32, 33, 200)) for _ in range(seqs)]
    b.reserve([0] * seqs, new)
    b.release([rng.choice((-1, 0, 1, 32, 64)) for _ in range(seqs)])


@pytest.mark.parametrize("seed", range(4))
def test_random_histories(seed):
    rng = random.Random(seed)
    page = rng.choice((16, 32, 64))
    seqs, cols = rng.choice((3, 12, 70)), 7
    b = Both(rng.choice((20, 200)), page, seqs, cols)
    ctx = [0] * seqs
    for _ in range(12):
        new = [rng.choice((0, 0, 1, 1, 3, page, 90)) for _ in range(seqs)]
        missing = b.reserve(ctx, new)[0]
        ctx = [c if m else c + n for c, n, m in zip(ctx, new, missing)]
        k = rng.randint(1, 6)
        parents = [rng.randint(-1, seqs) for _ in range(k)]
        children = [rng.randint(-1, seqs) for _ in range(k)]
        probe = C.Pool(b.ref.n, page, b.ref.refs, b.ref.table)
        done = probe.fork(ctx, parents, children)
        b.fork(ctx, parents, children)
        for p, c, d in zip(parents, children, done):
            if not d:
                ctx[c] = ctx[p]
        keep = [rng.choice((-1, -1, 0, rng.randint(0, 100))) for _ in range(seqs)]
        b.release(keep)
        ctx = [min(c, k) if k >= 0 else c for c, k in zip(ctx, keep)]
    b.release([0] * seqs)
    assert not any(b.refs.tolist())


def test_fork_refusals():
    b = Both(30, 16, 6, 4, held=[(0, [5, 6]), (1, [7]), (2, [8, -1, 9])])
    b.fork([20, 3, 40, 0, 0, 0], [0, 0, 1, 9, -1, 4, 2, 3], [3, 3, 0, 4, 5, 4, 5, 1])
    b.fork([20, 3, 40, 0, 0, 0], [0], [0])


def test_copy_pages():
    n_pages, kv, page = 30, 3, 64
    pool = torch.randn((n_pages, 2, kv, page, D), generator=torch.Generator().manual_seed(1)).to(BF)
    src = [0, 1, 2, 2, 7, -1, 31, 4, 5, 9]
    dst = [20, 21, 22, 23, 7, 24, 25, 30, -2, 26]
    rows = [1, 64, 63, 100, 5, 5, 5, 5, 5, 0]
    for with_rows in (True, False):
        gpu = pool.to(DEV)
        atp.atp_cache_copy_pages(atp.kv_cache(gpu), ints(src), ints(dst),
                                 ints(rows) if with_rows else None)
        want = pool.clone()
        for a, z, r in zip(src, dst, rows):
            r = min(r, page) if with_rows else page
            if r > 0 and a != z and 0 <= a < n_pages and 0 <= z < n_pages:
                want[z, :, :, :r] = pool[a, :, :, :r]
        assert torch.equal(gpu.cpu().view(torch.int16), want.view(torch.int16))


@pytest.mark.parametrize("page,kv", [(16, 2), (64, 1), (256, 3)])
def test_compact(page, kv):
    """Paths across pages, none, all, one, long lists; refused: descending, repeated,
    negative, beyond the table, a place without a page."""
    rng = random.Random(page)
    cols, seqs = 6, 11
    cap = cols * page
    n_pages = seqs * cols + 3
    order = list(range(n_pages))
    rng.shuffle(order)
    table = [[order[s * cols + i] for i in range(cols)] for s in range(seqs)]
    ctx = [rng.randint(0, cap // 2) for _ in range(seqs)]
    room = [cap - c for c in ctx]
    keep = [sorted(rng.sample(range(room[s]), min(room[s], k)))
            for s, k in zip(range(seqs), (5, 0, 1, 300, 2, 4, 3, 3, 4, 9, 6))]
    keep[4] = list(range(room[4]))                     # all: nothing moves
    keep[5] = [0, 3, 2, 5]
    keep[6] = [1, 1, 2]
    keep[7] = [-1, 0, 4]
    keep[8] = [0, 2, room[8]]
    ctx[9] = page - 3
    keep[9] = [0, 2, 3, 4, 9]
    table[9][1] = -1
    pool = torch.randn((n_pages, 2, kv, page, D), generator=torch.Generator().manual_seed(2)).to(BF)
    want, moved = pool.clone(), []
    for s in range(seqs):
        k = keep[s]
        bad = any(a >= b for a, b in zip(k, k[1:])) or any(j < 0 or ctx[s] + j >= cap for j in k)
        bad = bad or any(not 0 <= table[s][(ctx[s] + j) // page] < n_pages
                         for i, j0 in enumerate(k) for j in (i, j0))
        moved.append(-1 if bad else len(k))
        for i, j in enumerate(k if not bad else []):
            a, z = ctx[s] + j, ctx[s] + i
            want[table[s][z // page], :, :, z % page] = pool[table[s][a // page], :, :, a % page]
    cu = [0]
    for k in keep:
        cu.append(cu[-1] + len(k))
    gpu = pool.to(DEV)
    out = ints([9] * seqs)
    b = atp.kv_batch(torch.tensor(table, dtype=torch.int32, device=DEV), ints(ctx))
    flat = [j for k in keep for j in k]
    atp.atp_cache_compact(atp.kv_cache(gpu), b, ints(cu), ints(flat), out)
    assert out.tolist() == moved and moved.count(-1) == 5
    assert torch.equal(gpu.cpu().view(torch.int16), want.view(torch.int16))
    gpu = pool.to(DEV)                                  # without the counts: the same
    atp.atp_cache_compact(atp.kv_cache(gpu), b, ints(cu), ints(flat))
    assert torch.equal(gpu.cpu().view(torch.int16), want.view(torch.int16))
    gpu = pool.to(DEV)                                  # an empty list
    atp.atp_cache_compact(atp.kv_cache(gpu), b, ints([0] * (seqs + 1)), ints([]), out)
    assert out.tolist() == [0] * seqs and torch.equal(gpu.cpu(), pool)
