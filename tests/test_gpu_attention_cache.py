"""Attention over the paged cache on the GPU against its 64-bit definition: single
tokens, chunks of prompts, drafted trees; ragged lengths, shared heads, small and
large pages, strides, padding, masked places that hold anything."""
import math
import random

import pytest
import torch

import cache_reference as C
import paper_2301_08658_amd as atp

pytestmark = pytest.mark.gpu
DEV, BF, D = "cuda:0", torch.bfloat16, 128


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV).reshape(-1)


class Case:
    def __init__(self, ctx, new, kv, group, page, seed=1, spare=3, padding=0, cols=None, pad=0,
                 q_std=1.0):
        g = torch.Generator().manual_seed(seed)
        self.ctx, self.new, self.kv, self.group, self.page = ctx, new, kv, group, page
        self.cu = [0]
        for n in new:
            self.cu.append(self.cu[-1] + n)
        self.tokens = self.cu[-1] + padding
        need = [-(-(c + n) // page) for c, n in zip(ctx, new)]
        cols = cols or max(1, max(need))
        self.n_pages = sum(need) + spare
        order = torch.randperm(self.n_pages, generator=g).to(torch.int32)
        self.table = torch.full((len(ctx), cols), -1, dtype=torch.int32)
        at = 0
        for s, n in enumerate(need):
            n = min(n, cols)
            self.table[s, :n] = order[at:at + n]
            at += n
        # places that no sequence holds have NaN in them
        self.pool = torch.full((self.n_pages, 2, kv, page, D), math.nan).to(BF)
        for s, (c, n) in enumerate(zip(ctx, new)):
            for i in range(0, c + n, page):
                if i // page >= cols:
                    break
                rows = min(page, c + n - i)
                self.pool[self.table[s, i // page], :, :, :rows] = \
                    torch.randn((2, kv, rows, D), generator=g).to(BF)
        self.q = (q_std * torch.randn((self.tokens, kv * group * D + pad), generator=g)).to(BF)
        self.pad = pad
        self.mask = None

    def tree(self, seed=2, words=None, empty=()):
        r = random.Random(seed)
        words = words or max(1, -(-max(self.new) // 64))
        rows = []
        for n in self.new:
            anc = []
            for j in range(n):
                p = r.randint(max(0, j - 5), j - 1) if j else -1
                anc.append((anc[p] if p >= 0 else 0) | (1 << j))
            rows += anc
        rows += [0] * (self.tokens - len(rows))
        for t in empty:
            rows[t] = 0
        m = [[(w >> (64 * k)) & (2 ** 64 - 1) for k in range(words)] for w in rows]
        self.mask = torch.tensor([[v - 2 ** 64 if v >> 63 else v for v in row] for row in m],
                                 dtype=torch.int64).reshape(self.tokens, words)
        return self

    def rows_of(self, max_new):
        n = self.group * max_new
        return 16 if n <= 16 else (32 if n <= 32 else 128)

    def run(self, max_new=None, with_lse=True, stream=None, ws=None):
        max_new = max_new or max(1, max(self.new))
        pool, q = self.pool.to(DEV), self.q.to(DEV)
        out = torch.full((self.tokens, self.kv * self.group * D + self.pad), 9.0, dtype=BF,
                         device=DEV)
        lse = torch.full((self.kv * self.group, self.tokens), 9.0, device=DEV)
        ws = ws if ws is not None else torch.full(
            (atp.atp_attention_cache_workspace_bytes(self.kv, self.group, max_new),), 255,
            dtype=torch.uint8, device=DEV)
        w = self.kv * self.group * D
        atp.atp_attention_cache_fwd(
            atp.kv_cache(pool), atp.kv_batch(self.table.to(DEV), ints(self.ctx), ints(self.cu)),
            self.tokens, self.group, max_new, q[:, :w], out[:, :w], lse if with_lse else None,
            self.mask.to(DEV) if self.mask is not None else None, ws, stream)
        torch.cuda.synchronize()
        assert (out[:, w:] == 9).all()
        return out[:, :w], lse

    def check(self, max_new=None, **kw):
        out, lse = self.run(max_new, **kw)
        m = max_new or max(1, max(self.new))
        w = self.kv * self.group * D
        want, wl, ob, lb = C.attention(self.pool, self.table, self.ctx, self.cu, self.q[:, :w],
                                       self.kv, self.group, self.page, self.mask, self.tokens,
                                       wide=self.rows_of(m) == 128)
        n = self.cu[-1]
        assert (out[n:] == 9).all() and (lse[:, n:] == 9).all()       # padding rows
        got, gl = C.f64(out[:n]), C.f64(lse[:, :n])
        want, wl, ob, lb = want[:n], wl[:, :n], ob[:n], lb[:, :n]
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        fine = torch.isfinite(want)
        assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)])
        err = (got - want).abs()[fine]
        assert (err <= ob[fine]).all(), float((err - ob[fine]).max())
        none = wl == -math.inf
        assert (gl[none] == -math.inf).all()
        ok = torch.isfinite(wl)
        assert ((gl - wl).abs()[ok] <= lb[ok]).all(), float(((gl - wl).abs() - lb)[ok].max())
        return out, lse


@pytest.mark.parametrize("ctx", [0, 1, 15, 16, 31, 32, 63, 64, 65, 127, 128, 129, 1000])
@pytest.mark.parametrize("page", [16, 64])
def test_one_token(ctx, page):
    Case([ctx], [1], 2, 1, page).check()


@pytest.mark.parametrize("group", [1, 2, 3, 5, 8, 16, 17, 33, 64])
def test_shared_heads(group):
    Case([70, 0, 300], [1, 2, 1], 2, group, 32).check()


@pytest.mark.parametrize("page", [16, 32, 64, 128, 1024])
@pytest.mark.parametrize("new", [[1, 1, 1], [2, 0, 5], [16, 1, 7], [33, 0, 1], [130, 64, 3]])
def test_ragged_causal(page, new):
    Case([200, 5, 0], new, 2, 1, page, padding=3).check()


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("new,group", [([1, 3, 8], 1), ([7, 0, 16], 2), ([31, 12, 64], 1),
                                       ([40, 64, 1], 5), ([65, 128, 70], 1)])
def test_trees(page, new, group):
    Case([130, 63, 0], new, 2, group, page, padding=2).tree().check()


def test_rows_that_see_nothing():
    """No context and an empty mask: zeros and -inf; beside rows that see something."""
    for new, group in (([3, 2], 1), ([10, 3], 2), ([40, 2], 1)):
        c = Case([0, 50], new, 2, group, 16).tree(empty=(0, 1, new[0]))
        out, lse = c.check()
        assert (out[:2] == 0).all() and (lse[:, :2] == -math.inf).all()
        assert (lse[:, new[0]] > -math.inf).all()      # its context is seen


def test_tokens_beyond_the_mask_words():
    c = Case([20], [70], 1, 1, 16).tree(words=1)
    c.check()


@pytest.mark.parametrize("new,group", [([6], 1), ([6], 5), ([40], 1)])
def test_masked_places_may_hold_anything(new, group):
    """NaN and infinities in drafts that other rows do not see reach only the rows
    that do, in keys and in values."""
    c = Case([37], new, 2, group, 16).tree()
    at = 37 + 3                                      # draft 3: seen by itself and its children
    page, slot = int(c.table[0, at // 16]), at % 16
    c.pool[page, 1, 0, slot, 5] = math.nan
    c.pool[page, 1, 0, slot, 77] = math.inf
    c.pool[page, 1, 1, slot, 3] = -math.inf
    out, _ = c.check()
    sees = torch.tensor([bool(int(w) >> 3 & 1) for w in c.mask[:, 0]], device=DEV)
    assert torch.isnan(out[sees, 5]).all() and torch.isfinite(out[~sees].float()).all()
    d = Case([37], new, 2, group, 16).tree()
    d.pool[page, 0, :, slot] = math.nan
    out, _ = d.run()
    assert torch.isnan(out[sees].float()).all() and torch.isfinite(out[~sees].float()).all()


def test_causal_rows_do_not_see_later_infinities():
    for new in ([3], [20], [100]):
        c = Case([5], new, 1, 1, 16)
        at = 5 + new[0] - 1
        c.pool[int(c.table[0, at // 16]), :, 0, at % 16] = math.inf
        out, _ = c.run()
        assert torch.isfinite(out[:-1].float()).all() and torch.isnan(out[-1].float()).all()


@pytest.mark.parametrize("page,new", [(16, 1), (16, 40), (64, 2), (64, 50)])
def test_missing_and_invalid_pages(page, new):
    c = Case([5 * page + 3, 2 * page], [new, 1], 2, 1, page)
    c.table[0, 1] = -1
    c.table[0, 3] = c.n_pages
    c.table[0, 4] = 2 ** 31 - 1
    c.table[1, :] = -5                               # nothing at all
    out, lse = c.check()
    assert (out[new] == 0).all() and (lse[:, new] == -math.inf).all()


def test_context_beyond_the_table():
    Case([100, 10], [4, 3], 1, 2, 16, cols=3).check()


@pytest.mark.parametrize("max_new", [1, 2, 3, 200])
def test_the_hint_does_not_change_what_is_computed(max_new):
    Case([90, 0, 33], [9, 1, 70], 2, 2, 32, padding=1).check(max_new)
    Case([90, 0, 33], [9, 1, 70], 2, 2, 32).tree().check(max_new)


def test_wide_rows_and_large_scores():
    """Rows wider than their heads; scores of +-100, where one key takes it all."""
    Case([300, 7], [2, 30], 3, 4, 64, pad=24, q_std=10.0).check()
    Case([300, 7], [1, 3], 1, 1, 16, pad=8, q_std=30.0).check()


def test_long_context_is_split_and_joined():
    """A unit cut over all workgroups, with one and with several rows, small and
    large pages; the lengths of a batch far apart."""
    Case([33000], [1], 1, 1, 64, seed=3).check()
    Case([17000], [2], 2, 3, 16, seed=4).check()
    Case([9000], [40], 1, 1, 128, seed=5).check()
    Case([20000, 3, 0, 700], [1, 1, 1, 1], 2, 2, 32, seed=6).check()


def test_many_sequences():
    r = random.Random(1)
    n = 700
    Case([r.randint(0, 60) for _ in range(n)], [r.choice((0, 1, 1, 2)) for _ in range(n)], 1, 1, 16,
         seed=7).check()


def test_offsets_beyond_32_bits():
    """A pool of more than 2^31 elements (8 GiB), pages used at both of its ends."""
    kv, page, n_pages = 4, 64, 66000
    pool = torch.empty((n_pages, 2, kv, page, D), dtype=BF, device=DEV)
    assert pool.numel() > 2 ** 32
    c = Case([150, 100], [1, 2], kv, 1, page, seed=8)
    table = c.table.clone()
    for s in range(2):
        for i in range(table.shape[1]):
            if table[s, i] >= 0:
                new = n_pages - 1 - 7 * (3 * s + i) if i % 2 == 0 else int(table[s, i])
                pool[new] = c.pool[int(table[s, i])].to(DEV)
                table[s, i] = new
    out = torch.empty((3, kv * D), dtype=BF, device=DEV)
    ws = torch.empty(atp.atp_attention_cache_workspace_bytes(kv, 1, 2), dtype=torch.uint8,
                     device=DEV)
    atp.atp_attention_cache_fwd(atp.kv_cache(pool),
                                atp.kv_batch(table.to(DEV), ints(c.ctx), ints(c.cu)), 3, 1, 2,
                                c.q.to(DEV), out, workspace=ws)
    want, _ = c.run()
    assert torch.equal(out, want)


def test_repeats_and_streams():
    """The same bits again, without the log-sum-exps, on another stream, and with a
    workspace that another batch used before."""
    c = Case([5000, 64, 900], [1, 4, 20], 2, 2, 32, seed=9)
    out, lse = c.run()
    for _ in range(3):
        again, l2 = c.run()
        assert torch.equal(out, again) and torch.equal(lse, l2)
    s = torch.cuda.Stream()
    ws = torch.empty(atp.atp_attention_cache_workspace_bytes(2, 2, 20), dtype=torch.uint8,
                     device=DEV)
    Case([0, 1, 2], [20, 1, 1], 2, 2, 16, seed=10).run(20, ws=ws)
    torch.cuda.synchronize()
    again, l2 = c.run(stream=s, ws=ws)
    assert torch.equal(out, again) and torch.equal(lse, l2)
    again, l2 = c.run(with_lse=False)
    assert torch.equal(out, again) and (l2 == 9).all()


def test_lists_that_do_not_ascend_stay_inside():
    """cu_new and ctx values that the contract forbids: whatever the rows then are,
    only rows of the step are written."""
    pool = torch.randn((4, 2, 1, 16, D), generator=torch.Generator().manual_seed(1)).to(BF).to(DEV)
    q = torch.randn((40, D), generator=torch.Generator().manual_seed(2)).to(BF).to(DEV)
    out = torch.full((60, D), 9.0, dtype=BF, device=DEV)
    for cu, ctx in (([0, 100, 5, 8], [0, 0, 0]), ([7, 3, 9, 1], [5, -9, 2 ** 31 - 1]),
                    ([-4, 2, 2, 6], [31, 30, 0])):
        for max_new in (1, 20, 40):
            ws = torch.empty(atp.atp_attention_cache_workspace_bytes(1, 1, max_new),
                             dtype=torch.uint8, device=DEV)
            batch = atp.kv_batch(torch.tensor([[0, 1], [1, 0], [1, 9]], dtype=torch.int32,
                                              device=DEV), ints(ctx), ints(cu))
            atp.atp_attention_cache_fwd(atp.kv_cache(pool), batch, 40, 1, max_new, q, out[10:50],
                                        workspace=ws)
    assert (out[:10] == 9).all() and (out[50:] == 9).all()
