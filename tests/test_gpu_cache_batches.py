"""Attention over the paged cache and its page calls for batches of very many, mostly idle
sequences, and with tables, contexts and positions at their limits."""
import random

import pytest
import torch

import cache_reference as C
import paper_2301_08658_amd as atp
from test_gpu_attention_cache import BF, D, DEV, Case, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("seqs,active", [(3000, 40), (65536, 60), (65536, 1)])
@pytest.mark.parametrize("most", [1, 40])
def test_mostly_idle_sequences(seqs, active, most):
    """Long runs of sequences without new tokens before, between and behind the others."""
    rng = random.Random(active)
    ctx, new = [0] * seqs, [0] * seqs
    for s in rng.sample(range(10, seqs - 10), active):
        ctx[s], new[s] = rng.choice((0, 17, 400)), rng.choice((1, 1, most))
    c = Case(ctx, new, 1, 2, 16, seed=41, padding=2)
    c.check(max_new=most)


def test_as_many_sequences_as_there_may_be():
    """65536 sequences with a token each: pages, attention of single keys (the value itself)."""
    seqs, page = 65536, 16
    table = torch.full((seqs, 1), -1, dtype=torch.int32, device=DEV)
    refs = torch.zeros(seqs + 7, dtype=torch.int32, device=DEV)
    batch = atp.kv_batch(table, torch.zeros(seqs, dtype=torch.int32, device=DEV),
                         torch.arange(seqs + 1, dtype=torch.int32, device=DEV))
    lists = [torch.empty(seqs, dtype=torch.int32, device=DEV) for _ in range(4)]
    ws = torch.empty(atp.atp_cache_workspace_bytes(seqs + 7, seqs), dtype=torch.uint8, device=DEV)
    atp.atp_cache_reserve(page, refs, batch, *lists, ws)
    assert not lists[0].any() and torch.equal(table[:, 0].cpu(), torch.arange(seqs).int())
    pool = torch.zeros((seqs + 7, 2, 1, page, D), dtype=BF, device=DEV)
    x = torch.randn((seqs, 3 * D), generator=torch.Generator().manual_seed(1)).to(BF).to(DEV)
    q, out = torch.empty((seqs, D), dtype=BF, device=DEV), torch.empty((seqs, D), dtype=BF, device=DEV)
    cache = atp.kv_cache(pool)
    atp.atp_qk_norm_rope_cache(cache, batch, seqs, 1, atp.qk_norm_rope(), x, q)
    aws = torch.empty(atp.atp_attention_cache_workspace_bytes(1, 1, 1), dtype=torch.uint8, device=DEV)
    atp.atp_attention_cache_fwd(cache, batch, seqs, 1, 1, q, out, workspace=aws)
    assert torch.equal(out, x[:, 2 * D:])
    atp.atp_cache_release(page, refs, batch, torch.zeros(seqs, dtype=torch.int32, device=DEV))
    assert not refs.any() and (table == -1).all()


def test_rows_of_a_wider_table():
    """A table whose rows lie apart, in the attention and in the append."""
    c = Case([90, 0, 33], [9, 1, 70], 2, 2, 32, seed=42)
    want, _ = c.run()
    cols = c.table.shape[1]
    wide = torch.full((3, cols + 9), c.n_pages - 1, dtype=torch.int32, device=DEV)[:, :cols]
    wide.copy_(c.table)
    batch = atp.kv_batch(wide, ints(c.ctx), ints(c.cu))
    ws = torch.empty(atp.atp_attention_cache_workspace_bytes(2, 2, 70), dtype=torch.uint8, device=DEV)
    out = torch.empty_like(want)
    atp.atp_attention_cache_fwd(atp.kv_cache(c.pool.to(DEV)), batch, c.tokens, 2, 70, c.q.to(DEV),
                                out, workspace=ws)
    assert torch.equal(out, want)
    x = torch.randn((c.tokens, 2 * 4 * D), generator=torch.Generator().manual_seed(2)).to(BF).to(DEV)
    got = []
    for table in (wide, c.table.to(DEV)):
        pool, q = torch.zeros_like(c.pool).to(DEV), torch.empty_like(out)
        atp.atp_qk_norm_rope_cache(atp.kv_cache(pool), atp.kv_batch(table, ints(c.ctx), ints(c.cu)),
                                   c.tokens, 2, atp.qk_norm_rope(), x, q)
        got.append((pool, q))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


def test_positions_below_zero():
    """A rotation by -p is the one by p with its angles turned round."""
    t = 33
    inv = (10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)).float().to(DEV)
    gpu, ref = atp.qk_norm_rope(inv_freq=inv, rotary_dims=D), C.Rope(None, None, 1e-6, inv, D)
    pos = torch.randint(-10 ** 6, 1, (t,), generator=torch.Generator().manual_seed(3))
    pos[0] = -2 ** 31
    x = torch.randn((t, 3 * D), generator=torch.Generator().manual_seed(4)).to(BF).to(DEV)
    out = torch.empty_like(x)
    atp.atp_qk_norm_rope_fwd(1, t, 1, 1, gpu, x, out, positions=ints(pos.tolist()))
    want, bound = C.norm_rope(ref, C.heads(x, 1, 1), 1, pos)
    assert ((C.heads(out, 1, 1) - want).abs() <= bound).all()


def test_more_forks_than_a_workgroup_has_threads():
    """As many forks as a call takes, of parents that share their pages many times over."""
    forks, cols = 4096, 3
    seqs = forks + 5
    table = torch.full((seqs, cols), -1, dtype=torch.int32, device=DEV)
    for p in range(5):
        table[p] = torch.tensor([3 * p, 3 * p + 1, 3 * p + 2], dtype=torch.int32)
    refs = torch.zeros(20, dtype=torch.int32, device=DEV)
    refs[:15] = 1
    ctx = torch.zeros(seqs, dtype=torch.int32, device=DEV)
    ctx[:5] = ints([48, 33, 32, 1, 0])
    parents = torch.arange(forks, device=DEV).remainder(5).int()
    children = torch.arange(5, seqs, device=DEV).int()
    done = torch.full((forks,), 9, dtype=torch.int32, device=DEV)
    atp.atp_cache_fork(16, refs, atp.kv_batch(table, ctx), parents, children, done)
    assert not done.any()
    held = [3, 3, 2, 1, 0]
    counts = [1 + sum(1 for f in range(forks) if f % 5 == p) * (i < held[p])
              for p in range(5) for i in range(3)]
    assert refs.tolist() == counts + [0] * 5
    want = torch.tensor([[3 * p + i if i < held[p] else -1 for i in range(3)] for p in range(5)])
    assert torch.equal(table[5:].cpu().long(), want[parents.cpu().long()])
