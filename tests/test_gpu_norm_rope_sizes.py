"""Norms of queries and keys with the position rotation at sizes where a worker takes
several heads of a token, several rounds of them, and several tokens, and at batches whose
sequences are found in several steps, against the 64-bit definitions."""
import random

import pytest
import torch

import cache_reference as C
import paper_2301_08658_amd as atp
from test_gpu_norm_rope import BF, D, DEV, block, check, gen, setup

pytestmark = pytest.mark.gpu

# tokens, kv, group, rot, interleaved: 3000 x 30 heads (8 workers a token, one round of four
# heads), 5000 x 30 and 5001 x 45 (4 workers, several rounds), 9000 x 12 (4 workers), 16500 x 6
# and 20001 x 5 (one worker, two rounds)
FORWARD = [(3000, 10, 1, 128, False), (5000, 10, 1, 64, True), (5001, 5, 7, 48, False),
           (9000, 4, 1, 128, True), (16500, 1, 4, 96, False), (20001, 1, 3, 128, False)]


@pytest.mark.parametrize("tokens,kv,group,rot,inter", FORWARD)
def test_forward(tokens, kv, group, rot, inter):
    gpu, ref = setup(rot, inter)
    pos = torch.randint(0, 10 ** 6, (tokens,), generator=gen(3), dtype=torch.int64)
    x = block(tokens, kv, group, 4, pad=8)
    out = torch.full_like(x, 7.0).contiguous()
    atp.atp_qk_norm_rope_fwd(1, tokens, kv, group, gpu, x, out,
                             positions=pos.to(torch.int32).to(DEV))
    want, bound = C.norm_rope(ref, C.heads(x, kv, group), group, pos)
    check(C.heads(out, kv, group), want, bound, "y")
    x2 = x.clone()
    atp.atp_qk_norm_rope_fwd(1, tokens, kv, group, gpu, x2, x2,
                             positions=pos.to(torch.int32).to(DEV))
    assert torch.equal(x2, out)


# 5001 x 9 heads: two tokens a worker, the last ones one; 6000 x 3 and 17000 x 3: two and four;
# 9000 x 12: three tokens, several heads of each
@pytest.mark.parametrize("tokens,kv,group,rot,inter", [
    (5001, 1, 7, 48, True), (6000, 1, 1, 128, False), (17000, 1, 1, 64, False),
    (9000, 4, 1, 128, False), (8191, 2, 2, 96, False)])
@pytest.mark.parametrize("far", [False, True])
def test_backward(tokens, kv, group, rot, inter, far):
    """A lane adds at most 64 terms one after the other (16384 workers, or those of as many
    whole tokens as fit), then 16, 64 and 64 partial sums; every term carries 64 roundings of
    its own."""
    gpu, ref = setup(rot, inter)
    seq = 1000 if tokens % 1000 == 0 else tokens
    pos, positions = torch.arange(tokens) % seq, None
    if far:
        pos = torch.randint(0, 10 ** 6, (tokens,), generator=gen(3), dtype=torch.int64)
        positions = pos.to(torch.int32).to(DEV)
    x, dy = block(tokens, kv, group, 4, pad=16), block(tokens, kv, group, 5, pad=8)
    dx = torch.full_like(x, 7.0).contiguous()
    dqw, dkw = torch.full((D,), 7.0, device=DEV), torch.full((D,), 7.0, device=DEV)
    ws = torch.empty(atp.atp_qk_norm_rope_workspace_bytes(tokens), dtype=torch.uint8, device=DEV)
    args = (tokens // seq, seq, kv, group, gpu, x)
    atp.atp_qk_norm_rope_bwd(*args, dy, dx, dqw, dkw, ws, positions)
    want, bound, dws = C.norm_rope_bwd(ref, C.heads(x, kv, group), C.heads(dy, kv, group), group,
                                       pos)
    check(C.heads(dx, kv, group), want, bound, "dx")
    n = 64 + 64 + 16 + 128
    for got, w, size in ((dqw, dws[0], dws[2]), (dkw, dws[1], dws[3])):
        check(got, w, (n * C.EPS32) * size, "dw")
    dy2, again = dy.clone(), torch.empty_like(dqw)
    atp.atp_qk_norm_rope_bwd(*args, dy2, dy2, again, None, ws, positions)
    assert torch.equal(dy2, dx) and torch.equal(again, dqw)


@pytest.mark.parametrize("seqs,most", [(17, 40), (257, 12), (700, 9), (2500, 4)])
@pytest.mark.parametrize("kv,group", [(1, 1), (4, 2)])
def test_append(seqs, most, kv, group):
    """Batches of many sequences, some without new tokens (runs of them, the first and the
    last too), padding rows: every row goes to its own sequence's place."""
    rng, page = random.Random(seqs), 16
    new = [rng.choice((0, 1, rng.randint(0, most))) for _ in range(seqs)]
    for lo in (0, seqs // 3, seqs - 3):
        new[lo:lo + 3] = [0, 0, 0]
    ctx = [rng.randint(0, 30) for _ in range(seqs)]
    cu = [0]
    for m in new:
        cu.append(cu[-1] + m)
    n, cols = cu[-1], -(-(30 + most) // page)
    t = n + 5
    order = torch.randperm(seqs * cols, generator=gen(5))
    table = order.reshape(seqs, cols).to(torch.int32)
    pool = torch.randn((seqs * cols, 2, kv, page, D), generator=gen(6)).to(BF).to(DEV)
    before = pool.cpu()
    gpu, ref = setup(128, False)
    x = block(t, kv, group, 7)
    q = torch.full((t, kv * group * D), 5.0, dtype=BF, device=DEV)
    i32 = dict(dtype=torch.int32, device=DEV)
    atp.atp_qk_norm_rope_cache(
        atp.kv_cache(pool), atp.kv_batch(table.to(DEV), torch.tensor(ctx, **i32),
                                         torch.tensor(cu, **i32)), t, group, gpu, x, q)
    owner = torch.tensor([s for s, m in enumerate(new) for _ in range(m)])
    at = torch.tensor([ctx[s] + j for s, m in enumerate(new) for j in range(m)])
    want, bound = C.norm_rope(ref, C.heads(x[:n], kv, group), group, at)
    check(q[:n].reshape(n, kv, group, D), want[:, :, :group], bound[:, :, :group], "q")
    assert (q[n:] == 5).all()
    page_of, after = table[owner, at // page].long(), pool.cpu()
    check(after[page_of, 0, :, at % page], want[:, :, group], bound[:, :, group], "k")
    check(after[page_of, 1, :, at % page], want[:, :, group + 1], 0 * bound[:, :, group], "v")
    after[page_of, :, :, at % page] = before[page_of, :, :, at % page]
    assert torch.equal(after, before)
