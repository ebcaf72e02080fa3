"""Norms of queries and keys with the position rotation on the GPU, forward,
backward and into a cache, against their 64-bit definitions."""
import math

import pytest
import torch

import cache_reference as C
import paper_2301_08658_amd as atp

pytestmark = pytest.mark.gpu
DEV, BF, D = "cuda:0", torch.bfloat16, 128


def gen(seed):
    return torch.Generator().manual_seed(seed)


def setup(rot=128, inter=False, norm=True, weights=True, eps=1e-6, theta=10000.0, seed=1):
    g = gen(seed)
    qw = (1 + 0.2 * torch.randn(D, generator=g)).to(BF).to(DEV) if norm and weights else None
    kw = (1 + 0.2 * torch.randn(D, generator=g)).to(BF).to(DEV) if norm and weights else None
    inv = None
    if rot:
        inv = (theta ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)).float().to(DEV)
    gpu = atp.qk_norm_rope(qw, kw, eps, inv, rot, inter, norm)
    return gpu, C.Rope(qw, kw, eps, inv, rot, inter, norm)


def block(t, kv, group, seed, pad=0, std=1.0):
    x = torch.randn((t, kv * (group + 2) * D + pad), generator=gen(seed)) * std
    return x.to(BF).to(DEV)[:, :kv * (group + 2) * D]


def check(got, want, bound, what):
    err = (C.f64(got) - want).abs()
    bad = err > bound
    assert not bad.any(), (what, int(bad.sum()), float((err - bound).max()))


CASES = [  # batch, seq, kv, group, rot, inter, norm, weights, positions up to
    (1, 1, 1, 1, 128, False, True, True, 0), (2, 9, 2, 1, 128, True, True, True, 0),
    (1, 33, 3, 4, 64, False, True, True, 0), (3, 7, 1, 7, 48, True, True, False, 5000),
    (1, 130, 2, 3, 8, False, True, True, 1 << 20), (1, 5, 1, 64, 120, False, True, True, 100),
    (2, 17, 1, 16, 0, False, True, True, 0), (1, 64, 5, 1, 128, False, False, False, 2 ** 31 - 1),
    (1, 20, 2, 2, 0, False, False, False, 0), (4, 300, 1, 1, 16, True, True, True, 0)]


@pytest.mark.parametrize("case", CASES)
def test_forward_and_backward(case):
    b, s, kv, group, rot, inter, norm, weights, far = case
    t = b * s
    gpu, ref = setup(rot, inter, norm, weights)
    pos = torch.arange(t) % s
    positions = None
    if far:
        pos = torch.randint(0, far, (t,), generator=gen(3), dtype=torch.int64)
        pos[0] = far - 1
        positions = pos.to(torch.int32).to(DEV)
    x, dy = block(t, kv, group, 4, pad=16), block(t, kv, group, 5, pad=8)
    out = torch.full_like(x, 7.0).contiguous()
    atp.atp_qk_norm_rope_fwd(b, s, kv, group, gpu, x, out, positions=positions)
    want, bound = C.norm_rope(ref, C.heads(x, kv, group), group, pos)
    check(C.heads(out, kv, group), want, bound, "y")
    # in place: the same bits, values untouched
    x2 = x.clone()
    atp.atp_qk_norm_rope_fwd(b, s, kv, group, gpu, x2, x2, positions=positions)
    assert torch.equal(x2, out)

    dx = torch.full_like(x, 7.0).contiguous()
    dqw = torch.full((D,), 7.0, device=DEV) if norm else None
    dkw = torch.full((D,), 7.0, device=DEV) if norm else None
    ws = torch.empty(atp.atp_qk_norm_rope_workspace_bytes(t), dtype=torch.uint8, device=DEV)
    atp.atp_qk_norm_rope_bwd(b, s, kv, group, gpu, x, dy, dx, dqw, dkw, ws, positions)
    want, bound, dws = C.norm_rope_bwd(ref, C.heads(x, kv, group), C.heads(dy, kv, group), group,
                                       pos)
    check(C.heads(dx, kv, group), want, bound, "dx")
    if norm:
        # a lane adds at most t * heads terms one after the other, then 16, 64 and 64
        # partial sums; every term carries 64 roundings of its own
        n = 64 + 16 + 128 + t * kv * group
        for got, w, size in ((dqw, dws[0], dws[2]), (dkw, dws[1], dws[3])):
            check(got, w, (n * C.EPS32) * size + 1e-30, "dw")
    # in place, without and with one of the weights' gradients: the same bits
    dy2 = dy.clone()
    atp.atp_qk_norm_rope_bwd(b, s, kv, group, gpu, x, dy2, dy2, positions=positions)
    assert torch.equal(dy2, dx)
    if norm:
        one = torch.empty_like(dkw)
        atp.atp_qk_norm_rope_bwd(b, s, kv, group, gpu, x, dy, dx, None, one, ws, positions)
        assert torch.equal(one, dkw)


def test_gradient_against_differences():
    """<d_qkv, dir> and the weights' gradients against central differences of the
    64-bit forward; the calls' outputs carry one bf16 rounding each (2^-8 of sum
    |dx dir|), the differences h^2-sized errors far below that."""
    kv, group, t = 2, 3, 11
    gpu, ref = setup(96, False)
    x, dy = block(t, kv, group, 8), block(t, kv, group, 9)
    dx = torch.empty_like(x)
    dqw, dkw = torch.empty(D, device=DEV), torch.empty(D, device=DEV)
    ws = torch.empty(atp.atp_qk_norm_rope_workspace_bytes(t), dtype=torch.uint8, device=DEV)
    atp.atp_qk_norm_rope_bwd(1, t, kv, group, gpu, x, dy, dx, dqw, dkw, ws)
    xd, g, pos = C.heads(x, kv, group), C.heads(dy, kv, group), torch.arange(t)
    direction = torch.randn(xd.shape, generator=gen(10), dtype=torch.float64)
    h = 1e-5

    def f(x_):
        return float((C.norm_rope(ref, x_, group, pos)[0] * g).sum())

    diff = (f(xd + h * direction) - f(xd - h * direction)) / (2 * h)
    got = C.heads(dx, kv, group)
    size = float((got * direction).abs().sum())
    assert abs(float((got * direction).sum()) - diff) <= (2 ** -8 + 1e-6) * size
    for w, dw in ((ref.qw, dqw), (ref.kw, dkw)):
        for i in (0, 1, 64, 127):
            old = float(w[i])
            w[i] = old + h
            up = f(xd)
            w[i] = old - h
            down = f(xd)
            w[i] = old
            assert abs(float(dw[i]) - (up - down) / (2 * h)) <= 1e-4 * (1 + abs(float(dw[i])))


def test_extreme_rows():
    """Zero rows (only eps under the root), huge and tiny values, infinities: what
    the formula gives in 32 bits, and neighbours untouched."""
    kv, group, t = 1, 2, 6
    gpu, ref = setup(128, False)
    x = block(t, kv, group, 11)
    x[1] = 0
    x[2] *= 1e15
    x[3] *= 1e-15
    x[4, :D] = math.inf
    x[5, D + 5] = math.nan
    out = torch.empty_like(x)
    atp.atp_qk_norm_rope_fwd(1, t, kv, group, gpu, x, out)
    want, bound = C.norm_rope(ref, C.heads(x, kv, group), group, torch.arange(t))
    got = C.heads(out, kv, group)
    for row in (0, 1, 2, 3):
        check(got[row], want[row], bound[row], f"row {row}")
    assert torch.isnan(got[4, 0, 0]).all() and torch.isnan(got[5, 0, 1]).all()
    check(got[4, 0, 1:], want[4, 0, 1:], bound[4, 0, 1:], "beside an infinite head")
    check(got[5, 0, 0], want[5, 0, 0], bound[5, 0, 0], "beside a NaN head")


def test_no_tokens():
    gpu, _ = setup()
    x = torch.empty((0, 3 * D), dtype=BF, device=DEV)
    dqw, dkw = torch.full((D,), 3.0, device=DEV), torch.full((D,), 3.0, device=DEV)
    atp.atp_qk_norm_rope_fwd(0, 4, 1, 1, gpu, x, torch.empty_like(x))
    atp.atp_qk_norm_rope_bwd(0, 4, 1, 1, gpu, x, x.clone(), torch.empty_like(x), dqw, dkw)
    assert float(dqw.abs().sum()) == 0 and float(dkw.abs().sum()) == 0


def test_runs_of_a_block_and_rows_between():
    """A column run of a wider block (one device's heads): the columns beside it keep
    their bits, and so do the padding columns of a wider row."""
    kv, group, t = 2, 1, 37
    gpu, ref = setup(128, False)
    wide = block(t, 4, 1, 12)
    out = torch.full((t, 5 * 3 * D), 3.0, dtype=BF, device=DEV)
    x, y = wide[:, 3 * D:9 * D], out[:, 6 * D:12 * D]
    atp.atp_qk_norm_rope_fwd(1, t, kv, group, gpu, x, y)
    want, bound = C.norm_rope(ref, C.heads(x, kv, group), group, torch.arange(t))
    check(C.heads(y, kv, group), want, bound, "run")
    assert (out[:, :6 * D] == 3).all() and (out[:, 12 * D:] == 3).all()


@pytest.mark.parametrize("page,kv,group", [(16, 2, 1), (64, 1, 5), (1024, 3, 2)])
@pytest.mark.parametrize("tree", [False, True])
def test_append(page, kv, group, tree):
    """Ragged sequences (some with no new tokens, padding rows behind the last,
    empty, invalid and missing pages): queries in their rows, keys and values in
    their places, everything else as it was."""
    new, ctx = [3, 0, 1, 40, 0, 2, 5], [0, 9, page - 1, 5, 3, 2 * page - 1, 4 * page - 2]
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    t = cu[-1] + 4
    cols = 4
    n_pages = 40
    order = torch.randperm(n_pages, generator=gen(5)).tolist()
    table = torch.tensor([[order[s * cols + i] for i in range(cols)] for s in range(len(new))],
                         dtype=torch.int32)
    table[5, 1] = -1                    # first new token of sequence 5 has no page
    table[3, 0] = n_pages               # invalid
    pool = torch.randn((n_pages, 2, kv, page, D), generator=gen(6)).to(BF).to(DEV)
    gpu, ref = setup(128, tree, theta=500000.0)
    x = block(t, kv, group, 7)
    pos = torch.tensor([ctx[s] + j for s, n in enumerate(new) for j in range(n)] + [0] * 4)
    positions = None
    if tree:
        pos = torch.randint(0, 10 ** 6, (t,), generator=gen(8))
        positions = pos.to(torch.int32).to(DEV)
    q = torch.full((t, kv * group * D), 5.0, dtype=BF, device=DEV)
    before = pool.clone()
    atp.atp_qk_norm_rope_cache(
        atp.kv_cache(pool), atp.kv_batch(table.to(DEV),
                                         torch.tensor(ctx, dtype=torch.int32, device=DEV),
                                         torch.tensor(cu, dtype=torch.int32, device=DEV)),
        t, group, gpu, x, q, positions=positions)
    want, bound = C.norm_rope(ref, C.heads(x, kv, group), group, pos)
    n = cu[-1]
    check(q[:n].reshape(n, kv, group, D), want[:n, :, :group], bound[:n, :, :group], "q")
    assert (q[n:] == 5).all()
    touched = torch.zeros(pool.shape[:4], dtype=torch.bool)
    for s, m in enumerate(new):
        for j in range(m):
            at, row = ctx[s] + j, cu[s] + j
            pg = int(table[s, at // page]) if at // page < cols else -1
            if not 0 <= pg < n_pages:
                continue
            check(pool[pg, 0, :, at % page], want[row, :, group], bound[row, :, group], "k")
            check(pool[pg, 1, :, at % page], want[row, :, group + 1], 0 * bound[row, :, group], "v")
            touched[pg, :, :, at % page] = True
    assert torch.equal(pool.cpu()[~touched], before.cpu()[~touched])


def test_lists_that_do_not_ascend_stay_inside():
    """cu_new and ctx values that the contract forbids: whatever the rows then are,
    nothing outside the pool and q is written."""
    i32 = dict(dtype=torch.int32, device=DEV)
    gpu, _ = setup()
    buf = torch.zeros((6, 2, 1, 16, D), dtype=BF, device=DEV)
    pool = buf[2:4]
    q = torch.zeros((12, D), dtype=BF, device=DEV)
    for cu, ctx in (([0, 100, 5, 8], [0, 0, 0]), ([7, 3, 9, 1], [5, -9, 2 ** 31 - 1]),
                    ([-4, 2, 2, 6], [31, 30, 0])):
        batch = atp.kv_batch(torch.tensor([[0, 1], [1, 0], [1, 9]], **i32),
                             torch.tensor(ctx, **i32), torch.tensor(cu, **i32))
        atp.atp_qk_norm_rope_cache(atp.kv_cache(pool), batch, 8, 1, gpu, block(8, 1, 1, 3), q[2:10])
    assert not buf[:2].any() and not buf[4:].any() and not q[:2].any() and not q[10:].any()


def test_same_bits_with_the_block_and_the_cache():
    """The cached form's queries and keys are the block form's, bit for bit."""
    kv, group, t = 2, 2, 70
    gpu, _ = setup(64, True)
    x = block(t, kv, group, 9)
    out = torch.empty_like(x)
    atp.atp_qk_norm_rope_fwd(1, t, kv, group, gpu, x, out)
    pool = torch.zeros((5, 2, kv, 16, D), dtype=BF, device=DEV)
    q = torch.empty((t, kv * group * D), dtype=BF, device=DEV)
    i32 = dict(dtype=torch.int32, device=DEV)
    atp.atp_qk_norm_rope_cache(
        atp.kv_cache(pool), atp.kv_batch(torch.tensor([[4, 2, 0, 1, 3]], **i32),
                                         torch.tensor([0], **i32), torch.tensor([0, t], **i32)),
        t, group, gpu, x, q)
    rows = out.view(t, kv, group + 2, D)
    assert torch.equal(q.view(t, kv, group, D), rows[:, :, :group])
    flat = pool[[4, 2, 0, 1, 3]].permute(1, 0, 3, 2, 4).reshape(2, 80, kv, D)[:, :t]
    assert torch.equal(flat[0], rows[:, :, group]) and torch.equal(flat[1], rows[:, :, group + 1])
