"""Layer norms with the residual sum on the GPU, whole rows and rows on several
devices, against their 64-bit definitions."""
import pytest
import torch

import paper_2301_08658_amd as atp
import train_reference as R

pytestmark = pytest.mark.gpu
DEV, BF, F32 = "cuda:0", torch.bfloat16, torch.float32
EPS = 1e-5


def rand(shape, seed, std=1.0, mean=0.0, dtype=BF, pad=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((*shape[:-1], shape[-1] + pad), generator=g) * std + mean
    return x.to(dtype).to(DEV)[..., :shape[-1]]


def params(cols, seed, weight=True, bias=True):
    w = rand((cols,), seed, 0.3, 1.0) if weight else None
    b = rand((cols,), seed + 1, 0.5) if bias else None
    return w, b, atp.layer_norm(w, b, EPS)


def workspace(t, cols):
    return torch.full((atp.atp_layer_norm_workspace_bytes(t, cols),), 0xff, dtype=torch.uint8,
                      device=DEV)


# rows, columns: one lane, ragged lanes, every shape of the row's holders
SIZES = [(1, 8), (1, 512), (3, 24), (5, 520), (130, 512), (7, 1024), (9, 1032), (6, 2048),
         (4, 2056), (33, 4096), (2, 5000), (3, 10240), (5, 10248), (3, 12288), (17, 20480),
         (2, 32760), (3, 32768), (1100, 64), (4099, 256), (2100, 4096)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("case", SIZES)
def test_forward_and_backward(case, dtype):
    t, c = case
    print(case, dtype, flush=True)
    add = (t + c) % 3 != 0
    w, b, norm = params(c, 1, weight=t % 4 != 2, bias=t % 5 != 0)
    x = rand((t, c), 3, 2.0, 1.0, dtype, pad=8)
    more = rand((t, c), 4, pad=16) if add else None
    full = lambda d, k: torch.full((t + 1, c + k), float("nan"), dtype=d, device=DEV)  # noqa: E731
    xo, y = full(dtype, 8), full(BF, 24)
    mean, rstd = torch.empty(t, device=DEV), torch.empty(t, device=DEV)
    atp.atp_layer_norm_fwd(t, norm, x, y[:t, :c], mean, rstd, add=more,
                           x_out=xo[:t, :c] if add else None)
    if add:
        want = (x.float() + more.float()).to(dtype)
        assert torch.equal(xo[:t, :c], want)
        assert torch.isnan(xo[t]).all() and torch.isnan(xo[:, c:]).all()
        x = xo[:t, :c]
    m, m2, e_m, e_m2 = R.norm_stats(x)
    R.check(mean, m, e_m, "mean")
    want, r, bound, e_r = R.norm(x, w, b, EPS, m, m2, e_m, e_m2, c)
    R.check(rstd, r, e_r, "rstd")
    R.check(y[:t, :c], want, bound, "y")
    assert torch.isnan(y[t]).all() and torch.isnan(y[:, c:]).all()

    dy, res = rand((t, c), 5, pad=8), rand((t, c), 6, dtype=dtype) if t % 2 else None
    dx = full(dtype, 8)
    d_add = full(BF, 0) if t % 3 else None
    dw, db = torch.full((c,), 9.0, device=DEV), torch.full((c,), 9.0, device=DEV)
    ws = workspace(t, c)
    atp.atp_layer_norm_bwd(t, norm, x, mean, rstd, dy, dx[:t, :c], d_res=res,
                           d_add=None if d_add is None else d_add[:t], dweight=dw, dbias=db,
                           workspace=ws)
    ref = R.norm_bwd(x, w, mean, rstd, dy, res)
    half = R.rounding(dtype)
    R.check(dx[:t, :c], ref["dx"], ref["e_dx"] + half * (ref["dx"].abs() + ref["e_dx"]), "dx")
    assert torch.isnan(dx[t]).all() and torch.isnan(dx[:, c:]).all()
    if d_add is not None:
        R.check(d_add[:t], ref["dx"], ref["e_dx"] + R.H * (ref["dx"].abs() + ref["e_dx"]), "d_add")
        assert torch.isnan(d_add[t]).all()
    R.check(dw, ref["dw"], ref["e_dw"], "dw")
    R.check(db, ref["db"], ref["e_db"], "db")
    # in place, one of the weights' gradients, no workspace for none; the same bits
    if res is not None:
        mine, dw2 = res.clone(), torch.empty_like(dw)
        atp.atp_layer_norm_bwd(t, norm, x, mean, rstd, dy, mine, d_res=mine, dweight=dw2,
                               workspace=ws)
        assert torch.equal(mine, dx[:t, :c]) and torch.equal(dw2, dw)
        mine.copy_(res)
        atp.atp_layer_norm_bwd(t, norm, x, mean, rstd, dy, mine, d_res=mine)
        assert torch.equal(mine, dx[:t, :c])


def test_sum_in_place():
    t, c = 37, 1032
    w, b, norm = params(c, 1)
    x, more = rand((t, c), 3), rand((t, c), 4)
    y1, y2 = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = torch.empty(t, device=DEV), torch.empty(t, device=DEV)
    xo = torch.empty_like(x)
    atp.atp_layer_norm_fwd(t, norm, x, y1, mean, rstd, add=more, x_out=xo)
    atp.atp_layer_norm_fwd(t, norm, x, y2, mean, rstd, add=more, x_out=x)
    assert torch.equal(x, xo) and torch.equal(y1, y2)


def test_values_far_from_zero_and_rows_of_one_value():
    """Centred squares: a mean 10^4 times the spread keeps the spread's digits; a constant row
    has none, and its norm is the bias."""
    t, c = 6, 4096
    norm = atp.layer_norm(None, None, EPS)
    x = (1000.0 + rand((t, c), 3, 0.1, dtype=F32)).contiguous()
    x[3] = -7.25
    y, mean, rstd = (torch.empty((t, c), dtype=BF, device=DEV), torch.empty(t, device=DEV),
                     torch.empty(t, device=DEV))
    atp.atp_layer_norm_fwd(t, norm, x, y, mean, rstd)
    m, m2, e_m, e_m2 = R.norm_stats(x)
    want, r, bound, e_r = R.norm(x, None, None, EPS, m, m2, e_m, e_m2, c)
    R.check(y, want, bound, "y")
    assert (y[3] == 0).all() and mean[3] == -7.25


def test_infinities_and_nan_stay_in_their_rows():
    t, c = 9, 2056
    w, b, norm = params(c, 1)
    x = rand((t, c), 3).contiguous()
    y, mean, rstd = torch.empty_like(x), torch.empty(t, device=DEV), torch.empty(t, device=DEV)
    atp.atp_layer_norm_fwd(t, norm, x, y, mean, rstd)
    bad, y2 = x.clone(), torch.empty_like(x)
    bad[2, 100], bad[5, 0] = float("inf"), float("nan")
    atp.atp_layer_norm_fwd(t, norm, bad, y2, mean, rstd)
    rest = [r for r in range(t) if r not in (2, 5)]
    assert torch.equal(y[rest], y2[rest]) and torch.isnan(y2[[2, 5]]).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("case", [(1, 8, 2), (5, 1024, 4), (33, 640, 8), (7, 5120, 4),
                                  (9, 10248, 2), (2, 64, 64)])
def test_rows_on_several_devices(case, dtype):
    t, c, n = case
    print(case, dtype, flush=True)
    total, me = n * c, n // 2
    x, more = rand((t, total), 3, 2.0, 1.0, dtype), rand((t, total), 4)
    w, b, whole = params(total, 1)
    outs, stats, xs, norms = [], [], [], []
    for j in range(n):
        cols = slice(j * c, (j + 1) * c)
        xs.append(torch.empty((t, c), dtype=dtype, device=DEV))
        stats.append(torch.full((t, 2), float("nan"), device=DEV))
        atp.atp_layer_norm_stats(t, x[:, cols], stats[j], add=more[:, cols], x_out=xs[j])
        m, m2, e_m, e_m2 = R.norm_stats(xs[j])
        R.check(stats[j][:, 0], m, e_m, "mean")
        R.check(stats[j][:, 1], m2, e_m2, "m2")
        norms.append(atp.layer_norm(w[cols].contiguous(), b[cols].contiguous(), EPS))
    joined = torch.cat(xs, 1)
    assert torch.equal(joined, (x.float() + more.float()).to(dtype))
    got = [torch.empty((t, c), dtype=BF, device=DEV) for _ in range(n)]
    mean = [torch.empty(t, device=DEV) for _ in range(n)]
    rstd = [torch.empty(t, device=DEV) for _ in range(n)]
    for j in range(n):
        atp.atp_layer_norm_fwd(t, norms[j], xs[j], got[j], mean[j], rstd[j], stats=stats)
        assert torch.equal(mean[j], mean[0]) and torch.equal(rstd[j], rstd[0])
    # statistics of shards: each shard's errors, and those of joining n of them
    m, m2, _, _ = R.norm_stats(joined)
    own = [R.norm_stats(s) for s in xs]
    e_m = torch.stack([o[2] for o in own]).mean(0) + \
        (n + 2) * R.U * torch.stack([o[0].abs() for o in own]).mean(0)
    dev = torch.stack([(o[0] - m).abs() for o in own])
    e_dev = torch.stack([o[2] + e_m for o in own]) + R.U * dev
    e_m2 = torch.stack([o[3] for o in own]).sum(0) + (2 * n + 4) * R.U * m2 + \
        c * (2 * dev * e_dev + e_dev ** 2).sum(0)
    want, r, bound, e_r = R.norm(joined, w, b, EPS, m, m2, e_m, e_m2, total)
    R.check(rstd[0], r, e_r, "rstd")
    R.check(torch.cat(got, 1), want, bound, "y")

    dy, res = rand((t, total), 5), rand((t, total), 6, dtype=dtype)
    sums = [torch.empty((t, 2), device=DEV) for _ in range(n)]
    for j in range(n):
        cols = slice(j * c, (j + 1) * c)
        atp.atp_layer_norm_bwd_sums(t, norms[j], xs[j], mean[j], rstd[j], dy[:, cols], sums[j])
        ref = R.norm_bwd(xs[j], w[cols], mean[j], rstd[j], dy[:, cols], None)
        R.check(sums[j], ref["own"], ref["e_own"], "sums")
    dx = torch.empty((t, c), dtype=dtype, device=DEV)
    dw, db = torch.empty(c, device=DEV), torch.empty(c, device=DEV)
    cols = slice(me * c, (me + 1) * c)
    atp.atp_layer_norm_bwd(t, norms[me], xs[me], mean[me], rstd[me], dy[:, cols], dx,
                           d_res=res[:, cols], sums=sums, dweight=dw, dbias=db,
                           workspace=workspace(t, c))
    ref = R.norm_bwd(xs[me], w[cols], mean[me], rstd[me], dy[:, cols], res[:, cols],
                     [s for j, s in enumerate(sums) if j != me], total)
    half = R.rounding(dtype)
    R.check(dx, ref["dx"], ref["e_dx"] + half * (ref["dx"].abs() + ref["e_dx"]), "dx")
    R.check(dw, ref["dw"], ref["e_dw"], "dw")
    R.check(db, ref["db"], ref["e_db"], "db")


def test_gradient_against_differences():
    """Central differences of sum(y dy) in 64 bits: the reference itself is the gradient of
    the reference forward."""
    t, c, h = 2, 16, 1e-6
    x, dy = R.f64(rand((t, c), 1, dtype=F32)), R.f64(rand((t, c), 2))
    w, b = rand((c,), 3), rand((c,), 4)

    def value(x_):
        mean = x_.mean(1)
        m2 = ((x_ - mean[:, None]) ** 2).sum(1)
        zero = torch.zeros_like(mean)
        return (R.norm(x_, w, b, EPS, mean, m2, zero, zero, c)[0] * dy).sum()
    mean = x.mean(1)
    rstd = (((x - mean[:, None]) ** 2).mean(1) + EPS) ** -0.5
    dx = R.norm_bwd(x, w, mean, rstd, dy, None)["dx"]
    for i in range(t):
        for j in range(0, c, 5):
            e = torch.zeros_like(x)
            e[i, j] = h
            assert abs((value(x + e) - value(x - e)) / (2 * h) - dx[i, j]) < 1e-6


def test_no_rows():
    c = 64
    norm = atp.layer_norm(None, None, EPS)
    none, empty = torch.empty((0, c), dtype=BF, device=DEV), torch.empty(0, device=DEV)
    atp.atp_layer_norm_fwd(0, norm, none, none, empty, empty)
    dw, db = torch.full((c,), 9.0, device=DEV), torch.full((c,), 9.0, device=DEV)
    atp.atp_layer_norm_bwd(0, norm, none, empty, empty, none, none, dweight=dw, dbias=db)
    assert (dw == 0).all() and (db == 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, BF])
@pytest.mark.parametrize("c", [24, 520, 1000, 2056, 5120, 12288, 20480])
def test_rows_of_one_value_give_the_bias(c, dtype):
    # their sums are exact (multiples of 8 below 2^27), so the mean is the value itself and
    # nothing is left of it, whatever 1 / sqrt(eps) would make of a rounding
    t, values = 3, torch.tensor([1000.0, -24.0, 1656.0])
    x = values.to(dtype).to(DEV)[:, None].expand(t, c).contiguous()
    b = (torch.arange(c) % 7 - 3).to(BF).to(DEV)
    y, mean, rstd = torch.empty((t, c), dtype=BF, device=DEV), *(
        torch.empty(t, device=DEV) for _ in range(2))
    for bias in (None, b):
        atp.atp_layer_norm_fwd(t, atp.layer_norm(None, bias), x, y, mean, rstd)
        assert torch.equal(mean.cpu(), values)
        assert torch.equal(y, torch.zeros_like(y) if bias is None else b.expand(t, c))
    stats = torch.empty((t, 2), device=DEV)
    atp.atp_layer_norm_stats(t, x, stats)
    assert torch.equal(stats[:, 0].cpu(), values) and (stats[:, 1] == 0).all()
