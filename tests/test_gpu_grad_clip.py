"""Norm over many gradients and clipping on the GPU against their 64-bit definitions."""
import math

import pytest
import torch

import paper_2301_08658_amd as atp
import train_reference as R

pytestmark = pytest.mark.gpu
DEV, BF, F32 = "cuda:0", torch.bfloat16, torch.float32


def rand(shape, seed, dtype=F32, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(dtype).to(DEV)


def total_of(grads):
    ws = torch.full((atp.atp_grad_workspace_bytes(grads),), 0xff, dtype=torch.uint8, device=DEV)
    out = torch.full((3,), float("nan"), dtype=torch.float64, device=DEV)
    atp.atp_grad_sq_sum(grads, out[1:2], ws)
    assert torch.isnan(out[[0, 2]]).all()
    return out[1:2]


def check_clip(src, dst, before, scale, max_norm, extra=()):
    """before: the gradients as they were."""
    grads = atp.grad_list(src, dst)
    total = total_of(grads)
    want = sum(float((R.f64(s) ** 2).sum()) for s in before)
    assert abs(float(total) - want) <= 1e-12 * want
    parts = [torch.tensor([v], dtype=torch.float64, device=DEV) for v in extra]
    norm = torch.full((2,), float("nan"), device=DEV)
    atp.atp_grad_clip(grads, [total, *parts], norm, max_norm=max_norm, scale=scale)
    n, f = R.grad_factor(want + sum(extra), scale, max_norm)
    assert abs(float(norm[0]) - n) <= 2 * R.U * n
    assert abs(float(norm[1]) - f) <= 4 * R.U * f      # the scale as fp32, one rounding
    for s, d in zip(before, dst or src):
        ref = R.f64(s) * f
        e = 5 * R.U * ref.abs()
        # gradients below the type's normal range are rounded to its smallest steps
        R.check(d, ref, e + R.rounding(d.dtype) * (ref.abs() + e) + 2.0 ** -133, tuple(d.shape))


SIZES = [1, 2, 7, 8, 9, 63, 512, 2047, 16383, 16384, 16385, 40001]


@pytest.mark.parametrize("scale,max_norm", [(1.0, 1.0), (0.125, 1e9), (2.0, 3.0),
                                            (1.0, float("inf"))])
def test_types_and_sizes(scale, max_norm):
    src, dst = [], []
    for i, n in enumerate(SIZES * 2):
        st, dt = (F32, BF)[i % 2], (F32, BF)[(i // 2) % 2]
        src.append(rand((n,), i, st))
        dst.append(torch.full((n + 8,), float("nan"), dtype=dt, device=DEV))
    views = [d[:n] for d, n in zip(dst, SIZES * 2)]
    check_clip(src, views, src, scale, max_norm, extra=(3.5, 1e-3))
    for d in dst:
        assert torch.isnan(d[-8:]).all()


@pytest.mark.parametrize("max_norm", [0.5, 1e9])
def test_in_place_and_rows_with_gaps(max_norm):
    store = [rand((33, 136), 1), rand((7, 24), 2, BF), rand((1, 5), 3), rand((300, 4096), 4)]
    src = [store[0][:, :129], store[1][:, :17], store[2], store[3]]
    before = [s.clone() for s in store]
    old = [before[0][:, :129], before[1][:, :17], before[2], before[3]]
    check_clip(src, None, old, 1.0, max_norm)
    # what lies between the rows stays
    assert torch.equal(store[0][:, 129:], before[0][:, 129:])
    assert torch.equal(store[1][:, 17:], before[1][:, 17:])
    # rows with gaps to rows without and back
    a, b = rand((9, 64), 5), torch.full((9, 72), float("nan"), dtype=BF, device=DEV)
    check_clip([a], [b[:, :64]], [a], 1.0, 1.0)
    assert torch.isnan(b[:, 64:]).all()
    c = torch.empty((9, 64), device=DEV)
    check_clip([b[:, :64].contiguous()], [c], [b[:, :64]], 1.0, 1.0)


def test_hundreds_of_tensors():
    sizes = [1 + (i * 7919) % 3001 for i in range(700)]
    flat = torch.zeros((sum((n + 7) // 8 * 8 for n in sizes),), dtype=BF, device=DEV)
    src, dst, at = [], [], 0
    for i, n in enumerate(sizes):
        src.append(rand((n,), i, (F32, BF)[i % 2], 0.1))
        dst.append(flat[at:at + n])
        at += (n + 7) // 8 * 8
    check_clip(src, dst, src, 0.5, 1.0)


def test_squares_beyond_32_bits():
    """Squares of values near both ends of fp32 count."""
    big, small = torch.full((100,), 2.0 ** 120, device=DEV), torch.full((64,), 2.0 ** -120,
                                                                       device=DEV)
    assert float(total_of(atp.grad_list([big]))) == 100 * 2.0 ** 240
    assert float(total_of(atp.grad_list([small]))) == 64 * 2.0 ** -240
    norm = torch.empty(2, device=DEV)
    atp.atp_grad_clip(atp.grad_list([big]), [total_of(atp.grad_list([big]))], norm, max_norm=1.0)
    assert abs(float(norm[0]) / (10 * 2.0 ** 120) - 1) < 2 * R.U and \
        torch.allclose(big, torch.tensor(0.1, device=DEV), rtol=4 * R.U, atol=0)


def test_infinities_and_nan():
    for bad, want in ((float("inf"), (math.inf, 0.0)), (float("nan"), (math.nan, math.nan))):
        src = [rand((50,), 1), rand((20,), 2)]
        src[1][3] = bad
        dst = [torch.empty_like(s) for s in src]
        grads, norm = atp.grad_list(src, dst), torch.empty(2, device=DEV)
        atp.atp_grad_clip(grads, [total_of(grads)], norm, max_norm=1.0)
        got = norm.tolist()
        assert all(a == b or (math.isnan(a) and math.isnan(b)) for a, b in zip(got, want))
        assert torch.isnan(dst[1][3])
        assert torch.isnan(dst[0]).all() if math.isnan(bad) else (dst[0] == 0).all()


def test_nothing_and_zeros():
    none = atp.grad_list([])
    assert float(total_of(none)) == 0
    norm = torch.full((2,), 9.0, device=DEV)
    one = torch.full((1,), 4.0, dtype=torch.float64, device=DEV)
    atp.atp_grad_clip(none, [one], norm, max_norm=1.0)
    assert norm.tolist() == [2.0, 0.5]
    z = [torch.zeros((17,), device=DEV), torch.empty((0,), device=DEV)]
    grads = atp.grad_list(z)
    atp.atp_grad_clip(grads, [total_of(grads)], norm, max_norm=1.0)
    assert norm.tolist() == [0.0, 1.0] and (z[0] == 0).all()


def test_a_group_gets_the_same_bits_and_replicas_count_once():
    """Two devices' gradients, a third one held by both: each lists its own for the sum and
    all of them for the clipping."""
    a, b, both = rand((1000,), 1), rand((777,), 2, BF), rand((64,), 3)
    sums = [total_of(atp.grad_list([a, both])), total_of(atp.grad_list([b]))]
    norms, copies = [], []
    for mine in (a, b):
        dst = [torch.empty_like(mine), torch.empty_like(both)]
        norms.append(torch.empty(2, device=DEV))
        atp.atp_grad_clip(atp.grad_list([mine, both], dst), sums, norms[-1], max_norm=2.0)
        copies.append(dst[1])
    assert torch.equal(norms[0], norms[1]) and torch.equal(copies[0], copies[1])
    want = math.sqrt(sum(float((R.f64(t) ** 2).sum()) for t in (a, b, both)))
    assert abs(float(norms[0][0]) - want) <= 2 * R.U * want


def test_list_refuses_overlaps_and_shapes():
    x = rand((64,), 1)
    with pytest.raises(ValueError, match="overlap"):
        atp.grad_list([x[:32], x[32:]], [x[32:], rand((32,), 2)])
    with pytest.raises(ValueError, match="overlap"):
        atp.grad_list([rand((8,), 1), rand((8,), 2)], [x[:8], x[4:12]])
    with pytest.raises(ValueError, match="gaps"):
        atp.grad_list([rand((8, 8), 1).t()])
    with pytest.raises(ValueError, match="dst"):
        atp.grad_list([x], [x, x])
    with pytest.raises(ValueError, match="dst"):
        atp.grad_list([x], [x[:8]])
    with pytest.raises(TypeError):
        atp.grad_list([x.half()])
    atp.grad_list([x[:32], x[32:]])      # its own place
    with pytest.raises(atp.AtpError):     # 16-byte alignment
        atp.atp_grad_sq_sum(atp.grad_list([x[1:9]]), torch.empty(1, dtype=torch.float64,
                                                                 device=DEV),
                            torch.empty(64, dtype=torch.uint8, device=DEV))


@pytest.mark.parametrize("st,dt", [(F32, F32), (F32, BF), (BF, F32), (BF, BF)])
def test_more_than_the_caches_hold(st, dt):
    # above 128 MiB values go past the caches: runs, rows with gaps and ragged ends in one
    # list, apart and in place
    g = torch.Generator(device=DEV).manual_seed(9)
    shapes = [(7001, 5003), (1, 34000003), (3, 5)]
    wide = [torch.randn((r, c + 8 - c % 8), device=DEV, generator=g).to(st) for r, c in shapes]
    src = [w[:, :c] for w, (_, c) in zip(wide, shapes)]
    assert sum(s.numel() * s.element_size() for s in src) > 128 << 20
    dst = [torch.full((r, c + 16 - c % 8), float("nan"), dtype=dt, device=DEV) for r, c in shapes]
    views = [d[:, :c] for d, (_, c) in zip(dst, shapes)]
    check_clip(src, views, src, 0.5, 1.0, extra=(7.0,))
    for d, (_, c) in zip(dst, shapes):
        assert torch.isnan(d[:, c:]).all()
    if st == dt:
        gaps = [w[:, c:].clone() for w, (_, c) in zip(wide, shapes)]
        before = [s.clone() for s in src]
        check_clip(src, None, before, 0.5, 1.0)
        assert all(torch.equal(w[:, c:], k) for w, k, (_, c) in zip(wide, gaps, shapes))


@pytest.mark.parametrize("dtype", [F32, BF])
def test_columns_of_one_matrix_in_place(dtype):
    # a fused matrix' gradient, listed by its columns
    m = rand((37, 192), 21, dtype)
    before = m.clone()
    cut = [(0, 64), (64, 72), (72, 168)]
    check_clip([m[:, a:b] for a, b in cut], None, [before[:, a:b] for a, b in cut], 1.0, 2.0)
    assert torch.equal(m[:, 168:], before[:, 168:])


def test_more_values_than_one_launch_takes():
    # 2^36 values in place: 2^24 workgroups of 256 threads, more than HIP launches at once
    torch.cuda.empty_cache()
    n = (1 << 36) + 8
    if torch.cuda.mem_get_info()[0] < 2 * n + (8 << 30):
        pytest.skip("needs 136 GiB of device memory")
    g = torch.zeros(n, dtype=BF, device=DEV)
    at = torch.tensor([0, (1 << 30) - 1, 1 << 35, (1 << 36) - 1, 1 << 36, n - 1], device=DEV)
    g[at] = 3.0
    grads = atp.grad_list([g])
    total, norm = total_of(grads), torch.empty(2, device=DEV)
    assert float(total) == 54.0
    atp.atp_grad_clip(grads, [total], norm, max_norm=1.0)
    assert (g[at].cpu() == torch.tensor(3.0 / 54 ** 0.5).to(BF)).all()
    assert abs(float(norm[0]) - 54 ** 0.5) <= 2 * R.U * 54 ** 0.5
    del g, grads
    torch.cuda.empty_cache()
