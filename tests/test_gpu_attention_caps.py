"""Caps of the scores of the attention within documents, from small to far above the scores,
against the 64-bit definition."""
import math

import pytest
import torch

import paper_2301_08658_amd as atp
import train_reference as R
from test_gpu_attention_docs import D, Run

pytestmark = pytest.mark.gpu

# Capped scores are off by 2^-22 of a cap of up to 64; larger caps' are off by 2^-18 of the
# score (what tanh is off by 12 u at most is 49 u of a tanh above 1/4).
SMALL_CAP, OF_CAP, OF_SCORE = 64.0, 2.0 ** -22, 2.0 ** -18


def _score(q, k, cap, slope, far):
    """train_reference._score with the bound of the capping as stated above."""
    raw = q @ k.T.contiguous() / math.sqrt(D)
    e = (D + 2) * R.U * (q.abs() @ k.abs().T.contiguous()) / math.sqrt(D)
    t = torch.tanh(raw / cap)
    x, dx = cap * t, 1 - t * t
    e = dx * e + (OF_CAP * cap if cap <= SMALL_CAP else OF_SCORE * x.abs())
    if slope:
        x = x - slope * far
    return x, dx, e + 3 * R.U * x.abs()


SHAPES = dict(
    split=dict(lens=[190, 70, 1], kv=1, group=2),
    split_slopes=dict(lens=[190, 70, 1], kv=1, group=2, slopes=True, prefix=[20, 70, 0]),
    whole=dict(lens=[700, 129, 1300, 3], kv=8, group=4),
    whole_slopes=dict(lens=[700, 129, 1300, 3], kv=8, group=4, slopes=True),
)


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("cap,std", [(64.0, 1.0), (65.0, 4.0), (100.0, 5.0), (1e4, 1.0),
                                     (1e6, 1.0), (1e6, 4.0), (2.0 ** 100, 1.0)])
def test_caps_of_any_size(monkeypatch, cap, std, shape):
    print(shape, cap, std, flush=True)
    monkeypatch.setattr(R, "_score", _score)
    r = Run(seed=11, cap=cap, std=std, **SHAPES[shape])
    # Numbers below 2^-126 may become 0 (exp2, the matrix instructions).  A weight that does
    # moves dS by at most 2^-126 |dO . V - delta|, |dO . V| and |delta| <= D m^2 each with m the
    # largest |input|, and it and a dS that does move each gradient by m times that; a sum takes
    # one of either from every query of its head group, and as many sums of its own may.
    m = max(float(r.qkv.abs().max()), float(r.d_out.abs().max()), 1.0)
    least = 2.0 ** -126 * r.t * r.group * m * (2 + 2 * D * m * m)
    check = R.check
    monkeypatch.setattr(R, "check", lambda got, want, bound, what:
                        check(got, want, bound + least, what))
    r.check()


def test_the_smallest_and_largest_caps():
    """A denormal cap scores nothing (all weights alike); one above 2^100 is refused."""
    r = Run([70], 1, 1, cap=1e-40)
    r.qkv[5, :D] = 0                                      # products of 0
    out, lse = r.forward()
    rows = torch.arange(1, 71, device=out.device).double()
    assert ((lse[0] - torch.log(rows)).abs() <= 3 * R.EXP + 80 * R.U).all()
    mean = R.f64(r.qkv[:, 2 * D:3 * D]).cumsum(0) / rows[:, None]
    size = R.f64(r.qkv[:, 2 * D:3 * D]).abs().cumsum(0) / rows[:, None]
    R.check(out[:70, :D], mean, 2 * R.H * (size + mean.abs()), "means")
    with pytest.raises(atp.AtpError, match="cap"):
        Run([70], 1, 1, cap=2.0 ** 101).forward()


@pytest.mark.parametrize("kv,n", [(2, 300), (16, 4096)])
@pytest.mark.parametrize("cap", [2.0, 50.0, 1000.0])
def test_seen_products_of_minus_infinity_score_minus_the_cap(kv, n, cap):
    """Under a cap alone a product of -inf is a score of -cap, in the first tiles of a row,
    among others and where a row sees nothing else; masked ones still weigh nothing."""
    run = Run([n], kv, 1, cap=cap)
    got = []
    for low in (-float("inf"), -1e30):
        qkv = run.qkv.clone()
        heads = qkv.view(n, kv, 3, D)
        heads[:, :, 0, 0] = heads[:, :, 0, 0].abs() + 0.5
        for at in (slice(0, 130), slice(135, 141), slice(190, 191)):
            heads[at, :, 1, 0] = low
        out, lse = run.forward(qkv)
        got.append((out[:n, :run.heads * D], lse))
    (out, lse), (out0, lse0) = got
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    assert torch.equal(out.view(torch.int16), out0.view(torch.int16))
    assert torch.equal(lse, lse0)
    # rows that see such scores alone: their values' mean
    rows = torch.arange(1, 131, device=out.device).double()
    want = torch.log(rows) - cap
    assert ((lse[:, :130] - want).abs() <= 6 * R.U * cap + 3 * R.EXP + 160 * R.U).all()
    v = R.f64(run.qkv[:130]).view(130, kv, 3, D)[:, :, 2]
    mean = v.cumsum(0) / rows[:, None, None]
    size = v.abs().cumsum(0) / rows[:, None, None]
    bound = size * (6 * R.U * cap + 2 * R.EXP + 2 * R.H + 160 * R.U) + R.H * mean.abs()
    R.check(out[:130].reshape(130, kv, D), mean, bound, "means")
