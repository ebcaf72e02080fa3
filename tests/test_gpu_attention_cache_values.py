"""Attention over the paged cache where the values leave the ordinary range: infinities and
NaN that every row of a tile sees, and finite values near the end of the range."""
import math

import pytest
import torch

from test_gpu_attention_cache import BF, Case

pytestmark = pytest.mark.gpu


def put(case, seq, key, which, head, column, value):
    case.pool[int(case.table[seq, key // case.page]), which, head, key % case.page, column] = value


# rows of a unit: one token; 16; 17 to 32; more than 32
UNITS = [([1], 1), ([1], 16), ([4], 2), ([20], 1), ([9], 3), ([1], 33), ([40], 1), ([7], 8)]


@pytest.mark.parametrize("new,group", UNITS)
@pytest.mark.parametrize("page", [16, 64])
def test_infinities_that_every_row_sees(new, group, page):
    """Where every key of a tile is seen by every row, far behind the drafts' masks: an
    infinity comes out as it is, two of opposite signs in one column and a NaN as NaN, and
    the other columns and heads keep their values."""
    c = Case([200], new, 2, group, page, seed=21)
    put(c, 0, 5, 1, 0, 9, math.inf)
    put(c, 0, 130, 1, 0, 20, -math.inf)
    put(c, 0, 63, 1, 1, 127, math.inf)
    put(c, 0, 64, 1, 1, 0, math.nan)
    put(c, 0, 3, 1, 1, 50, math.inf)
    put(c, 0, 199, 1, 1, 50, -math.inf)
    out, _ = c.check()
    rows = out.view(new[0], 2, group, 128).float()
    assert (rows[:, 0, :, 9] == math.inf).all() and (rows[:, 0, :, 20] == -math.inf).all()
    assert (rows[:, 1, :, 127] == math.inf).all() and torch.isnan(rows[:, 1, :, [0, 50]]).all()
    assert int(torch.isfinite(rows).sum()) == new[0] * group * (2 * 128 - 5)


@pytest.mark.parametrize("new,group", UNITS)
def test_an_infinity_with_all_the_weight(new, group):
    """One key takes (nearly) all the weight, which is then 1 to the last bit."""
    c = Case([200], new, 1, group, 32, seed=22)
    c.q[:, :] = 1.0
    page, slot = int(c.table[0, 0]), 5
    c.pool[page, 0, 0, slot] = 4.0                   # score 4 sqrt(128) = 45
    c.pool[page, 1, 0, slot, 3] = -math.inf
    out, _ = c.check()
    assert (out.view(-1, 128)[:, 3] == -math.inf).all()


@pytest.mark.parametrize("new,group", UNITS)
def test_infinities_in_a_context_that_is_split(new, group):
    """The unit is cut over many workgroups: an infinity in one piece, in two, a NaN."""
    c = Case([9000], new, 1, group, 64, seed=23)
    put(c, 0, 700, 1, 0, 4, math.inf)
    put(c, 0, 8100, 1, 0, 4, math.inf)
    put(c, 0, 4500, 1, 0, 5, -math.inf)
    put(c, 0, 1300, 1, 0, 6, math.inf)
    put(c, 0, 6100, 1, 0, 6, -math.inf)
    put(c, 0, 0, 1, 0, 7, math.nan)
    c.check()


def test_infinities_beside_drafts_that_do_not_see_them():
    """In one sequence: infinities in the context, seen by all, and among the drafts, seen
    by some, in the same column and in others."""
    for new, group in (([6], 1), ([6], 5), ([40], 1)):
        c = Case([150], new, 1, group, 16, seed=24).tree()
        put(c, 0, 7, 1, 0, 1, math.inf)
        put(c, 0, 153, 1, 0, 1, math.inf)
        put(c, 0, 153, 1, 0, 2, -math.inf)
        put(c, 0, 152, 1, 0, 3, math.nan)
        c.check()


@pytest.mark.parametrize("new,group", UNITS)
def test_values_near_the_end_of_the_range(new, group):
    """Finite values whose sum with weights of at most 1 fits give finite results, also
    where single keys behind the first 128 have scores of 6.9 above all others, 987 times
    their weight: the twelve of them sum values of 1e35 to 1.2e36, and to 1.2e39 if the
    first keys' weights were 1.  Units of few rows are cut every 128 keys unless there are
    many of them."""
    seqs = 600 if new[0] * group <= 32 else 1
    c = Case([290] * seqs, new * seqs, 1, group, 32, seed=25)
    c.q[:, :] = 1.0
    k, v = c.pool[:, 0], c.pool[:, 1]
    c.pool[:, 0] = torch.where(torch.isnan(k), k, torch.zeros_like(k))
    for key in range(128, 290):
        if key % 64 in (0, 4, 8, 12):
            c.pool[c.table[:, key // 32].long(), 0, 0, key % 32] = 39 / 64      # x sqrt(128)
    c.pool[:, 1] = torch.where(torch.isnan(v), v, ((1 + v.float() / 16) * 1e35).to(BF))
    out, _ = c.check()
    assert torch.isfinite(out.float()).all()
