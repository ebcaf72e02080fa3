"""Which lists of gradients and destinations are refused because a result would land in another
gradient or result: looked at before any device work, so on tensors of the CPU here."""
import random

import pytest
import torch

import paper_2301_08658_amd as atp
from paper_2301_08658_amd import binding as B


@pytest.fixture(autouse=True)
def _any_device(monkeypatch):
    monkeypatch.setattr(B, "_on_device", lambda t, name: None)


def refused(src, dst=None):
    try:
        atp.grad_list(src, dst)
    except ValueError as e:
        assert "overlap" in str(e)
        return True
    return False


def test_results_inside_longer_gradients():
    x, other = torch.zeros(100), [torch.zeros(100), torch.zeros(10), torch.zeros(10)]
    y = torch.zeros(10)
    # the result of the third lies in the first, the second begins between them
    assert refused([x, x[10:20], y], [other[0], other[1], x[30:40]])
    assert refused([y, x[10:20], x], [x[30:40], other[1], other[0]])
    assert not refused([x, x[10:20], y], [other[0], other[1], other[2]])
    # a gradient listed twice, once in place: the second is read while it is written
    assert refused([x, x], [x, other[0]]) and refused([x, x], [other[0], x])
    assert refused([x, x]) and refused([y, x], [x[:10], x])
    assert not refused([x, x], [other[0], torch.zeros(100)])


def test_against_every_pair_of_values():
    rng = random.Random(7)
    store = torch.zeros(400)
    for _ in range(300):
        n = rng.randrange(1, 6)
        src, dst = [], []
        for _ in range(n):
            size = rng.choice((0, 1, 5, 20, 60))
            a, b = rng.randrange(0, 401 - size), rng.randrange(0, 401 - size)
            src.append(store[a:a + size])
            dst.append(src[-1] if rng.random() < 0.4 else store[b:b + size])

        def values(t):
            return set(range(t.storage_offset(), t.storage_offset() + t.numel()))
        meet = any(i != j and values(dst[i]) & (values(src[j]) | values(dst[j]))
                   for i in range(n) for j in range(n))
        assert refused(src, dst) == meet


def test_columns_of_one_matrix():
    m = torch.zeros(8, 128)
    assert not refused([m[:, :64], m[:, 64:]])            # in place, side by side
    assert not refused([m[:, :32], m[:, 40:72], m[:, 72:]])
    assert not refused([torch.zeros(8, 64), torch.zeros(8, 64)], [m[:, :64], m[:, 64:]])
    assert not refused([m[:, 64:], torch.zeros(8, 64)], [torch.zeros(8, 64), m[:, :64]])
    assert refused([m[:, :72], m[:, 64:]]) and refused([m[:, :64], m[:, 56:]])
    assert not refused([m[:4, :72], m[4:, 64:]])
    # a run between two rows, and one that reaches into the next
    flat = m.view(-1)
    assert not refused([m[:, :64], flat[64:128]]) and refused([m[:, :64], flat[64:129]])
    assert not refused([m[:, 64:], flat[:64]]) and refused([m[:, 64:], flat[60:200]])
    # rows of another length over the same memory
    w = flat.view(4, 256)
    assert not refused([m[:, :64], w[:, 64:128]]) and not refused([m[:, :64], w[:, 192:]])
    assert refused([m[:, :64], w[:, 64:136]]) and refused([m[:, :64], w[:, 100:200]])
    # types of other sizes
    half = m.view(torch.bfloat16)                         # rows of 256
    assert not refused([m[:, :64], half[:, 128:]]) and refused([m[:, :64], half[:, 120:]])


def test_rows_against_every_pair_of_values():
    rng = random.Random(8)
    store = torch.zeros(600)

    def view():
        if rng.random() < 0.3:
            n = rng.randrange(1, 40)
            return store[(a := rng.randrange(0, 601 - n)):a + n]
        ld = rng.choice((16, 16, 16, 24, 40))
        rows, cols = rng.randrange(1, 600 // ld), rng.randrange(1, ld)
        return store.as_strided((rows, cols), (ld, 1), rng.randrange(0, 600 - rows * ld))

    def values(t):
        if t.dim() == 1:
            return set(range(t.storage_offset(), t.storage_offset() + t.numel()))
        return {t.storage_offset() + r * t.stride(0) + c for r in range(t.size(0))
                for c in range(t.size(1))}
    seen = set()
    for _ in range(2000):
        a, b = view(), view()
        meet = bool(values(a) & values(b))
        assert refused([a, b]) == meet, (a.shape, a.stride(), b.shape, b.stride())
        seen.add(meet)
    assert seen == {True, False}
