"""Attention within packed documents on the GPU, forward and backward, against its
64-bit definition."""
import math

import pytest
import torch

import paper_2301_08658_amd as atp
import train_reference as R

pytestmark = pytest.mark.gpu
DEV, BF, D = "cuda:0", torch.bfloat16, 128


def rand(shape, seed, std=1.0, pad=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((*shape[:-1], shape[-1] + pad), generator=g) * std
    return x.to(BF).to(DEV)[..., :shape[-1]]


def starts(lens, first=0):
    out = [first]
    for n in lens:
        out.append(out[-1] + n)
    return out


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def slopes_of(heads):
    return [2.0 ** (-8.0 * (h + 1) / heads) for h in range(heads)]


class Run:
    """One batch of documents, padded in front and behind, through both calls."""

    def __init__(self, lens, kv, group, cap=0.0, slopes=False, prefix=None, first=0, behind=0,
                 seed=1, std=1.0):
        self.cu = starts(lens, first)
        self.t, self.kv, self.group = self.cu[-1] + behind, kv, group
        self.heads = kv * group
        self.cap, self.prefix = cap, prefix
        # slopes as the kernels read them
        self.slopes = torch.tensor(slopes_of(self.heads)) if slopes else None
        self.docs = atp.attention_docs(
            ints(self.cu), prefix=None if prefix is None else ints(prefix),
            slopes=None if self.slopes is None else self.slopes.to(DEV), cap=cap)
        t = self.t
        self.qkv = rand((t, kv * (group + 2) * D), seed, std, pad=8)
        self.d_out = rand((t, self.heads * D), seed + 1, pad=16)
        self.rows = torch.zeros(t, dtype=torch.bool, device=DEV)
        self.rows[first:self.cu[-1]] = True

    def buffers(self):
        nan = float("nan")
        out = torch.full((self.t + 1, self.heads * D + 8), nan, dtype=BF, device=DEV)
        lse = torch.full((self.heads, self.t), nan, device=DEV)
        d_qkv = torch.full((self.t + 1, self.qkv.shape[1] + 8), nan, dtype=BF, device=DEV)
        return out, lse, d_qkv

    def forward(self, qkv=None, buf=None):
        out, lse, _ = buf or self.buffers()
        atp.atp_attention_docs_fwd(self.t, self.kv, self.group, self.docs,
                                   self.qkv if qkv is None else qkv, out[:self.t, :self.heads * D],
                                   lse)
        return out, lse

    def backward(self, out, lse, d_qkv, qkv=None, d_out=None, ws=None):
        if ws is None:
            n = atp.atp_attention_docs_workspace_bytes(self.t, self.kv, self.group)
            ws = torch.full((n,), 0xff, dtype=torch.uint8, device=DEV)
        atp.atp_attention_docs_bwd(self.t, self.kv, self.group, self.docs,
                                   self.qkv if qkv is None else qkv, out[:self.t, :self.heads * D],
                                   lse, self.d_out if d_out is None else d_out,
                                   d_qkv[:self.t, :self.qkv.shape[1]], ws)

    def reference(self, **kw):
        return R.attention(self.qkv, self.kv, self.group, self.cu, self.prefix,
                           None if self.slopes is None else self.slopes.tolist(), self.cap, **kw)

    def check(self):
        c, w, rows = self.heads * D, self.qkv.shape[1], self.rows
        out, lse, d_qkv = self.buffers()
        self.forward(buf=(out, lse, d_qkv))
        want, z, e_o, e_z = self.reference()
        R.check(out[:self.t, :c][rows], want[rows], e_o[rows], "out")
        R.check(lse[:, rows], z[:, rows], e_z[:, rows], "lse")
        self.backward(out, lse, d_qkv)
        grad, e_g = self.reference(out=out[:self.t, :c], lse=lse, d_out=self.d_out)
        R.check(d_qkv[:self.t, :w][rows], grad[rows], e_g[rows], "d_qkv")
        # padding rows, the columns and the row behind stay as they were
        for t, n in ((out, c), (d_qkv, w)):
            assert torch.isnan(t[:self.t][~rows]).all() and torch.isnan(t[self.t]).all()
            assert torch.isnan(t[:, n:]).all()
        assert torch.isnan(lse[:, ~rows]).all()
        # the same bits again
        again = self.buffers()
        self.forward(buf=again)
        self.backward(again[0], again[1], again[2])
        assert torch.equal(again[0].view(torch.int16), out.view(torch.int16))
        assert torch.equal(again[2].view(torch.int16), d_qkv.view(torch.int16))


CASES = dict(
    one_row=dict(lens=[1], kv=1, group=1),
    two_rows=dict(lens=[2], kv=1, group=2, slopes=True),
    tile=dict(lens=[64], kv=2, group=1),
    tile_and_one=dict(lens=[65], kv=1, group=1, cap=30.0),
    ragged=dict(lens=[127, 1, 0, 130, 63, 64, 65, 0], kv=2, group=1, first=3, behind=70),
    shared=dict(lens=[200, 33, 129], kv=1, group=5, first=1),
    shared_cap=dict(lens=[300, 7], kv=2, group=4, cap=5.0, behind=9),
    prefix=dict(lens=[150, 64, 1, 90], kv=1, group=2, prefix=[100, 64, 5, -3]),
    prefix_whole=dict(lens=[333], kv=1, group=1, prefix=[1000], slopes=True),
    slopes=dict(lens=[400, 50], kv=2, group=2, slopes=True),
    everything=dict(lens=[77, 260, 0, 128], kv=2, group=3, slopes=True, cap=20.0,
                    prefix=[10, 200, 3, 0], first=5, behind=3),
    tiny_documents=dict(lens=[1, 2, 3, 1, 1, 5, 0, 0, 2] * 30, kv=1, group=1),
    # enough tiles for the 128-row kernels, forward and backward
    wide=dict(lens=[700, 129, 1300, 3], kv=8, group=4),
    wide_all=dict(lens=[1000, 515, 650], kv=4, group=8, slopes=True, cap=50.0,
                  prefix=[300, 0, 650], behind=40),
    wide_cap=dict(lens=[2100], kv=16, group=2, cap=10.0),
    wide_slopes=dict(lens=[1025, 1025], kv=32, group=1, slopes=True),
    # heads divided over workgroups, or not
    many_heads=dict(lens=[130, 64], kv=1, group=64),
    odd_heads=dict(lens=[500], kv=3, group=7),
)


@pytest.mark.parametrize("name", CASES)
def test_against_the_definition(name):
    print(name, flush=True)
    Run(seed=len(name), **CASES[name]).check()


def test_large_scores():
    """Scores up to a few hundred: one key takes nearly all the weight."""
    Run([190, 70], 1, 2, std=4.0, seed=3).check()
    Run([190, 70], 1, 2, std=4.0, seed=3, cap=50.0).check()


def test_thousands_of_documents():
    lens = [(i * 37) % 9 for i in range(5000)]
    Run(lens, 1, 1, seed=5).check()


def test_documents_are_alone():
    """What other documents and padding rows hold does not reach a document: its bits are
    those of a call with that document alone."""
    lens = [70, 200, 129]
    r = Run(lens, 2, 2, first=10, behind=20, cap=30.0, slopes=True, prefix=[5, 100, 0])
    w, c = r.qkv.shape[1], r.heads * D
    for spoiled in (float("nan"), float("inf")):
        for d, n in enumerate(lens):
            rows = slice(r.cu[d], r.cu[d + 1])
            qkv, d_out = torch.full_like(r.qkv, spoiled), torch.full_like(r.d_out, spoiled)
            qkv[rows], d_out[rows] = r.qkv[rows], r.d_out[rows]
            out, lse, d_qkv = r.buffers()
            r.forward(qkv, (out, lse, d_qkv))
            r.backward(out, lse, d_qkv, qkv, d_out)
            want, _, e_o, _ = r.reference()
            R.check(out[rows, :c], want[rows], e_o[rows], d)
            grad, e_g = r.reference(out=out[:r.t, :c].nan_to_num(0.0),
                                    lse=lse.nan_to_num(0.0), d_out=r.d_out)
            R.check(d_qkv[rows, :w], grad[rows], e_g[rows], d)


@pytest.mark.parametrize("kv,group,n", [(1, 1, 300), (8, 8, 1100)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_later_rows_do_not_reach_earlier_ones(bad, kv, group, n):
    """Forward: a row behind holds infinities or NaN as key and value; earlier rows keep their
    bits, later ones get what the sum gives."""
    r = Run([n], kv, group)
    c = r.heads * D
    clean, _ = r.forward()
    at = n - 90
    spoiled = r.qkv.clone()
    heads = spoiled.view(r.t, kv, group + 2, D)
    heads[at, :, group + 1, 5] = bad                # one column of the values
    got, _ = r.forward(spoiled)
    assert torch.equal(got[:at, :c], clean[:at, :c])
    cols = torch.zeros(c, dtype=torch.bool, device=DEV)
    cols[5::D] = True
    later = got[at:r.t, :c].float()
    assert torch.isfinite(later[:, ~cols]).all()
    assert torch.isnan(later[:, cols]).all() if math.isnan(bad) else (later[:, cols] == bad).all()
    assert torch.equal(got[at:r.t, :c][:, ~cols], clean[at:r.t, :c][:, ~cols])
    heads[at, :, group] = bad                       # the key
    got, _ = r.forward(spoiled)
    assert torch.equal(got[:at, :c], clean[:at, :c])


def test_lists_that_are_wrong_stay_inside():
    """Lists that leave the rows or do not ascend: other rows' results stay in place, and
    nothing outside the buffers is touched (results are undefined where lists are)."""
    r = Run([100, 60], 1, 2, behind=20)
    for cu in ([0, 100, 5000], [-70, 100, 160], [0, 150, 60], [200, 300, 400], [-5, -4, -3],
               [2 ** 31 - 1, -2 ** 31, 7]):
        docs = atp.attention_docs(ints(cu), prefix=ints([2 ** 31 - 1, -2 ** 31]))
        out, lse, d_qkv = r.buffers()
        c, w = r.heads * D, r.qkv.shape[1]
        atp.atp_attention_docs_fwd(r.t, 1, 2, docs, r.qkv, out[:r.t, :c], lse)
        ws = torch.zeros(atp.atp_attention_docs_workspace_bytes(r.t, 1, 2), dtype=torch.uint8,
                         device=DEV)
        atp.atp_attention_docs_bwd(r.t, 1, 2, docs, r.qkv, out[:r.t, :c], lse, r.d_out,
                                   d_qkv[:r.t, :w], ws)
        torch.cuda.synchronize()
        assert torch.isnan(out[r.t]).all() and torch.isnan(d_qkv[r.t]).all()
        assert torch.isnan(out[:, c:]).all() and torch.isnan(d_qkv[:, w:]).all()


def test_the_causal_core_is_a_document_of_each_sequence():
    """Group 1, equal lengths: the values of atp_attention_fwd, whose tiles and order of
    sums are the same."""
    batch, seq, heads = 3, 200, 4
    h = heads * D
    m = atp.mesh(1, 1)
    t = batch * seq
    qkv = rand((t, 3 * h), 9)
    out, lse = torch.empty((t, h), dtype=BF, device=DEV), torch.empty((heads, t), device=DEV)
    atp.atp_attention_fwd(m, atp.ATP_BLOCK_COL, batch, seq, h, heads, qkv, out, lse)
    docs = atp.attention_docs(ints(starts([seq] * batch)))
    out2, lse2 = torch.empty_like(out), torch.empty_like(lse)
    atp.atp_attention_docs_fwd(t, heads, 1, docs, qkv, out2, lse2)
    assert (out.float() - out2.float()).abs().max() <= 2 * R.H * out.float().abs().max()
    assert (lse - lse2).abs().max() <= 8 * R.U * lse.abs().max() + 4 * R.EXP


def test_gradient_against_differences():
    """The reference's gradient against central differences of its own forward."""
    n, kv, group, h = 9, 1, 2, 1e-6
    g = torch.Generator().manual_seed(3)
    x = torch.randn((n, (group + 2) * D), generator=g).double()
    do = torch.randn((n, group * D), generator=g).double()
    kw = dict(prefix=[4], slopes=[0.5, 0.0625], cap=2.0)

    def forward(v):
        return R.attention(v, kv, group, [0, n], **kw)
    out, lse, _, _ = forward(x)
    grad, _ = R.attention(x, kv, group, [0, n], **kw, out=out, lse=lse, d_out=do)
    for i, j in ((0, 0), (3, 200), (8, 255), (5, 256), (2, 300), (0, 383), (7, 384), (8, 511)):
        e = torch.zeros_like(x)
        e[i, j] = h
        num = ((forward(x + e)[0] - forward(x - e)[0]) * do).sum() / (2 * h)
        assert abs(num - grad[i, j]) < 1e-6 * max(1.0, abs(grad[i, j]))


def test_nothing():
    docs = atp.attention_docs(ints([0]))
    r = Run([5], 1, 1)
    out, lse, d_qkv = r.buffers()
    atp.atp_attention_docs_fwd(r.t, 1, 1, docs, r.qkv, out[:r.t, :D], lse)
    assert torch.isnan(out).all() and torch.isnan(lse).all()
    empty = atp.attention_docs(ints([0, 0, 0]))
    atp.atp_attention_docs_fwd(r.t, 1, 1, empty, r.qkv, out[:r.t, :D], lse)
    assert torch.isnan(out).all() and torch.isnan(lse).all()


@pytest.mark.parametrize("kv,n,slopes", [(2, 300, False), (2, 300, True), (16, 4096, False),
                                         (16, 4096, True)])
def test_seen_scores_of_minus_infinity_weigh_nothing(kv, n, slopes):
    # a first tile of such scores, and some among others: what scores of -1e30 give, whose
    # weights are exactly zero beside any other (rows that see nothing else are NaN)
    run = Run([n], kv, 1, slopes=slopes)
    got = []
    for low in (-float("inf"), -1e30):
        qkv = run.qkv.clone()
        heads = qkv.view(n, kv, 3, D)
        heads[:, :, 0, 0] = heads[:, :, 0, 0].abs() + 0.5
        for at in (slice(0, 64), slice(70, 76), slice(190, 191)):
            heads[at, :, 1, 0] = low
        out, lse = run.forward(qkv)
        got.append((out[64:n, :run.heads * D], lse[:, 64:]))
    (out, lse), (out0, lse0) = got
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    assert torch.equal(out.view(torch.int16), out0.view(torch.int16))
    assert torch.equal(lse, lse0)


@pytest.mark.parametrize("kv,group,kw", [(4, 3, {}), (1, 12, dict(slopes=True)),
                                         (8, 1, dict(cap=20.0)),
                                         (2, 5, dict(slopes=True, cap=9.0))])
def test_many_short_documents(kv, group, kw):
    # enough tiles for the kernels of 128 rows, though no document has many
    lens = [1 + 37 * d % 250 for d in range(30)]
    prefix = [0 if d % 3 else n // 2 for d, n in enumerate(lens)] if kw.get("slopes") else None
    Run(lens, kv, group, prefix=prefix, first=2, behind=61, seed=kv, **kw).check()


@pytest.mark.parametrize("kv,cap", [(86, 0.0), (86, 20.0), (255, 0.0)])
def test_lists_padded_to_the_most_documents(kv, cap):
    # 65536 documents, nearly all empty: more tiles than the kernels of 768 threads can have
    lens = [60] + [0] * 40000 + [1, 0, 67] + [0] * 25532
    Run(lens, kv, 1, cap=cap, seed=4).check()


def bits(t):
    return t.contiguous().view(torch.int16 if t.dtype is BF else torch.int32)


@pytest.mark.parametrize("kv,group,lens", [(2, 2, [70, 200, 129]), (4, 8, [700, 130, 1100])])
@pytest.mark.parametrize("kw", [{}, dict(cap=30.0), dict(slopes=True, prefix=True),
                                dict(cap=30.0, slopes=True, prefix=True)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf"), 3e38])
def test_documents_keep_their_bits_beside_others(kv, group, lens, kw, bad):
    """Whatever other documents and padding rows hold, a document's results have the same bits,
    forward and backward."""
    kw = dict(kw, prefix=[5, 100, 0] if kw.get("prefix") else None)
    r = Run(lens, kv, group, first=10, behind=20, **kw)
    w, c = r.qkv.shape[1], r.heads * D
    out, lse, d_qkv = r.buffers()
    r.forward(buf=(out, lse, d_qkv))
    r.backward(out, lse, d_qkv)
    for d in range(len(lens)):
        rows = slice(r.cu[d], r.cu[d + 1])
        qkv, d_out = torch.full_like(r.qkv, bad), torch.full_like(r.d_out, bad)
        qkv[rows], d_out[rows] = r.qkv[rows], r.d_out[rows]
        o, z, g = r.buffers()
        r.forward(qkv, (o, z, g))
        r.backward(o, z, g, qkv, d_out)
        assert torch.equal(bits(o[rows, :c]), bits(out[rows, :c])), d
        assert torch.equal(bits(z[:, rows]), bits(lse[:, rows])), d
        assert torch.equal(bits(g[rows, :w]), bits(d_qkv[rows, :w])), d
        assert torch.isfinite(g[rows, :w]).all()


@pytest.mark.parametrize("kv,group", [(1, 2), (16, 2)])
def test_long_lists_that_are_wrong_stay_inside(kv, group):
    """More than 64 documents that leave the rows or do not ascend: nothing outside the
    buffers is touched, and rows behind stay as they were."""
    r = Run([300], kv, group, behind=1000)
    c, w = r.heads * D, r.qkv.shape[1]
    g = torch.Generator().manual_seed(2)
    wild = torch.randint(-2 ** 31, 2 ** 31, (90,), generator=g).tolist()
    near = torch.randint(-100, 1500, (90,), generator=g).tolist()
    for cu in (wild, near, sorted(near)[::-1], [1300] * 45 + [0] * 45, [-2 ** 31] * 90,
               [2 ** 31 - 1] * 90, [0] * 89 + [2 ** 31 - 1]):
        prefix = torch.randint(-2 ** 31, 2 ** 31, (89,), generator=g).tolist()
        docs = atp.attention_docs(ints(cu), prefix=ints(prefix))
        out, lse, d_qkv = r.buffers()
        atp.atp_attention_docs_fwd(r.t, kv, group, docs, r.qkv, out[:r.t, :c], lse)
        n = atp.atp_attention_docs_workspace_bytes(r.t, kv, group)
        ws = torch.zeros(n + 64, dtype=torch.uint8, device=DEV)
        atp.atp_attention_docs_bwd(r.t, kv, group, docs, r.qkv, out[:r.t, :c], lse, r.d_out,
                                   d_qkv[:r.t, :w], ws[:n])
        torch.cuda.synchronize()
        assert torch.isnan(out[r.t]).all() and torch.isnan(d_qkv[r.t]).all()
        assert torch.isnan(out[:, c:]).all() and torch.isnan(d_qkv[:, w:]).all()
        assert (ws[n:] == 0).all()
