"""Refusals of the calls around the layers -- embedding, layer norm, attention within
documents, gradient norm and clipping -- before any device work (the pointers are never
dereferenced), and the sizes of their workspaces."""
import ctypes

import pytest
import torch

import paper_2301_08658_amd as atp
from paper_2301_08658_amd import binding as B

P = 0x10000000              # 16-byte aligned, never dereferenced
Q, R, S, T = 0x40000000, 0x50000000, 0x60000000, 0x70000000
ODD = 0x10000004
INV, UNS, OK = B.ATP_ERR_INVALID_ARGUMENT, B.ATP_ERR_UNSUPPORTED, B.ATP_OK
NAN, INF = float("nan"), float("inf")
LIB = atp.load_library()


def ref(x):
    return None if x is None else ctypes.byref(x)


def table(ptrs):
    return None if ptrs is None else (ctypes.c_void_p * max(1, len(ptrs)))(*ptrs)


def emb(t=5, ids=P, v=100, off=0, c=64, w=Q, ldw=64, scale=1.0, out=R, dt=1, ldo=64):
    return LIB.atp_embedding_fwd(t, ids, v, off, c, w, ldw, scale, out, dt, ldo, None)


def emb_bwd(t=5, ids=P, v=100, off=0, c=64, dy=Q, ldy=64, scale=1.0, dw=R, ldw=64, acc=0, ws=S,
            wsb=1 << 20):
    return LIB.atp_embedding_bwd(t, ids, v, off, c, dy, ldy, scale, dw, ldw, acc, ws, wsb, None)


@pytest.mark.parametrize("call", [emb, emb_bwd])
def test_embedding(call):
    assert call(t=-1) == INV and call(t=(1 << 24) + 1) == UNS
    assert call(v=0) == INV and call(v=(1 << 24) + 1) == UNS and call(off=-1) == INV
    assert call(c=0) == INV and call(c=12) == UNS and call(c=(1 << 22) + 8) == UNS
    assert call(scale=NAN) == INV and call(scale=INF) == INV
    assert call(ids=None) == INV and call(ids=ODD) == UNS
    assert call(ldw=56) == INV and call(ldw=68) == UNS


def test_embedding_buffers():
    assert emb(w=None) == INV and emb(w=ODD) == UNS and emb(out=None) == INV
    assert emb(out=ODD) == UNS and emb(ldo=60) == INV and emb(dt=2) == INV
    assert emb(out=Q + 16) == INV and "overlap" in B.last_error()
    assert emb(t=0, ids=None, out=None) == OK
    assert emb_bwd(dy=None) == INV and emb_bwd(dw=None) == INV and emb_bwd(dw=ODD) == UNS
    assert emb_bwd(acc=2) == INV and emb_bwd(ws=None) == INV and emb_bwd(ws=ODD) == UNS
    need = atp.atp_embedding_workspace_bytes(5, 100, 64)
    assert need > 0 and emb_bwd(wsb=need - 1) == INV
    assert emb_bwd(dw=Q) == INV and "overlap" in B.last_error()
    assert emb_bwd(t=0, ids=None, dy=None, ws=None, wsb=0, acc=1) == OK
    for bad in ((-1, 5, 8), (5, 0, 8), (5, 5, 0), ((1 << 24) + 1, 5, 8), (5, (1 << 24) + 1, 8)):
        assert atp.atp_embedding_workspace_bytes(*bad) == 0
    assert atp.atp_embedding_workspace_bytes(0, 5, 8) == 0
    sizes = [atp.atp_embedding_workspace_bytes(1 << i, 50000, 64) for i in range(25)]
    assert sizes == sorted(sizes)


def norm(w=P, b=P, eps=1e-5):
    return B.atp_layer_norm(w, b, eps)


def fwd(t=5, c=64, dt=1, p=norm(), x=P, ldx=64, add=Q, lda=64, xo=R, ldxo=64, n=1, st=None, y=S,
        ldy=64, m=T, r=T):
    return LIB.atp_layer_norm_fwd(t, c, dt, ref(p), x, ldx, add, lda, xo, ldxo, n, table(st), y,
                                  ldy, m, r, None)


def stats(t=5, c=64, dt=1, x=P, ldx=64, add=Q, lda=64, xo=R, ldxo=64, st=T):
    return LIB.atp_layer_norm_stats(t, c, dt, x, ldx, add, lda, xo, ldxo, st, None)


def bwd(t=5, c=64, dt=1, p=norm(), x=P, ldx=64, m=T, r=T, dy=Q, ldy=64, res=None, ldr=64, n=1,
        su=None, dx=R, ldd=64, da=None, lda=64, dw=T, db=T, ws=S, wsb=1 << 24):
    return LIB.atp_layer_norm_bwd(t, c, dt, ref(p), x, ldx, m, r, dy, ldy, res, ldr, n, table(su),
                                  dx, ldd, da, lda, dw, db, ws, wsb, None)


def sums(t=5, c=64, dt=1, p=norm(), x=P, ldx=64, m=T, r=T, dy=Q, ldy=64, su=S):
    return LIB.atp_layer_norm_bwd_sums(t, c, dt, ref(p), x, ldx, m, r, dy, ldy, su, None)


@pytest.mark.parametrize("call", [fwd, stats, bwd, sums])
def test_layer_norm_sizes(call):
    assert call(t=-1) == INV and call(t=(1 << 24) + 1) == UNS
    assert call(c=0) == INV and call(c=60) == UNS and call(c=32776, ldx=32776) == UNS
    assert call(dt=2) == INV and call(x=None) == INV and call(x=ODD) == UNS
    assert call(ldx=56) == INV and call(ldx=68) == UNS
    if call is not stats:
        for p, want in ((None, INV), (norm(eps=-1.0), INV), (norm(eps=NAN), INV),
                        (norm(eps=INF), INV), (norm(w=ODD), UNS), (norm(b=ODD), UNS)):
            assert call(p=p) == want


def test_layer_norm_buffers():
    for call in (fwd, stats):
        assert call(add=None) == INV and call(xo=None) == INV
        assert call(lda=56) == INV and call(ldxo=56) == INV and call(add=ODD) == UNS
        assert call(xo=P + 16) == INV and call(xo=P, ldxo=72) == INV and call(xo=Q) == INV
        assert call(dt=0, xo=P + 5 * 64 * 2) == INV          # fp32 rows are twice as long
    assert stats(st=None) == INV and stats(st=ODD) == UNS
    assert fwd(y=None) == INV and fwd(y=P) == INV and fwd(y=R) == INV and fwd(y=Q) == INV
    assert fwd(m=None) == INV and fwd(r=ODD) == UNS
    lone = dict(add=None, xo=None)
    assert fwd(n=0, **lone) == INV and fwd(n=2, **lone) == INV and fwd(n=65, **lone) == UNS
    assert fwd(n=2, st=[T, None], **lone) == INV
    assert fwd(n=2, st=[T, T]) == INV and "add belongs" in B.last_error()
    assert fwd(t=0, x=None, y=None, m=None, r=None, **lone) == OK
    for call in (bwd, sums):
        assert call(dy=None) == INV and call(ldy=56) == INV and call(m=None) == INV
        assert call(r=ODD) == UNS
    assert sums(su=None) == INV
    assert bwd(dx=None) == INV and bwd(dx=P) == INV and bwd(dx=Q) == INV
    assert bwd(res=R + 16) == INV and bwd(res=R, ldr=72) == INV and bwd(res=ODD) == UNS
    assert bwd(da=R) == INV and bwd(da=P) == INV and bwd(da=Q) == INV and bwd(da=ODD) == UNS
    assert bwd(n=2) == INV and bwd(n=2, su=[T, None]) == INV and bwd(n=65, su=[T] * 65) == UNS
    assert bwd(dw=ODD) == UNS and bwd(ws=None) == INV
    assert bwd(wsb=atp.atp_layer_norm_workspace_bytes(5, 64) - 1) == INV
    assert bwd(t=0, x=None, dy=None, dx=None, m=None, r=None, dw=None, db=None, ws=None) == OK
    for bad in ((-1, 64), (5, 0), (5, 60), (5, 32776), ((1 << 24) + 1, 64)):
        assert atp.atp_layer_norm_workspace_bytes(*bad) == 0
    assert atp.atp_layer_norm_workspace_bytes(0, 64) == 0
    for c in (8, 512, 2048, 2056, 10240, 20480, 32768):
        sizes = [atp.atp_layer_norm_workspace_bytes(1 << i, c) for i in range(25)]
        assert all(0 < s <= 1280 * 2 * 4 * c for s in sizes)


def docs(cu=P, pre=None, sl=None, n=3, cap=0.0):
    return B.atp_attention_docs(cu, pre, sl, n, cap)


W = 2 * 3 * 128


def att(t=9, kv=2, g=1, d=docs(), x=Q, ldx=W, o=R, ldo=256, z=T):
    return LIB.atp_attention_docs_fwd(t, kv, g, ref(d), x, ldx, o, ldo, z, None)


def att_bwd(t=9, kv=2, g=1, d=docs(), x=Q, ldx=W, o=R, ldo=256, z=T, do=S, lddo=256, dx=T,
            lddx=W, ws=P, wsb=1 << 24):
    return LIB.atp_attention_docs_bwd(t, kv, g, ref(d), x, ldx, o, ldo, z, do, lddo, dx, lddx, ws,
                                      wsb, None)


@pytest.mark.parametrize("call", [att, att_bwd])
def test_attention_docs(call):
    assert call(t=-1) == INV and call(t=(1 << 24) + 1) == UNS
    assert call(kv=0) == INV and call(g=0) == INV and call(g=65) == UNS and call(kv=1 << 20) == UNS
    for d, want in ((None, INV), (docs(cu=None), INV), (docs(cu=ODD), UNS), (docs(pre=ODD), UNS),
                    (docs(sl=ODD), UNS), (docs(n=-1), INV), (docs(n=65537), UNS),
                    (docs(cap=-1.0), INV), (docs(cap=NAN), INV), (docs(cap=INF), INV)):
        assert call(d=d) == want, B.last_error()
    assert call(t=1 << 24, kv=10000, ldx=10000 * 384, ldo=10000 * 128) == UNS
    assert "tiles" in B.last_error()
    assert call(x=None) == INV and call(x=ODD) == UNS and call(ldx=W - 8) == INV
    assert call(o=None) == INV and call(ldo=128) == INV and call(z=None) == INV
    assert call(z=ODD) == UNS
    assert call(d=docs(n=0, cu=None)) == OK


def test_attention_docs_buffers():
    assert att(o=Q + 64) == INV and "overlap" in B.last_error()
    assert att(t=0, x=None, o=None, z=None) == OK
    assert att_bwd(do=None) == INV and att_bwd(dx=None) == INV and att_bwd(lddo=128) == INV
    for p in (Q, R, S):
        assert att_bwd(dx=p) == INV and "overlap" in B.last_error()
    need = atp.atp_attention_docs_workspace_bytes(9, 2, 1)
    assert att_bwd(ws=None) == INV and att_bwd(wsb=need - 1) == INV
    for bad in ((-1, 1, 1), (5, 0, 1), (5, 1, 0), (5, 1, 65), ((1 << 24) + 1, 1, 1)):
        assert atp.atp_attention_docs_workspace_bytes(*bad) == 0
    assert atp.atp_attention_docs_workspace_bytes(0, 1, 1) == 0


def grad(src=P, dst=Q, rows=1, cols=100, lds=100, ldd=100, st=0, dt=1):
    return B.atp_grad(src, dst, rows, cols, lds, ldd, st, dt)


def sq(gs=(grad(),), n=None, out=R, ws=S, wsb=1 << 20):
    arr = (B.atp_grad * max(1, len(gs)))(*gs)
    return LIB.atp_grad_sq_sum(len(gs) if n is None else n, arr, out, ws, wsb, None)


def clip(gs=(grad(),), n=None, parts=(R,), red=None, scale=1.0, top=1.0, norm=T):
    arr = (B.atp_grad * max(1, len(gs)))(*gs)
    return LIB.atp_grad_clip(len(gs) if n is None else n, arr, len(parts) if red is None else red,
                             table(list(parts)), scale, top, norm, None)


@pytest.mark.parametrize("call", [sq, clip])
def test_gradients(call):
    assert call(n=-1) == INV
    for g, want in ((grad(src=None), INV), (grad(src=ODD), UNS), (grad(rows=-1), INV),
                    (grad(cols=-1), INV), (grad(st=2), INV), (grad(rows=3, lds=99), INV),
                    (grad(rows=3, lds=101), UNS), (grad(rows=3, lds=(1 << 22) + 8), UNS),
                    (grad(rows=1 << 31), UNS), (grad(cols=(1 << 40) + 1), UNS),
                    (grad(rows=1 << 20, cols=1 << 21, lds=1 << 21, ldd=1 << 21), UNS)):
        assert call(gs=(grad(), g)) == want, B.last_error()


def test_gradient_scalars():
    assert sq(out=None) == INV and sq(out=ODD + 2) == UNS and sq(ws=None) == INV
    assert sq(wsb=7) == INV
    assert clip(gs=(grad(dst=None),)) == INV and clip(gs=(grad(dst=ODD),)) == UNS
    assert clip(gs=(grad(dt=5),)) == INV and clip(gs=(grad(dst=P),)) == INV      # another type
    assert clip(gs=(grad(dst=P + 16, dt=0),)) == INV
    assert clip(gs=(grad(rows=3, lds=100, ldd=104),)) == UNS     # 100 is no multiple of 8
    assert clip(parts=()) == INV and clip(parts=(None,)) == INV and clip(parts=(R, ODD + 2)) == UNS
    assert clip(parts=[R] * 65) == UNS
    for bad in (0.0, -1.0, NAN, INF):
        assert clip(scale=bad) == INV
    for bad in (0.0, -1.0, NAN):
        assert clip(top=bad) == INV
    assert clip(norm=None) == INV and clip(norm=ODD) == UNS
    assert LIB.atp_grad_workspace_bytes(-1, None) == 0 == LIB.atp_grad_workspace_bytes(0, None)
    arr = (B.atp_grad * 2)(grad(cols=16384), grad(cols=16385))
    assert LIB.atp_grad_workspace_bytes(2, arr) == 3 * 8
    arr[1].src = None
    assert LIB.atp_grad_workspace_bytes(2, arr) == 0


def test_binding_checks_sizes_and_devices():
    cpu = torch.zeros((8, 16), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU"):
        atp.layer_norm(cpu[0])
    with pytest.raises(ValueError, match="weight has 16"):
        atp.layer_norm(cpu[0], torch.zeros(8, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="GPU"):
        atp.attention_docs(torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError, match="n_docs"):
        atp.attention_docs(torch.zeros(0, dtype=torch.int32))
    with pytest.raises(ValueError, match="GPU"):
        atp.grad_list([torch.zeros(8)])


def _docs_need(t, kv, group, most):
    """Bytes of a backward of t rows whose heads are divided for `most` tiles."""
    want = min(group, -(-most // (max(1, t // 64) * kv)))
    heads = -(-group // want)
    parts = -(-group // heads)
    return 4 * (-(-t * kv * group // 64) * 64 + (parts * t * kv * 256 if parts > 1 else 0))


@pytest.mark.parametrize("kv,group", [(2, 8), (1, 64), (4, 3), (1, 12), (20, 1), (3, 7), (700, 2)])
def test_attention_workspace_of_the_largest_batch(kv, group):
    # what is enough for a batch is enough for every smaller one, however it is divided
    sizes, t = [], 1
    while t < 1 << 18:
        sizes.append((t, atp.atp_attention_docs_workspace_bytes(t, kv, group)))
        t += 1 if t < 130 else 63 + t // 50
    for (_, a), (_, b) in zip(sizes, sizes[1:]):
        assert a <= b
    largest = 0
    for t, have in sizes:
        largest = max(largest, _docs_need(t, kv, group, 1024))
        assert have >= largest
    # not more than the largest of them and the last one's row values
    assert sizes[-1][1] <= max(_docs_need(t, kv, group, 1024) for t in range(1, 70000, 7)) * 1.02 \
        + _docs_need(sizes[-1][0], kv, group, 1)


@pytest.mark.parametrize("cols", [8, 64, 520, 2048, 4096, 20480, 1 << 20])
def test_embedding_workspace_of_the_largest_batch(cols):
    # lists of sorted tokens, and two rows of sums for each chunk of tokens
    def need(t):
        values = t * cols
        chunk = 8 if values < 1 << 22 else 16 if values < 1 << 25 else 32 if values < 1 << 27 else 64
        chunk = max(chunk, -(-(-(-t // 2048)) // 8) * 8)
        lists = 8 * t if t <= 16384 else 16 * t + 1024 * -(-t // 8192)
        return lists + -(-t // chunk) * 2 * cols * 4
    sizes, t = [], 1
    while t <= 1 << 24:
        sizes.append((t, atp.atp_embedding_workspace_bytes(t, 50000, cols)))
        t += 1 if t < 40 else 7 + t // 90
    for edge in (1 << 22, 1 << 25, 1 << 27):               # where the chunks change
        t = edge // cols
        sizes += [(k, atp.atp_embedding_workspace_bytes(k, 50000, cols))
                  for k in (t - 1, t, t + 1) if 1 <= k <= 1 << 24]
    sizes.sort()
    largest = 0
    for (_, a), (t, b) in zip([(0, 0)] + sizes, sizes):
        largest = max(largest, need(t))
        assert a <= b and largest <= b
    # a row of sums above the largest batch's, and the lists' alignment
    assert sizes[-1][1] <= largest + 8 * sizes[-1][0] + 8 * cols * 64


@pytest.mark.parametrize("cols", [8, 512, 1024, 2048, 2056, 5120, 10240, 20480, 32768])
def test_layer_norm_workspace_of_the_largest_batch(cols):
    # two rows of sums for each workgroup
    vecs = cols // 8
    one = vecs <= 256
    nv = 2 if vecs <= 1280 else 4
    most = 1024 if one else 256 * max(1, 1024 // (64 * -(-vecs // (64 * nv))))
    rows = 4 if one else 1

    def need(t):
        visits = max(-(-t // (most * rows)), 2 if one else 4)
        return -(-t // (visits * rows)) * 2 * cols * 4
    largest, last, t = 0, 0, 1
    while t <= 1 << 24:
        have = atp.atp_layer_norm_workspace_bytes(t, cols)
        largest = max(largest, need(t))
        assert last <= have and largest <= have
        last, t = have, t + (1 if t < 30000 else t // 90)
    assert last == largest


def test_workspaces_of_refused_columns():
    for cols in (1, 4, 12, 1 << 22 | 8):
        assert emb_bwd(c=cols, ldy=1 << 22, ldw=1 << 22) == UNS
        assert atp.atp_embedding_workspace_bytes(5, 100, cols) == 0


@pytest.mark.parametrize("call", [att, att_bwd])
def test_attention_tiles_of_one_launch(call):
    # 65538 tiles of 256 heads, in workgroups of 256 threads: a launch of 2^32
    wide = dict(t=128, kv=256, ldx=256 * 384, ldo=256 * 128, d=docs(n=65536))
    assert call(**wide) == UNS and "tiles" in B.last_error()


def test_rows_of_one_launch():
    # 2^32 threads: HIP drops what a launch has beyond them without an error
    most = 1 << 24
    assert emb(t=most, c=8192, ldw=8192, ldo=8192, w=1 << 46) == UNS
    assert "2^37" in B.last_error()
    for t, c in ((most, 4096), (13421773, 5120), (6710887, 20480), (1 << 22, 32768)):
        for call in (stats, fwd):
            assert call(t=t, c=c, ldx=c, add=None, xo=None) == UNS and "rows" in B.last_error()


def test_written_memory_is_apart():
    """Buffers far from each other but for the named pair."""
    at = {k: (i + 1) << 32 for i, k in enumerate("ids w out dy dw ws x add xo y m r st p b res dx da "
                                                 "db su qkv o z do cu pre sl".split())}

    def pairs(call, base, written, read):
        for a in written:
            for b in list(written) + list(read):
                if a == b:
                    continue
                assert call(**{**base, a: base[b]}) == INV, (a, b)
                assert "overlap" in B.last_error(), (a, b)
    pairs(emb, dict(ids=at["ids"], w=at["w"], out=at["out"]), ["out"], ["ids", "w"])
    pairs(emb_bwd, dict(ids=at["ids"], dy=at["dy"], dw=at["dw"], ws=at["ws"]), ["dw", "ws"],
          ["ids", "dy"])
    lone = {k: at[k] for k in ("x", "y", "m", "r")}
    pairs(fwd, dict(lone, add=None, xo=None, p=norm(at["p"], at["b"])), ["y", "m", "r"], ["x"])
    both = dict(lone, add=at["add"], xo=at["xo"], p=norm(at["p"], at["b"]))
    pairs(fwd, both, ["y", "m", "r"], ["x", "add", "xo"])
    for k in ("y", "m", "r", "xo"):
        for q in ("p", "b"):
            assert fwd(**{**both, k: at[q]}) == INV and "overlap" in B.last_error(), (k, q)
        if k != "xo":
            assert fwd(**{**lone, k: at["st"]}, add=None, xo=None, n=2, p=norm(at["p"], at["b"]),
                       st=[at["su"], at["st"]]) == INV and "overlap" in B.last_error()
    pairs(stats, {k: at[k] for k in ("x", "add", "xo", "st")}, ["st"], ["x", "add", "xo"])
    back = dict(x=at["x"], m=at["m"], r=at["r"], dy=at["dy"], p=norm(at["p"], at["b"]))
    pairs(sums, dict(back, su=at["su"]), ["su"], ["x", "m", "r", "dy"])
    assert sums(**back, su=at["p"]) == INV and "overlap" in B.last_error()
    back.update(res=at["res"], dx=at["dx"], da=at["da"], dw=at["dw"], db=at["db"], ws=at["ws"])
    pairs(bwd, back, ["da", "dw", "db", "ws"], ["x", "m", "r", "dy", "res", "dx"])
    pairs(bwd, back, ["dx"], ["x", "m", "r", "dy"])          # dx may be res
    for k in ("dx", "da", "dw", "db", "ws"):
        assert bwd(**{**back, k: at["p"]}) == INV and "overlap" in B.last_error()
        assert bwd(**{**back, k: at["su"]}, n=2, su=[at["st"], at["su"]]) == INV
        assert "overlap" in B.last_error()
    lists = docs(cu=at["cu"], pre=at["pre"], sl=at["sl"])
    fore = dict(x=at["qkv"], o=at["o"], z=at["z"], d=lists)
    pairs(att, fore, ["o", "z"], ["x"])
    aft = dict(fore, do=at["do"], dx=at["dx"], ws=at["ws"])
    pairs(att_bwd, aft, ["dx", "ws"], ["x", "o", "z", "do"])
    for call, base, written in ((att, fore, "oz"), (att_bwd, aft, ("dx", "ws"))):
        for k in written:
            for q in ("cu", "pre", "sl"):
                assert call(**{**base, k: at[q]}) == INV and "overlap" in B.last_error()
