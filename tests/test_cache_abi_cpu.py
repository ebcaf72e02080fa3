"""Refusals of the position, cache and cached-attention calls, before any device
work (the pointers are never dereferenced), and the sizes of their workspaces."""
import ctypes

import pytest

import paper_2301_08658_amd as atp
from paper_2301_08658_amd import binding as B

P = 0x100000                # 16-byte aligned, never dereferenced
Q, R, S, T = 0x40000000, 0x50000000, 0x60000000, 0x70000000
ODD = 0x100004
INV, SHAPE, UNS, OK = (B.ATP_ERR_INVALID_ARGUMENT, B.ATP_ERR_SHAPE, B.ATP_ERR_UNSUPPORTED,
                       B.ATP_OK)


def params(qw=P, kw=P, inv=P, eps=1e-6, norm=1, rot=128, inter=0):
    return B.atp_qk_norm_rope(qw, kw, inv, eps, norm, rot, inter)


def cache(pages=T, n=16, kv=2, page=64):
    return B.atp_kv_cache(pages, n, kv, page)


def batch(table=P, ld=8, cols=8, n=3, ctx=P, cu=P):
    return B.atp_kv_batch(table, ld, cols, n, ctx, cu)


def ref(x):
    return None if x is None else ctypes.byref(x)


LIB = atp.load_library()
W1 = 2 * 3 * 128            # two heads, group 1


def fwd(b=2, s=8, kv=2, g=1, p=params(), pos=None, x=P, ldx=W1, y=Q, ldy=W1):
    return LIB.atp_qk_norm_rope_fwd(b, s, kv, g, ref(p), pos, x, ldx, y, ldy, None)


def bwd(b=2, s=8, kv=2, g=1, p=params(), x=P, ldx=W1, dy=Q, lddy=W1, dx=R, lddx=W1, dq=S, dk=S,
        ws=T, wsb=1 << 20, pos=None):
    return LIB.atp_qk_norm_rope_bwd(b, s, kv, g, ref(p), pos, x, ldx, dy, lddy, dx, lddx, dq, dk,
                                    ws, wsb, None)


def app(c=cache(), b=batch(), t=5, g=1, p=params(), x=P, ldx=W1, q=Q, ldq=256, pos=None):
    return LIB.atp_qk_norm_rope_cache(ref(c), ref(b), t, g, ref(p), pos, x, ldx, q, ldq, None)


def att(c=cache(), b=batch(), t=5, g=1, mx=1, q=P, ldq=256, mask=None, words=0, out=Q, ldo=256,
        lse=R, ws=S, wsb=1 << 30):
    return LIB.atp_attention_cache_fwd(ref(c), ref(b), t, g, mx, q, ldq, mask, words, out, ldo, lse,
                                       ws, wsb, None)


BAD_PARAMS = [(None, INV), (params(norm=2), INV), (params(inter=-1), INV),
              (params(eps=-1.0), INV), (params(eps=float("nan")), INV),
              (params(eps=float("inf")), INV), (params(norm=0), INV), (params(rot=-8), INV),
              (params(rot=136), INV), (params(rot=4), UNS), (params(inv=None), INV),
              (params(inv=ODD), UNS), (params(qw=ODD), UNS), (params(kw=ODD), UNS)]


@pytest.mark.parametrize("call", [fwd, bwd, app])
def test_parameters(call):
    for p, want in BAD_PARAMS:
        assert call(p=p) == want, (call.__name__, atp.binding.last_error())


def test_norm_rope_sizes_and_buffers():
    for call in (fwd, bwd):
        assert call(b=-1) == INV and call(s=-1) == INV
        assert call(kv=0) == INV and call(g=0) == INV and call(g=65) == UNS
        assert call(kv=1 << 20) == UNS
        assert call(b=1 << 25) == UNS and call(b=1 << 13, s=1 << 13) == UNS
        assert call(x=None) == INV and call(x=ODD) == UNS and call(ldx=W1 - 8) == INV
        assert call(ldx=W1 + 4) == UNS and call(pos=ODD) == UNS
    assert fwd(y=None) == INV and fwd(ldy=128) == INV
    assert fwd(y=P + 64) == INV and "overlap" in atp.binding.last_error()
    assert fwd(y=P, ldy=W1 + 8) == INV          # in place with another leading dimension
    assert fwd(b=0, x=None, y=None) == OK and fwd(s=0, x=None, y=None) == OK
    assert bwd(dx=P) == INV and bwd(dx=Q + 256) == INV and bwd(dx=Q, lddx=W1 + 8) == INV
    assert bwd(ws=None) == INV and bwd(ws=ODD) == UNS
    assert bwd(wsb=atp.atp_qk_norm_rope_workspace_bytes(16) - 1) == INV
    assert bwd(dq=ODD) == UNS and bwd(dk=ODD) == UNS
    assert bwd(p=params(qw=None, kw=None, norm=0)) == INV
    assert "without norm" in atp.binding.last_error()
    assert bwd(b=0, dq=None, dk=None, ws=None, wsb=0, x=None, dy=None, dx=None) == OK
    assert atp.atp_qk_norm_rope_workspace_bytes(-1) == 0
    assert atp.atp_qk_norm_rope_workspace_bytes(0) == 0
    assert atp.atp_qk_norm_rope_workspace_bytes(1) == 1024
    big = [atp.atp_qk_norm_rope_workspace_bytes(1 << i) for i in range(25)]
    assert big == sorted(big) and big[-1] == big[-2]


BAD_CACHE = [(None, INV), (cache(pages=None), INV), (cache(pages=ODD), UNS), (cache(n=0), INV),
             (cache(n=(1 << 28) + 1), UNS), (cache(kv=0), INV), (cache(page=0), INV),
             (cache(page=8), UNS), (cache(page=48), UNS), (cache(page=2048), UNS)]
BAD_BATCH = [(None, INV), (batch(table=None), INV), (batch(table=ODD), UNS), (batch(ld=7), INV),
             (batch(cols=0), INV), (batch(cols=1 << 26, ld=1 << 26), UNS), (batch(n=-1), INV),
             (batch(n=(1 << 16) + 1), UNS)]


@pytest.mark.parametrize("call", [app, att])
def test_cache_and_batch(call):
    for c, want in BAD_CACHE:
        assert call(c=c) == want, atp.binding.last_error()
    for b, want in BAD_BATCH + [(batch(ctx=None), INV), (batch(cu=None), INV),
                                (batch(ctx=ODD), UNS), (batch(cu=ODD), UNS)]:
        assert call(b=b) == want, atp.binding.last_error()
    assert call(t=-1) == INV and call(t=(1 << 24) + 1) == UNS
    assert call(g=0) == INV and call(g=65) == UNS
    assert call(b=batch(n=0)) == OK


def test_append_and_attention_buffers():
    assert app(x=None) == INV and app(q=None) == INV and app(ldx=W1 - 8) == INV
    assert app(ldq=128) == INV and app(q=P) == INV and app(x=T) == INV and app(q=T + 1024) == INV
    assert app(t=0, x=None, q=None) == OK
    assert att(q=None) == INV and att(out=None) == INV and att(ldq=260) == UNS
    assert att(out=P) == INV and att(out=T) == INV and att(lse=ODD) == UNS
    assert att(mx=0) == INV and att(mask=P, words=0) == INV and att(mask=ODD, words=1) == UNS
    assert att(ws=None) == INV and att(ws=ODD) == UNS
    assert att(wsb=atp.atp_attention_cache_workspace_bytes(2, 1, 1) - 1) == INV
    # more rows than the workspace was made for
    assert att(mx=64, wsb=atp.atp_attention_cache_workspace_bytes(2, 1, 1)) == INV
    assert att(t=0, q=None, out=None, lse=None, ws=None, wsb=0) == OK
    sizes = [atp.atp_attention_cache_workspace_bytes(2, 4, n) for n in (1, 4, 5, 8, 9, 1000)]
    assert sizes[0] == sizes[1] < sizes[2] == sizes[3] < sizes[4] == sizes[5]
    for args in ((0, 1, 1), (1, 0, 1), (1, 65, 1), (1, 1, 0)):
        assert atp.atp_attention_cache_workspace_bytes(*args) == 0


def reserve(n=16, page=64, refs=P, b=batch(), m=P, s=P, d=P, r=P, ws=S, wsb=1 << 20):
    return LIB.atp_cache_reserve(n, page, refs, ref(b), m, s, d, r, ws, wsb, None)


def fork(n=16, page=64, refs=P, b=batch(), f=2, p=P, c=P, d=P):
    return LIB.atp_cache_fork(n, page, refs, ref(b), f, p, c, d, None)


def release(n=16, page=64, refs=P, b=batch(), k=P):
    return LIB.atp_cache_release(n, page, refs, ref(b), k, None)


def copy(c=cache(), n=2, s=P, d=P, r=None):
    return LIB.atp_cache_copy_pages(ref(c), n, s, d, r, None)


def compact(c=cache(), b=batch(), cu=P, k=P, n=4, m=None):
    return LIB.atp_cache_compact(ref(c), ref(b), cu, k, n, m, None)


@pytest.mark.parametrize("call", [reserve, fork, release])
def test_pages(call):
    assert call(n=0) == INV and call(n=(1 << 28) + 1) == UNS and call(page=24) == UNS
    assert call(page=0) == INV and call(refs=None) == INV and call(refs=ODD) == UNS
    for b, want in BAD_BATCH:
        assert call(b=b) == want


def test_page_lists():
    assert reserve(b=batch(ctx=None)) == INV and reserve(b=batch(cu=None)) == INV
    for k in "msdr":
        assert reserve(**{k: None}) == INV and reserve(**{k: ODD}) == UNS
    assert reserve(ws=None) == INV and reserve(wsb=4 * (16 + 3) - 1) == INV
    assert reserve(b=batch(n=0), m=None, ws=None) == OK
    assert atp.atp_cache_workspace_bytes(16, 3) == 76
    assert atp.atp_cache_workspace_bytes(0, 3) == 0 == atp.atp_cache_workspace_bytes(1, -1)
    assert fork(b=batch(ctx=None)) == INV and fork(f=-1) == INV and fork(f=4097) == UNS
    for k in "pcd":
        assert fork(**{k: None}) == INV and fork(**{k: ODD}) == UNS
    assert fork(f=0, p=None, c=None, d=None) == OK
    assert release(k=None) == INV and release(k=ODD) == UNS
    assert release(b=batch(n=0), k=None) == OK
    for c, want in BAD_CACHE:
        assert copy(c=c) == want and compact(c=c) == want
    assert copy(n=-1) == INV and copy(s=None) == INV and copy(d=ODD) == UNS and copy(r=ODD) == UNS
    assert copy(n=0, s=None, d=None) == OK
    for b, want in BAD_BATCH + [(batch(ctx=None), INV)]:
        assert compact(b=b) == want
    assert compact(cu=None) == INV and compact(k=None) == INV and compact(n=-1) == INV
    assert compact(m=ODD) == UNS and compact(b=batch(n=0), cu=None) == OK


def test_binding_checks_sizes_and_devices():
    import torch
    cpu = torch.zeros((4, 2, 1, 16, 128), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU"):
        atp.kv_cache(cpu)
    with pytest.raises(TypeError):
        atp.kv_cache(cpu.float())
    with pytest.raises(ValueError, match="contiguous"):
        atp.kv_cache(cpu[:, :, :, ::2])
    with pytest.raises(TypeError):
        atp.kv_batch(torch.zeros((2, 3), dtype=torch.int64))
    with pytest.raises(ValueError, match="row-major"):
        atp.kv_batch(torch.zeros((3, 2), dtype=torch.int32).t())
    with pytest.raises(ValueError, match="frequencies"):
        atp.qk_norm_rope(rotary_dims=64)
    with pytest.raises(ValueError, match="GPU"):
        atp.qk_norm_rope(q_weight=torch.ones(128, dtype=torch.bfloat16))


def test_copy_list_length():
    """More entries than a grid has workgroups are refused before anything is launched."""
    assert copy(n=(1 << 23) + 1) == UNS and copy(n=-1) == INV and copy(n=0, s=None) == OK
