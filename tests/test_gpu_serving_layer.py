"""A layer's attention answers with the framework's own linears around the position, cache
and cached-attention calls: a prompt in two chunks, then single tokens."""
import pytest
import torch

import cache_reference as C
import paper_2301_08658_amd as atp
from test_gpu_serving import BF, D, DEV, Server, close, whole

pytestmark = pytest.mark.gpu


def linear(mode, x, w, b):
    y = torch.empty((x.shape[0], w.shape[1]), dtype=BF, device=DEV)
    atp.atp_shard_linear_fwd(atp.mesh(1, 1), mode, x.shape[0], w.shape[0], w.shape[1], 1, x, w, b,
                             atp.ATP_EPI_BIAS, y)
    # one rounding of the result; sums of k products and the bias in fp32
    xd, wd = C.f64(x), C.f64(w)
    want = xd @ wd + C.f64(b)
    size = xd.abs() @ wd.abs() + C.f64(b).abs()
    close(y, want, C.HALF_BF16 * want.abs() + (w.shape[0] + 2) * C.EPS32 * 2 * size)
    return y


@pytest.mark.parametrize("kv,group,page", [(2, 1, 16), (1, 4, 64)])
def test_prompt_and_single_tokens_through_the_layer(kv, group, page):
    """Every step's QKV rows, attention and out-proj against 64 bits, each from the bits
    that the call before it gave."""
    h, width = 256, kv * group * D
    g = torch.Generator().manual_seed(31)
    wq = (torch.randn((h, kv * (group + 2) * D), generator=g) / 16).to(BF).to(DEV)
    wo = (torch.randn((width, h), generator=g) / 16).to(BF).to(DEV)
    bq, bo = torch.randn(wq.shape[1], generator=g).to(BF).to(DEV), \
        torch.randn(h, generator=g).to(BF).to(DEV)
    srv = Server(kv, group, page, 16, 1, 8)
    qkv = None
    for n in (50, 37, 1, 1, 1):
        x = torch.randn((n, h), generator=g).to(BF).to(DEV)
        rows = linear(atp.ATP_COL_FIRST, x, wq, bq)
        qkv = rows if qkv is None else torch.cat((qkv, rows))
        attn = srv.step(rows, [n])
        want, bound = whole(srv, qkv)
        close(attn, want[-n:], bound[-n:])
        linear(atp.ATP_ROW_FIRST, attn, wo, bo)
