"""A training step of one layer on packed documents, through the public calls in the order
of their use: embedding, norms with residual sums, linears, query/key norms with
rotation, attention within documents, the way back, and the clipping of all gradients.
Every call around the linears is held to its 64-bit definition on the values it got;
the step is captured into a graph and replayed with other documents and tokens; and the
calls take sizes beyond 32-bit offsets, other streams and threads."""
import gc
import threading

import pytest
import torch

import paper_2301_08658_amd as atp
import train_reference as R

pytestmark = pytest.mark.gpu
DEV, BF, F32, D = "cuda:0", torch.bfloat16, torch.float32, 128


@pytest.fixture(autouse=True)
def _no_collection_during_a_capture():
    gc.collect()
    gc.disable()
    yield
    gc.enable()


def rand(shape, seed, std=1.0, mean=0.0, dtype=BF):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std + mean).to(dtype).to(DEV)


class Step:
    """Buffers of a step over at most t rows, and the step itself."""

    def __init__(self, t, h, kv, group, vocab, n_docs, stream=F32):
        self.t, self.h, self.kv, self.group, self.dtype = t, h, kv, group, stream
        self.m = atp.mesh(1, 1)
        qc, ac = kv * (group + 2) * D, kv * group * D
        self.qc, self.ac = qc, ac
        self.ids = torch.zeros(t, dtype=torch.int32, device=DEV)
        self.positions = torch.zeros(t, dtype=torch.int32, device=DEV)
        self.cu = torch.zeros(n_docs + 1, dtype=torch.int32, device=DEV)
        self.docs = atp.attention_docs(self.cu, cap=30.0)
        self.table = rand((vocab, h), 1, 0.05)
        self.shapes = dict(qkv=(h, qc), out=(ac, h), fc1=(h, 4 * h), fc2=(4 * h, h))
        self.w = {k: rand(s, 2 + i, 0.03) for i, (k, s) in enumerate(self.shapes.items())}
        self.b = {k: rand((s[1],), 12 + i, 0.02) for i, (k, s) in enumerate(self.shapes.items())}
        self.nw = [(rand((h,), 20 + i, 0.1, 1.0), rand((h,), 30 + i, 0.1)) for i in range(3)]
        self.norms = [atp.layer_norm(w, b) for w, b in self.nw]
        inv = (10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)).float().to(DEV)
        self.rope = atp.qk_norm_rope(inv_freq=inv, rotary_dims=D)
        self.dy = rand((t, h), 40, 0.1)                   # the gradient of the last norm

        def new(*shape, dtype=BF):
            return torch.zeros(shape, dtype=dtype, device=DEV)
        self.a = {k: new(t, h, dtype=stream) for k in ("x0", "x1", "x2", "g0", "g1", "g2")}
        self.a.update({k: new(t, h) for k in ("n0", "n1", "n2", "o", "z", "d_o", "d_z", "dn",
                                              "d_emb")})
        self.a.update(qkv=new(t, qc), turned=new(t, qc), attn=new(t, ac), d_attn=new(t, ac),
                      d_turned=new(t, qc), pre=new(t, 4 * h), act=new(t, 4 * h),
                      d_act=new(t, 4 * h), lse=new(kv * group, t, dtype=F32))
        self.stat = [(new(t, dtype=F32), new(t, dtype=F32)) for _ in range(3)]
        self.part = {n: new(t, n, dtype=F32) for n in {h, ac, 4 * h}}
        self.grads = {k: new(*s, dtype=F32) for k, s in self.shapes.items()}
        self.grads.update({k + "_b": new(s[1], dtype=F32) for k, s in self.shapes.items()})
        self.grads.update({f"n{i}{p}": new(h, dtype=F32) for i in range(3) for p in "wb"})
        self.grads["table"] = new(vocab, h, dtype=F32)
        self.clipped = {k: torch.zeros_like(v, dtype=BF) for k, v in self.grads.items()}
        self.list = atp.grad_list(list(self.grads.values()), list(self.clipped.values()))
        self.total, self.norm = new(1, dtype=torch.float64), new(2, dtype=F32)
        sizes = [atp.atp_embedding_workspace_bytes(t, vocab, h),
                 atp.atp_layer_norm_workspace_bytes(t, h),
                 atp.atp_attention_docs_workspace_bytes(t, kv, group),
                 atp.atp_grad_workspace_bytes(self.list)]
        self.ws = torch.full((max(sizes),), 0xff, dtype=torch.uint8, device=DEV)   # one for all

    def batch(self, lens, seed):
        cu = [0]
        for n in lens:
            cu.append(cu[-1] + n)
        g = torch.Generator().manual_seed(seed)
        ids = torch.randint(0, 2 * self.table.shape[0], (self.t,), generator=g) // 2
        self.ids.copy_(ids.to(torch.int32))
        self.cu.copy_(torch.tensor(cu, dtype=torch.int32))
        pos = torch.cat([torch.arange(n) for n in lens] + [torch.zeros(self.t - cu[-1])])
        self.positions.copy_(pos.to(torch.int32))
        self.lens, self.starts = lens, cu

    def linear(self, k, x, y, epi=None, preact=None):
        kk, n = self.shapes[k]
        atp.atp_shard_linear_fwd(self.m, atp.ATP_COL_FIRST, self.t, kk, n, 1, x, self.w[k],
                                 self.b[k], atp.ATP_EPI_BIAS if epi is None else epi, y,
                                 preact=preact)

    def linear_bwd(self, k, x, dy, dx, preact=None):
        """dx (bf16) through the reduction of a group of one, where the GeLU's slope belongs."""
        kk, n = self.shapes[k]
        p = self.part[kk]
        atp.atp_shard_linear_bwd(self.m, atp.ATP_COL_FIRST, self.t, kk, n, 1, x, self.w[k], dy, p,
                                 self.grads[k], self.grads[k + "_b"])
        epi = atp.ATP_EPI_NONE if preact is None else atp.ATP_EPI_GELU_BWD
        atp.atp_chunked_partial_reduce(1, self.t, kk, 1, [p], None, epi, dx, preact_in=preact)

    def norm_bwd(self, i, x, dy, dx, d_res, d_add):
        atp.atp_layer_norm_bwd(self.t, self.norms[i], x, *self.stat[i], dy, dx, d_res=d_res,
                               d_add=d_add, dweight=self.grads[f"n{i}w"],
                               dbias=self.grads[f"n{i}b"], workspace=self.ws)

    def run(self):
        a, t = self.a, self.t
        atp.atp_embedding_fwd(t, self.ids, self.table, a["x0"], scale=2.0)
        atp.atp_layer_norm_fwd(t, self.norms[0], a["x0"], a["n0"], *self.stat[0])
        self.linear("qkv", a["n0"], a["qkv"])
        atp.atp_qk_norm_rope_fwd(1, t, self.kv, self.group, self.rope, a["qkv"], a["turned"],
                                 positions=self.positions)
        args = (t, self.kv, self.group, self.docs, a["turned"], a["attn"], a["lse"])
        atp.atp_attention_docs_fwd(*args)
        self.linear("out", a["attn"], a["o"])
        atp.atp_layer_norm_fwd(t, self.norms[1], a["x0"], a["n1"], *self.stat[1], add=a["o"],
                               x_out=a["x1"])
        self.linear("fc1", a["n1"], a["act"], atp.ATP_EPI_BIAS_GELU, a["pre"])
        self.linear("fc2", a["act"], a["z"])
        atp.atp_layer_norm_fwd(t, self.norms[2], a["x1"], a["n2"], *self.stat[2], add=a["z"],
                               x_out=a["x2"])
        wide = self.dtype is F32
        self.norm_bwd(2, a["x2"], self.dy, a["g2"], None, a["d_z"] if wide else None)
        d_z = a["d_z"] if wide else a["g2"]
        self.linear_bwd("fc2", a["act"], d_z, a["d_act"], a["pre"])
        self.linear_bwd("fc1", a["n1"], a["d_act"], a["dn"])
        self.norm_bwd(1, a["x1"], a["dn"], a["g1"], a["g2"], a["d_o"] if wide else None)
        d_o = a["d_o"] if wide else a["g1"]
        self.linear_bwd("out", a["attn"], d_o, a["d_attn"])
        atp.atp_attention_docs_bwd(*args, a["d_attn"], a["d_turned"], self.ws)
        atp.atp_qk_norm_rope_bwd(1, t, self.kv, self.group, self.rope, a["qkv"], a["d_turned"],
                                 a["d_turned"], positions=self.positions)
        self.linear_bwd("qkv", a["n0"], a["d_turned"], a["dn"])
        self.norm_bwd(0, a["x0"], a["dn"], a["g0"], a["g1"], a["d_emb"] if wide else None)
        atp.atp_embedding_bwd(t, self.ids, a["d_emb"] if wide else a["g0"], self.grads["table"],
                              self.ws, scale=2.0)
        atp.atp_grad_sq_sum(self.list, self.total, self.ws)
        atp.atp_grad_clip(self.list, [self.total], self.norm, max_norm=1.0, scale=0.5)

    def outputs(self):
        return {**self.a, **self.grads, **{"c_" + k: v for k, v in self.clipped.items()},
                "norm": self.norm, **{f"s{i}": torch.stack(s) for i, s in enumerate(self.stat)}}


@pytest.mark.parametrize("stream", [F32, BF])
def test_every_call_of_a_step(stream):
    lens = [130, 1, 64, 77, 20]
    s = Step(300, 256, 2, 2, 500, len(lens), stream)
    s.batch(lens, 5)                                      # 292 rows, 8 of padding
    s.run()
    a, rows, t = s.a, s.starts[-1], s.t
    want = R.embedding(s.ids, s.table, 2.0, 0)
    half = R.rounding(stream)
    R.check(a["x0"], want, want.abs() * (half + 2 * R.U), "embedding")
    x_in = {0: a["x0"], 1: a["x1"], 2: a["x2"]}
    for i, (x, y) in enumerate((("x0", "n0"), ("x1", "n1"), ("x2", "n2"))):
        m, m2, e_m, e_m2 = R.norm_stats(a[x])
        y_, r, e_y, e_r = R.norm(a[x], *s.nw[i], 1e-5, m, m2, e_m, e_m2, s.h)
        R.check(a[y], y_, e_y, y)
        R.check(s.stat[i][1], r, e_r, "rstd")
    assert torch.equal(a["x1"], (a["x0"].float() + a["o"].float()).to(stream))
    assert torch.equal(a["x2"], (a["x1"].float() + a["z"].float()).to(stream))
    o, z, e_o, e_z = R.attention(a["turned"], 2, 2, s.starts, cap=30.0)
    R.check(a["attn"][:rows], o[:rows], e_o[:rows], "attention")
    assert (a["attn"][rows:] == 0).all() and (a["d_turned"][rows:] == 0).all()
    # d_turned holds the rotation's gradient by now: the attention's again, beside it
    again = torch.zeros_like(a["d_turned"])
    atp.atp_attention_docs_bwd(t, 2, 2, s.docs, a["turned"], a["attn"], a["lse"], a["d_attn"],
                               again, s.ws)
    g, e_g = R.attention(a["turned"], 2, 2, s.starts, cap=30.0, out=a["attn"], lse=a["lse"],
                         d_out=a["d_attn"])
    R.check(again[:rows], g[:rows], e_g[:rows], "attention's gradient")
    for i, dy, dx, res in ((2, s.dy, "g2", None), (0, a["dn"], "g0", a["g1"])):
        ref = R.norm_bwd(x_in[i], s.nw[i][0], *s.stat[i], dy, res)
        R.check(a[dx], ref["dx"], ref["e_dx"] + half * (ref["dx"].abs() + ref["e_dx"]), dx)
        R.check(s.grads[f"n{i}w"], ref["dw"], ref["e_dw"], "dw")
        R.check(s.grads[f"n{i}b"], ref["db"], ref["e_db"], "db")
    d_emb = a["d_emb"] if stream is F32 else a["g0"]
    g, e = R.embedding_bwd(s.ids, d_emb, 500, 2.0, 0)
    R.check(s.grads["table"], g, e, "table")
    total = sum(float((R.f64(v) ** 2).sum()) for v in s.grads.values())
    norm, f = R.grad_factor(total, 0.5, 1.0)
    assert abs(float(s.norm[0]) - norm) <= 2 * R.U * norm
    for k, v in s.clipped.items():
        w = R.f64(s.grads[k]) * f
        R.check(v, w, w.abs() * (R.H + 8 * R.U) + 2.0 ** -133, k)


def test_replays_with_other_documents():
    """One graph, replayed as tokens, documents and positions change, with eager work and
    synchronizations in between: every replay has the eager step's bits."""
    s = Step(400, 256, 1, 4, 300, 6)
    eager = Step(400, 256, 1, 4, 300, 6)
    s.batch([100, 50, 0, 200, 1, 9], 1)
    s.run()                                               # warm
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        s.run()
    for k, lens in enumerate(([100, 50, 0, 200, 1, 9], [400, 0, 0, 0, 0, 0], [1, 2, 3, 4, 5, 6],
                              [0, 0, 0, 0, 0, 0], [66, 66, 66, 66, 66, 66])):
        for b in (s, eager):
            b.batch(lens, 10 + k)
            for n in ("attn", "d_turned", "lse"):         # rows outside documents are not written
                b.a[n].zero_()
        graph.replay()
        eager.run()
        torch.cuda.synchronize()
        got, want = s.outputs(), eager.outputs()
        for n in want:
            assert torch.equal(got[n], want[n]) or torch.isnan(want[n]).any(), (lens, n)
            assert torch.equal(torch.isnan(got[n]), torch.isnan(want[n])), (lens, n)


def test_two_graphs_share_a_workspace():
    s = Step(200, 128, 1, 1, 100, 2)
    s.batch([150, 40], 3)
    s.run()
    torch.cuda.synchronize()
    want = {k: v.clone() for k, v in s.outputs().items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g in graphs:
        with torch.cuda.graph(g, stream=side):
            s.run()
    for g in graphs + graphs[::-1]:
        s.ws.fill_(0xff)
        g.replay()
    torch.cuda.synchronize()
    for k, v in s.outputs().items():
        assert torch.equal(v, want[k]), k


def test_other_streams_and_threads():
    """Steps of two threads, each on a stream of its own."""
    steps, wants = [], []
    for i in range(2):
        s = Step(260, 128, 1, 2, 90, 3)
        s.batch([200 - 60 * i, 40, 20], 7 + i)
        s.run()
        torch.cuda.synchronize()
        wants.append({k: v.clone() for k, v in s.outputs().items()})
        steps.append(s)
    errors = []

    def work(s):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                for _ in range(5):
                    s.run()
            stream.synchronize()
        except Exception as e:                            # noqa: BLE001
            errors.append(e)
    threads = [threading.Thread(target=work, args=(s,)) for s in steps]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    assert not errors, errors
    for s, want in zip(steps, wants):
        for k, v in s.outputs().items():
            assert torch.equal(v, want[k]), k


# ------------------------------------------------------------------ beyond 32-bit offsets
def test_embedding_of_a_large_table():
    vocab, cols = 110000, 20480                           # 2.25e9 values
    ids = torch.tensor([vocab - 1, 0, 104858, vocab - 1, 52429], dtype=torch.int32, device=DEV)
    table = torch.zeros((vocab, cols), dtype=BF, device=DEV)
    rows = rand((5, cols), 1)
    table[ids[[0, 1, 2, 4]].long()] = rows[[0, 1, 2, 4]]
    out = torch.empty((5, cols), dtype=BF, device=DEV)
    atp.atp_embedding_fwd(5, ids, table, out)
    assert torch.equal(out, rows[[0, 1, 2, 0, 4]])
    del table
    grad = torch.full((vocab, cols), 9.0, device=DEV)
    ws = torch.empty(atp.atp_embedding_workspace_bytes(5, vocab, cols), dtype=torch.uint8,
                     device=DEV)
    atp.atp_embedding_bwd(5, ids, rows, grad, ws)
    assert torch.equal(grad[vocab - 1], rows[0].float() + rows[3].float())
    for i in (1, 2, 4):
        assert torch.equal(grad[int(ids[i])], rows[i].float())
    used = ids[:5].long().unique()
    assert float(grad.abs().sum(1, dtype=torch.float64).sum()) == pytest.approx(
        float(grad[used].abs().sum(1, dtype=torch.float64).sum()))


def test_layer_norm_of_many_wide_rows():
    t, c = 70000, 32768                                   # 2.29e9 values
    norm = atp.layer_norm(None, None)
    x = torch.zeros((t, c), dtype=BF, device=DEV)
    last = rand((3, c), 1, 2.0, 1.0)
    x[-3:] = last
    y = torch.empty_like(x)
    mean, rstd = torch.empty(t, device=DEV), torch.empty(t, device=DEV)
    atp.atp_layer_norm_fwd(t, norm, x, y, mean, rstd)
    m, m2, e_m, e_m2 = R.norm_stats(last)
    want, r, e_y, e_r = R.norm(last, None, None, 1e-5, m, m2, e_m, e_m2, c)
    R.check(y[-3:], want, e_y, "y")
    assert (y[:4] == 0).all() and float(y[:-3].abs().max()) == 0
    dy = torch.zeros_like(x)
    dy[-3:] = rand((3, c), 2)
    dw = torch.empty(c, device=DEV)
    ws = torch.empty(atp.atp_layer_norm_workspace_bytes(t, c), dtype=torch.uint8, device=DEV)
    atp.atp_layer_norm_bwd(t, norm, x, mean, rstd, dy, y, dweight=dw, workspace=ws)
    ref = R.norm_bwd(last, None, mean[-3:], rstd[-3:], dy[-3:], None)
    R.check(y[-3:], ref["dx"], ref["e_dx"] + R.H * (ref["dx"].abs() + ref["e_dx"]), "dx")
    R.check(dw, ref["dw"], ref["e_dw"], "dw")             # the other rows add zeros
    assert float(y[:-3].abs().max()) == 0


def test_attention_of_many_rows():
    """Rows past 2^31 values: the last documents have the results of a call with them alone."""
    kv, n, docs = 20, 500, 700                            # 350000 rows of 7680 columns
    t = n * docs
    qkv = torch.zeros((t, kv * 3 * D), dtype=BF, device=DEV)
    d_out = torch.zeros((t, kv * D), dtype=BF, device=DEV)
    qkv[-2 * n:], d_out[-2 * n:] = rand((2 * n, kv * 3 * D), 1), rand((2 * n, kv * D), 2)
    res = []
    for rows, k in ((t, docs), (2 * n, 2)):
        cu = torch.arange(k + 1, device=DEV, dtype=torch.int32) * n
        d = atp.attention_docs(cu)
        x, do = qkv[-rows:], d_out[-rows:]
        out, lse = torch.empty((rows, kv * D), dtype=BF, device=DEV), torch.empty((kv, rows),
                                                                                  device=DEV)
        dx = torch.empty_like(x)
        ws = torch.empty(atp.atp_attention_docs_workspace_bytes(rows, kv, 1), dtype=torch.uint8,
                         device=DEV)
        atp.atp_attention_docs_fwd(rows, kv, 1, d, x, out, lse)
        atp.atp_attention_docs_bwd(rows, kv, 1, d, x, out, lse, do, dx, ws)
        res.append((out[-2 * n:], lse[:, -2 * n:], dx[-2 * n:]))
    (o1, z1, g1), (o2, z2, g2) = res
    # the small call may split its loops: equal within the roundings of one result
    for a, b in ((o1, o2), (g1, g2)):
        assert (a.float() - b.float()).abs().max() <= 4 * R.H * b.float().abs().max()
    assert (z1 - z2).abs().max() <= 1e-4
    assert float(o1.float().abs().sum()) > 0


def test_gradients_of_billions_of_values():
    n = (1 << 31) + 12345
    g = torch.zeros(n, dtype=BF, device=DEV)
    at = torch.tensor([0, (1 << 30) - 1, 1 << 30, (1 << 31) - 1, 1 << 31, n - 1], device=DEV)
    g[at] = 3.0
    grads = atp.grad_list([g])
    total = torch.empty(1, dtype=torch.float64, device=DEV)
    ws = torch.empty(atp.atp_grad_workspace_bytes(grads), dtype=torch.uint8, device=DEV)
    atp.atp_grad_sq_sum(grads, total, ws)
    assert float(total) == 54.0
    norm = torch.empty(2, device=DEV)
    atp.atp_grad_clip(grads, [total], norm, max_norm=1.0)
    want = torch.tensor(3.0 / 54 ** 0.5).to(BF)
    assert (g[at].cpu() == want).all() and int((g != 0).sum()) == 6


def _bits(t):
    return t.contiguous().view({2: torch.int16, 4: torch.int32, 8: torch.int64}[t.element_size()])


@pytest.mark.parametrize("stream", [F32, BF])
def test_replays_have_the_bits_of_eager_steps(stream):
    """As above, but every value counts, also beside a NaN."""
    s = Step(400, 256, 1, 4, 300, 6, stream)
    eager = Step(400, 256, 1, 4, 300, 6, stream)
    s.batch([100, 50, 0, 200, 1, 9], 1)
    s.run()                                               # warm
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        s.run()
    for k, lens in enumerate(([9, 1, 200, 0, 50, 100], [400, 0, 0, 0, 0, 0], [1, 2, 3, 4, 5, 6],
                              [64, 64, 64, 64, 64, 80], [9, 1, 200, 0, 50, 100])):
        for b in (s, eager):
            b.batch(lens, 20 + k)
            for n in ("attn", "d_turned", "lse"):
                b.a[n].zero_()
        graph.replay()
        eager.run()
        torch.cuda.synchronize()
        got, want = s.outputs(), eager.outputs()
        for n in want:
            assert torch.equal(_bits(got[n]), _bits(want[n])), (lens, n)
        assert torch.isfinite(want["norm"]).all()
