// C ABI of the calls around the layers -- embedding, layer norm, gradient norm and
// clipping, attention within documents: argument checking and launches.
// Declarations and contracts: include/atp.h.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <new>

#include "../../include/atp.h"
#include "abi_common.h"
#include "errors.h"
#include "train_kernels.h"

namespace {

using namespace atp::abi;
using atp::set_error;

constexpr int64_t kMaxVocab = 1 << 24;
constexpr int32_t kMaxDocs = 1 << 16;
constexpr float kMaxCap = 0x1p100f;         // its reciprocal and base-2 score stay normal numbers

atp_status overlap(const char* a, const char* b) {
    return set_error(ATP_ERR_INVALID_ARGUMENT, "%s must not overlap %s", a, b);
}
// Row-major buffers of `rows` rows, as the overlap checks take them.
struct Buf {
    const void* p;
    int64_t bytes;
};
Buf buf(const void* p, int64_t rows, int64_t ld, int64_t cols, int64_t size = 2) {
    return Buf{p, p ? extent(rows, ld, cols, size) : 0};
}
Buf vec(const void* p, int64_t n, int64_t size = 4) { return Buf{p, p ? n * size : 0}; }
bool share(const Buf& a, const Buf& b) { return share_bytes(a.p, a.bytes, b.p, b.bytes); }

// What a call writes must share no memory with what it reads or writes elsewhere.
struct Named {
    Buf b;
    const char* name;
};
template <int N, int M>
atp_status check_apart(const Named (&out)[N], const Named (&in)[M]) {
    for (int i = 0; i < N; ++i) {
        for (int j = 0; j < M; ++j)
            if (share(out[i].b, in[j].b)) return overlap(out[i].name, in[j].name);
        for (int j = 0; j < i; ++j)
            if (share(out[i].b, out[j].b)) return overlap(out[i].name, out[j].name);
    }
    return ATP_OK;
}
template <int N>
atp_status check_parts_apart(const Named (&out)[N], int n, const float* const* parts,
                             int64_t tokens, const char* name) {
    for (int j = 0; j < n; ++j) {
        const Named part[] = {{vec(parts[j], 2 * tokens), name}};
        ATP_CHECK(check_apart(out, part));
    }
    return ATP_OK;
}

atp_status check_dtype(int32_t dtype, const char* name) {
    if (dtype != ATP_F32 && dtype != ATP_BF16)
        return set_error(ATP_ERR_INVALID_ARGUMENT, "%s %d is neither ATP_F32 nor ATP_BF16", name,
                         dtype);
    return ATP_OK;
}
int64_t size_of(int32_t dtype) { return dtype == ATP_F32 ? 4 : 2; }

// Row width: a multiple of 8, like every local column count.
atp_status check_cols(int64_t cols, int64_t most) {
    if (cols < 1) return set_error(ATP_ERR_INVALID_ARGUMENT, "cols %lld", (long long)cols);
    if (cols % 8 != 0)
        return set_error(ATP_ERR_UNSUPPORTED, "cols %lld is not a multiple of 8", (long long)cols);
    if (cols > most)
        return set_error(ATP_ERR_UNSUPPORTED, "cols %lld: at most %lld", (long long)cols,
                         (long long)most);
    return ATP_OK;
}

// A group's tables of fp32 values, or none for a group of one.
template <class T>
atp_status check_parts(int32_t red_size, const T* const* parts, const char* name) {
    if (red_size < 1) return set_error(ATP_ERR_INVALID_ARGUMENT, "red_size %d", red_size);
    if (red_size > ATP_MAX_GROUP)
        return set_error(ATP_ERR_UNSUPPORTED, "red_size %d: at most %d", red_size, ATP_MAX_GROUP);
    if (!parts) return set_error(ATP_ERR_INVALID_ARGUMENT, "%s is NULL", name);
    for (int j = 0; j < red_size; ++j)
        if (!parts[j]) return set_error(ATP_ERR_INVALID_ARGUMENT, "%s[%d] is NULL", name, j);
    return ATP_OK;
}

// ------------------------------------------------------------------ embedding
atp_status check_embedding(int64_t tokens, const int32_t* ids, int64_t vocab, int64_t off,
                           int64_t cols, float scale) {
    ATP_CHECK(check_tokens(tokens));
    if (vocab < 1 || off < 0)
        return set_error(ATP_ERR_INVALID_ARGUMENT, "vocab_loc %lld, vocab_off %lld",
                         (long long)vocab, (long long)off);
    if (vocab > kMaxVocab)
        return set_error(ATP_ERR_UNSUPPORTED, "vocab_loc %lld: at most 2^24", (long long)vocab);
    ATP_CHECK(check_cols(cols, kMaxLd));
    if (!isfinite(scale)) return set_error(ATP_ERR_INVALID_ARGUMENT, "scale must be finite");
    if (tokens > 0) ATP_CHECK(check_vector(ids, "ids"));
    return ATP_OK;
}

// ------------------------------------------------------------------ layer norm
atp_status check_norm(const atp_layer_norm* p) {
    if (!p) return set_error(ATP_ERR_INVALID_ARGUMENT, "norm is NULL");
    if (!(p->eps >= 0.f) || isinf(p->eps))
        return set_error(ATP_ERR_INVALID_ARGUMENT, "eps must be finite and not negative");
    ATP_CHECK(check_optional(p->weight, "weight"));
    return check_optional(p->bias, "bias");
}

struct NormSum {
    int64_t tokens, cols;
    int32_t dtype;
    const void* x; int64_t ldx;
    const void* add; int64_t ldadd;
    void* x_out; int64_t ldxo;
};
// x, add and x_out of the two calls that form the sum.
atp_status check_sum(const NormSum& s) {
    ATP_CHECK(check_tokens(s.tokens));
    ATP_CHECK(check_cols(s.cols, atp::kMaxNormCols));
    ATP_CHECK(check_dtype(s.dtype, "dtype"));
    if (!atp::layer_norm_fits(s.tokens, s.cols))
        return set_error(ATP_ERR_UNSUPPORTED, "%lld rows of %lld columns: 2^32 threads or more",
                         (long long)s.tokens, (long long)s.cols);
    ATP_CHECK(check_matrix(s.x, s.tokens, s.ldx, s.cols, "x"));
    if (!s.add != !s.x_out)
        return set_error(ATP_ERR_INVALID_ARGUMENT, "add and x_out go together");
    if (!s.add) return ATP_OK;
    ATP_CHECK(check_matrix(s.add, s.tokens, s.ldadd, s.cols, "add"));
    ATP_CHECK(check_matrix(s.x_out, s.tokens, s.ldxo, s.cols, "x_out"));
    const int64_t z = size_of(s.dtype);
    const Buf x = buf(s.x, s.tokens, s.ldx, s.cols, z);
    const Buf o = buf(s.x_out, s.tokens, s.ldxo, s.cols, z);
    if (!(s.x_out == s.x && s.ldxo == s.ldx) && share(x, o))
        return set_error(ATP_ERR_INVALID_ARGUMENT, "x_out must be x itself or not overlap it");
    if (share(o, buf(s.add, s.tokens, s.ldadd, s.cols))) return overlap("x_out", "add");
    return ATP_OK;
}
atp::LayerNormProblem problem(const NormSum& s) {
    atp::LayerNormProblem p = {};
    p.tokens = s.tokens;
    p.cols = s.cols;
    p.f32 = s.dtype == ATP_F32;
    p.x = s.x; p.ldx = s.ldx;
    p.add = bits(s.add); p.ldadd = s.ldadd;
    p.x_out = s.x_out; p.ldxo = s.ldxo;
    return p;
}

atp_status check_norm_bwd(int64_t tokens, int64_t cols, int32_t dtype, const atp_layer_norm* norm,
                          const void* x, int64_t ldx, const float* mean, const float* rstd,
                          const void* dy, int64_t lddy) {
    ATP_CHECK(check_tokens(tokens));
    ATP_CHECK(check_cols(cols, atp::kMaxNormCols));
    ATP_CHECK(check_dtype(dtype, "dtype"));
    ATP_CHECK(check_norm(norm));
    ATP_CHECK(check_matrix(x, tokens, ldx, cols, "x"));
    ATP_CHECK(check_matrix(dy, tokens, lddy, cols, "dy"));
    if (tokens > 0) {
        ATP_CHECK(check_vector(mean, "mean"));
        ATP_CHECK(check_vector(rstd, "rstd"));
    }
    return ATP_OK;
}
atp::LayerNormBwdProblem bwd_problem(int64_t tokens, int64_t cols, int32_t dtype,
                                     const atp_layer_norm* norm, const void* x, int64_t ldx,
                                     const float* mean, const float* rstd, const void* dy,
                                     int64_t lddy) {
    atp::LayerNormBwdProblem p = {};
    p.tokens = tokens;
    p.cols = cols;
    p.f32 = dtype == ATP_F32;
    p.x = x; p.ldx = ldx;
    p.weight = bits(norm->weight);
    p.mean = mean;
    p.rstd = rstd;
    p.dy = bits(dy); p.lddy = lddy;
    return p;
}

// ------------------------------------------------------------------ gradients
atp_status check_side(const void* p, int64_t rows, int64_t cols, int64_t ld, int32_t dtype, int i,
                      const char* name) {
    if (dtype != ATP_F32 && dtype != ATP_BF16)
        return set_error(ATP_ERR_INVALID_ARGUMENT, "gradient %d: %s_dtype %d", i, name, dtype);
    if (rows == 0 || cols == 0) return ATP_OK;
    if (!p) return set_error(ATP_ERR_INVALID_ARGUMENT, "gradient %d: %s is NULL", i, name);
    if (reinterpret_cast<uintptr_t>(p) % 16 != 0)
        return set_error(ATP_ERR_UNSUPPORTED, "gradient %d: %s is not 16-byte aligned", i, name);
    if (rows == 1) return ATP_OK;
    if (ld < cols)
        return set_error(ATP_ERR_INVALID_ARGUMENT, "gradient %d: ld_%s %lld < cols %lld", i, name,
                         (long long)ld, (long long)cols);
    if (ld != cols && (ld % 8 != 0 || ld > kMaxLd))
        return set_error(ATP_ERR_UNSUPPORTED,
                         "gradient %d: ld_%s %lld of rows with gaps is no multiple of 8 up to 4M",
                         i, name, (long long)ld);
    return ATP_OK;
}

// The list as the kernels take it; dst is looked at by the calls that write it.
atp_status check_grads(int32_t n, const atp_grad* g, bool with_dst) {
    if (n < 0) return set_error(ATP_ERR_INVALID_ARGUMENT, "n %d", n);
    if (n > 0 && !g) return set_error(ATP_ERR_INVALID_ARGUMENT, "grads is NULL");
    for (int i = 0; i < n; ++i) {
        const int64_t rows = g[i].rows, cols = g[i].cols;
        if (rows < 0 || cols < 0)
            return set_error(ATP_ERR_INVALID_ARGUMENT, "gradient %d: negative size", i);
        if (rows > 0x7fffffff || cols > (int64_t)1 << 40 ||
            (cols > 0 && rows > ((int64_t)1 << 40) / cols))
            return set_error(ATP_ERR_UNSUPPORTED, "gradient %d: more than 2^40 values", i);
        ATP_CHECK(check_side(g[i].src, rows, cols, g[i].ld_src, g[i].src_dtype, i, "src"));
        if (!with_dst) continue;
        ATP_CHECK(check_side(g[i].dst, rows, cols, g[i].ld_dst, g[i].dst_dtype, i, "dst"));
        // rows with gaps on one side are written with gaps on both
        if (rows > 1 && (g[i].ld_src != cols || g[i].ld_dst != cols) &&
            (g[i].ld_src % 8 != 0 || g[i].ld_dst % 8 != 0 || g[i].ld_src > kMaxLd ||
             g[i].ld_dst > kMaxLd))
            return set_error(ATP_ERR_UNSUPPORTED,
                             "gradient %d: leading dimensions of rows with gaps must be multiples "
                             "of 8 up to 4M", i);
        const bool same = g[i].dst == g[i].src && g[i].dst_dtype == g[i].src_dtype &&
                          (rows <= 1 || g[i].ld_dst == g[i].ld_src);
        if (!same && share(buf(g[i].src, rows, g[i].ld_src, cols, size_of(g[i].src_dtype)),
                           buf(g[i].dst, rows, g[i].ld_dst, cols, size_of(g[i].dst_dtype))))
            return set_error(ATP_ERR_INVALID_ARGUMENT,
                             "gradient %d: dst must be src itself or not overlap it", i);
    }
    return ATP_OK;
}
// atp_grad and the kernels' view hold the same fields.
struct Views {
    atp::GradView* v;
    explicit Views(int32_t n, const atp_grad* g)
        : v(n > kFew ? new (std::nothrow) atp::GradView[n] : few) {
        for (int i = 0; v && i < n; ++i)
            v[i] = atp::GradView{g[i].src, g[i].dst, g[i].rows, g[i].cols, g[i].ld_src, g[i].ld_dst,
                                 g[i].src_dtype == ATP_F32, g[i].dst_dtype == ATP_F32};
    }
    ~Views() {
        if (v != few) delete[] v;
    }
    Views(const Views&) = delete;
    Views& operator=(const Views&) = delete;
    static constexpr int kFew = 64;
    atp::GradView few[kFew];
};
double grad_bytes(int32_t n, const atp_grad* g, bool with_dst) {
    double b = 0;
    for (int i = 0; i < n; ++i)
        b += (double)g[i].rows * g[i].cols *
             (size_of(g[i].src_dtype) + (with_dst ? size_of(g[i].dst_dtype) : 0));
    return b;
}
atp_status check_scalar(const void* p, size_t align, const char* name) {
    if (!p) return set_error(ATP_ERR_INVALID_ARGUMENT, "%s is NULL", name);
    if (reinterpret_cast<uintptr_t>(p) % align != 0)
        return set_error(ATP_ERR_UNSUPPORTED, "%s is not %zu-byte aligned", name, align);
    return ATP_OK;
}

// ------------------------------------------------------------------ attention
atp_status check_docs(const atp_attention_docs* d, int64_t tokens, int32_t kv_heads,
                      int32_t group) {
    ATP_CHECK(check_tokens(tokens));
    ATP_CHECK(check_heads(kv_heads, group));
    if (!d) return set_error(ATP_ERR_INVALID_ARGUMENT, "docs is NULL");
    if (d->n_docs < 0) return set_error(ATP_ERR_INVALID_ARGUMENT, "n_docs %d", d->n_docs);
    if (d->n_docs > kMaxDocs)
        return set_error(ATP_ERR_UNSUPPORTED, "n_docs %d: at most %d", d->n_docs, kMaxDocs);
    if (!(d->cap >= 0.f) || isinf(d->cap))
        return set_error(ATP_ERR_INVALID_ARGUMENT, "cap must be finite and not negative");
    if (d->cap > kMaxCap) return set_error(ATP_ERR_UNSUPPORTED, "cap %g: at most 2^100", d->cap);
    if (!atp::fits_launch((tokens / 64 + d->n_docs) * kv_heads * group, 256))
        return set_error(ATP_ERR_UNSUPPORTED, "%lld tokens of %d documents and %lld heads: 2^24 "
                         "tiles or more", (long long)tokens, d->n_docs,
                         (long long)kv_heads * group);
    if (d->n_docs == 0) return ATP_OK;
    ATP_CHECK(check_vector(d->cu_docs, "cu_docs"));
    ATP_CHECK(check_optional(d->prefix, "prefix"));
    return check_optional(d->slopes, "slopes");
}
template <int N>
atp_status check_lists_apart(const Named (&out)[N], const atp_attention_docs* d, int64_t heads) {
    const Named lists[] = {{vec(d->cu_docs, d->n_docs + (int64_t)1), "cu_docs"},
                           {vec(d->prefix, d->n_docs), "prefix"},
                           {vec(d->slopes, heads), "slopes"}};
    return check_apart(out, lists);
}
atp::DocsView view(const atp_attention_docs* d) {
    return atp::DocsView{d->cu_docs, d->prefix, d->slopes, d->n_docs, d->cap};
}

}  // namespace

extern "C" {

atp_status atp_embedding_fwd(int64_t tokens, const int32_t* ids, int64_t vocab_loc,
                             int64_t vocab_off, int64_t cols, const void* table, int64_t ld_table,
                             float scale, void* out, int32_t out_dtype, int64_t ld_out,
                             void* stream) {
    ATP_CHECK(check_embedding(tokens, ids, vocab_loc, vocab_off, cols, scale));
    ATP_CHECK(check_dtype(out_dtype, "out_dtype"));
    ATP_CHECK(check_matrix(table, vocab_loc, ld_table, cols, "table"));
    ATP_CHECK(check_matrix(out, tokens, ld_out, cols, "out"));
    if (tokens == 0) return ATP_OK;
    if (!atp::embedding_fits(tokens, cols))
        return set_error(ATP_ERR_UNSUPPORTED, "%lld tokens of %lld columns: 2^37 values or more",
                         (long long)tokens, (long long)cols);
    const int64_t z = size_of(out_dtype);
    const Named to[] = {{buf(out, tokens, ld_out, cols, z), "out"}};
    const Named from[] = {{buf(table, vocab_loc, ld_table, cols), "table"},
                          {vec(ids, tokens), "ids"}};
    ATP_CHECK(check_apart(to, from));
    atp::EmbeddingProblem p = {};
    p.ids = ids;
    p.tokens = tokens;
    p.vocab = vocab_loc;
    p.off = vocab_off;
    p.cols = cols;
    p.table = bits(table); p.ldt = ld_table;
    p.scale = scale;
    p.out = out; p.ldo = ld_out;
    p.out_f32 = out_dtype == ATP_F32;
    const double el = (double)tokens * cols;
    hipStream_t s = stream_of(stream);
    return run_timed("embedding_fwd", el, el * (2 + z), s,
                     [&] { return atp::launch_embedding(p, s); });
}

size_t atp_embedding_workspace_bytes(int64_t tokens, int64_t vocab_loc, int64_t cols) {
    if (tokens < 0 || tokens > kMaxTokens || vocab_loc < 1 || vocab_loc > kMaxVocab || cols < 8 ||
        cols % 8 != 0 || cols > kMaxLd)
        return 0;
    return (size_t)atp::embedding_ws_bytes(tokens, vocab_loc, cols);
}

atp_status atp_embedding_bwd(int64_t tokens, const int32_t* ids, int64_t vocab_loc,
                             int64_t vocab_off, int64_t cols, const void* dy, int64_t ld_dy,
                             float scale, float* dtable, int64_t ld_dtable, int32_t accumulate,
                             void* workspace, size_t ws_bytes, void* stream) {
    ATP_CHECK(check_embedding(tokens, ids, vocab_loc, vocab_off, cols, scale));
    if (accumulate != 0 && accumulate != 1)
        return set_error(ATP_ERR_INVALID_ARGUMENT, "accumulate %d is neither 0 nor 1", accumulate);
    ATP_CHECK(check_matrix(dy, tokens, ld_dy, cols, "dy"));
    ATP_CHECK(check_matrix(dtable, vocab_loc, ld_dtable, cols, "dtable"));
    const size_t need = atp_embedding_workspace_bytes(tokens, vocab_loc, cols);
    ATP_CHECK(check_workspace(workspace, ws_bytes, need));
    const Named out[] = {{buf(dtable, vocab_loc, ld_dtable, cols, 4), "dtable"},
                         {vec(workspace, (int64_t)need, 1), "workspace"}};
    const Named in[] = {{buf(dy, tokens, ld_dy, cols), "dy"}, {vec(ids, tokens), "ids"}};
    ATP_CHECK(check_apart(out, in));
    atp::EmbeddingBwdProblem p = {};
    p.ids = ids;
    p.tokens = tokens;
    p.vocab = vocab_loc;
    p.off = vocab_off;
    p.cols = cols;
    p.dy = bits(dy); p.lddy = ld_dy;
    p.scale = scale;
    p.dtable = dtable; p.ldt = ld_dtable;
    p.accumulate = accumulate != 0;
    p.ws = workspace;
    const double el = (double)tokens * cols;
    hipStream_t s = stream_of(stream);
    return run_timed("embedding_bwd", 2.0 * el, 2.0 * el + 4.0 * vocab_loc * cols, s,
                     [&] { return atp::launch_embedding_bwd(p, s); });
}

atp_status atp_layer_norm_stats(int64_t tokens, int64_t cols, int32_t dtype, const void* x,
                                int64_t ldx, const void* add, int64_t ld_add, void* x_out,
                                int64_t ld_xout, float* stats, void* stream) {
    const NormSum sum{tokens, cols, dtype, x, ldx, add, ld_add, x_out, ld_xout};
    ATP_CHECK(check_sum(sum));
    if (tokens == 0) return ATP_OK;
    ATP_CHECK(check_vector(stats, "stats"));
    const int64_t z = size_of(dtype);
    const Named out[] = {{vec(stats, 2 * tokens), "stats"}};
    const Named in[] = {{buf(x, tokens, ldx, cols, z), "x"},
                        {buf(add, tokens, ld_add, cols), "add"},
                        {buf(x_out, tokens, ld_xout, cols, z), "x_out"}};
    ATP_CHECK(check_apart(out, in));
    atp::LayerNormProblem p = problem(sum);
    p.stats_out = stats;
    const double el = (double)tokens * cols;
    hipStream_t s = stream_of(stream);
    return run_timed("layer_norm_stats", 5.0 * el,
                     el * (z + (add ? 2 + z : 0)), s,
                     [&] { return atp::launch_layer_norm(p, s); });
}

atp_status atp_layer_norm_fwd(int64_t tokens, int64_t cols, int32_t dtype,
                              const atp_layer_norm* norm, const void* x, int64_t ldx,
                              const void* add, int64_t ld_add, void* x_out, int64_t ld_xout,
                              int32_t red_size, const float* const* stats, void* y, int64_t ld_y,
                              float* mean, float* rstd, void* stream) {
    const NormSum sum{tokens, cols, dtype, x, ldx, add, ld_add, x_out, ld_xout};
    ATP_CHECK(check_sum(sum));
    ATP_CHECK(check_norm(norm));
    ATP_CHECK(check_matrix(y, tokens, ld_y, cols, "y"));
    if (red_size != 1 || stats) {
        ATP_CHECK(check_parts(red_size, stats, "stats"));
        if (add)
            return set_error(ATP_ERR_INVALID_ARGUMENT,
                             "add belongs to atp_layer_norm_stats where stats are given");
    }
    if (tokens == 0) return ATP_OK;
    ATP_CHECK(check_vector(mean, "mean"));
    ATP_CHECK(check_vector(rstd, "rstd"));
    const int64_t z = size_of(dtype);
    const Named sum_out[] = {{buf(x_out, tokens, ld_xout, cols, z), "x_out"}};
    const Named params[] = {{vec(norm->weight, cols, 2), "weight"},
                            {vec(norm->bias, cols, 2), "bias"}};
    const Named out[] = {{buf(y, tokens, ld_y, cols), "y"}, {vec(mean, tokens), "mean"},
                         {vec(rstd, tokens), "rstd"}};
    const Named in[] = {{buf(x, tokens, ldx, cols, z), "x"},
                        {buf(add, tokens, ld_add, cols), "add"}};
    ATP_CHECK(check_apart(out, in));
    ATP_CHECK(check_apart(out, params));
    ATP_CHECK(check_apart(out, sum_out));
    ATP_CHECK(check_apart(sum_out, params));
    ATP_CHECK(check_parts_apart(out, stats ? red_size : 0, stats, tokens, "stats"));
    atp::LayerNormProblem p = problem(sum);
    p.weight = bits(norm->weight);
    p.bias = bits(norm->bias);
    p.eps = norm->eps;
    p.nparts = stats ? red_size : 0;
    for (int j = 0; j < p.nparts; ++j) p.parts[j] = stats[j];
    p.y = bits(y); p.ldy = ld_y;
    p.mean = mean;
    p.rstd = rstd;
    const double el = (double)tokens * cols;
    hipStream_t s = stream_of(stream);
    return run_timed("layer_norm_fwd", 8.0 * el, el * (2 + z + (add ? 2 + z : 0)), s,
                     [&] { return atp::launch_layer_norm(p, s); });
}

atp_status atp_layer_norm_bwd_sums(int64_t tokens, int64_t cols, int32_t dtype,
                                   const atp_layer_norm* norm, const void* x, int64_t ldx,
                                   const float* mean, const float* rstd, const void* dy,
                                   int64_t ld_dy, float* sums, void* stream) {
    ATP_CHECK(check_norm_bwd(tokens, cols, dtype, norm, x, ldx, mean, rstd, dy, ld_dy));
    if (tokens == 0) return ATP_OK;
    ATP_CHECK(check_vector(sums, "sums"));
    const Named out[] = {{vec(sums, 2 * tokens), "sums"}};
    const Named in[] = {{buf(x, tokens, ldx, cols, size_of(dtype)), "x"},
                        {buf(dy, tokens, ld_dy, cols), "dy"}, {vec(mean, tokens), "mean"},
                        {vec(rstd, tokens), "rstd"}, {vec(norm->weight, cols, 2), "weight"}};
    ATP_CHECK(check_apart(out, in));
    atp::LayerNormBwdProblem p =
        bwd_problem(tokens, cols, dtype, norm, x, ldx, mean, rstd, dy, ld_dy);
    p.sums_out = sums;
    const double el = (double)tokens * cols;
    hipStream_t s = stream_of(stream);
    return run_timed("layer_norm_bwd_sums", 6.0 * el, el * (2 + size_of(dtype)), s,
                     [&] { return atp::launch_layer_norm_bwd(p, s); });
}

size_t atp_layer_norm_workspace_bytes(int64_t tokens, int64_t cols) {
    if (tokens < 0 || tokens > kMaxTokens || cols < 8 || cols % 8 != 0 ||
        cols > atp::kMaxNormCols)
        return 0;
    return sizeof(float) * (size_t)atp::layer_norm_ws_floats(tokens, cols);
}

atp_status atp_layer_norm_bwd(int64_t tokens, int64_t cols, int32_t dtype,
                              const atp_layer_norm* norm, const void* x, int64_t ldx,
                              const float* mean, const float* rstd, const void* dy, int64_t ld_dy,
                              const void* d_res, int64_t ld_dres, int32_t red_size,
                              const float* const* sums, void* dx, int64_t ld_dx, void* d_add,
                              int64_t ld_dadd, float* dweight, float* dbias, void* workspace,
                              size_t ws_bytes, void* stream) {
    ATP_CHECK(check_norm_bwd(tokens, cols, dtype, norm, x, ldx, mean, rstd, dy, ld_dy));
    ATP_CHECK(check_matrix(dx, tokens, ld_dx, cols, "dx"));
    if (d_res) ATP_CHECK(check_matrix(d_res, tokens, ld_dres, cols, "d_res"));
    if (d_add) ATP_CHECK(check_matrix(d_add, tokens, ld_dadd, cols, "d_add"));
    if (red_size != 1 || sums) ATP_CHECK(check_parts(red_size, sums, "sums"));
    ATP_CHECK(check_optional(dweight, "dweight"));
    ATP_CHECK(check_optional(dbias, "dbias"));
    const bool weights = dweight || dbias;
    const size_t need = weights ? atp_layer_norm_workspace_bytes(tokens, cols) : 0;
    ATP_CHECK(check_workspace(workspace, ws_bytes, need));
    if (tokens == 0 && !weights) return ATP_OK;
    const int64_t z = size_of(dtype);
    const Buf bres = buf(d_res, tokens, ld_dres, cols, z), bdx = buf(dx, tokens, ld_dx, cols, z);
    const bool in_place = dx == d_res && ld_dx == ld_dres;
    if (!in_place && share(bdx, bres))
        return set_error(ATP_ERR_INVALID_ARGUMENT, "dx must be d_res itself or not overlap it");
    const Named out[] = {{bdx, "dx"}, {buf(d_add, tokens, ld_dadd, cols), "d_add"},
                         {vec(dweight, cols), "dweight"}, {vec(dbias, cols), "dbias"},
                         {vec(weights ? workspace : nullptr, (int64_t)need, 1), "workspace"}};
    const Named in[] = {{buf(x, tokens, ldx, cols, z), "x"}, {buf(dy, tokens, ld_dy, cols), "dy"},
                        {in_place ? Buf{} : bres, "d_res"}, {vec(mean, tokens), "mean"},
                        {vec(rstd, tokens), "rstd"}, {vec(norm->weight, cols, 2), "weight"}};
    ATP_CHECK(check_apart(out, in));
    ATP_CHECK(check_parts_apart(out, sums ? red_size : 0, sums, tokens, "sums"));
    atp::LayerNormBwdProblem p =
        bwd_problem(tokens, cols, dtype, norm, x, ldx, mean, rstd, dy, ld_dy);
    p.nparts = sums ? red_size : 0;
    for (int j = 0; j < p.nparts; ++j) p.parts[j] = sums[j];
    p.dres = d_res; p.lddres = ld_dres;
    p.dx = dx; p.lddx = ld_dx;
    p.dadd = bits(d_add); p.lddadd = ld_dadd;
    p.dw = dweight;
    p.db = dbias;
    p.ws = static_cast<float*>(workspace);
    const double el = (double)tokens * cols;
    hipStream_t s = stream_of(stream);
    return run_timed("layer_norm_bwd", 14.0 * el,
                     el * (2 + 2 * z + (d_res ? z : 0) + (d_add ? 2 : 0)), s,
                     [&] { return atp::launch_layer_norm_bwd(p, s); });
}

size_t atp_grad_workspace_bytes(int32_t n, const atp_grad* grads) {
    if (check_grads(n, grads, false) != ATP_OK) return 0;
    const Views v(n, grads);
    return v.v ? sizeof(double) * (size_t)atp::grad_sum_blocks(n, v.v) : 0;
}

atp_status atp_grad_sq_sum(int32_t n, const atp_grad* grads, double* sum, void* workspace,
                           size_t ws_bytes, void* stream) {
    ATP_CHECK(check_grads(n, grads, false));
    ATP_CHECK(check_scalar(sum, 8, "sum"));
    const Views v(n, grads);
    if (!v.v) return set_error(ATP_ERR_DEVICE, "no memory for %d gradients", n);
    ATP_CHECK(check_workspace(workspace, ws_bytes,
                              sizeof(double) * (size_t)atp::grad_sum_blocks(n, v.v)));
    const double b = grad_bytes(n, grads, false);
    hipStream_t s = stream_of(stream);
    return run_timed("grad_sq_sum", b / 2, b, s, [&] {
        return atp::launch_grad_sq_sum(n, v.v, sum, static_cast<double*>(workspace), s);
    });
}

atp_status atp_grad_clip(int32_t n, const atp_grad* grads, int32_t red_size,
                         const double* const* sums, float scale, float max_norm, float* norm,
                         void* stream) {
    ATP_CHECK(check_grads(n, grads, true));
    ATP_CHECK(check_parts(red_size, sums, "sums"));
    for (int j = 0; j < red_size; ++j) ATP_CHECK(check_scalar(sums[j], 8, "sums"));
    if (!(scale > 0.f) || isinf(scale))
        return set_error(ATP_ERR_INVALID_ARGUMENT, "scale must be finite and positive");
    if (!(max_norm > 0.f))
        return set_error(ATP_ERR_INVALID_ARGUMENT, "max_norm must be positive");
    ATP_CHECK(check_scalar(norm, 8, "norm"));
    const Views v(n, grads);
    if (!v.v) return set_error(ATP_ERR_DEVICE, "no memory for %d gradients", n);
    const double b = grad_bytes(n, grads, true);
    hipStream_t s = stream_of(stream);
    return run_timed("grad_clip", b / 6, b, s, [&] {
        return atp::launch_grad_clip(n, v.v, red_size, sums, scale, max_norm, norm, s);
    });
}

atp_status atp_attention_docs_fwd(int64_t tokens, int32_t kv_heads, int32_t group,
                                  const atp_attention_docs* docs, const void* qkv, int64_t ld_qkv,
                                  void* out, int64_t ld_out, float* lse, void* stream) {
    ATP_CHECK(check_docs(docs, tokens, kv_heads, group));
    const int64_t cols = (int64_t)kv_heads * (group + 2) * 128;
    const int64_t ocols = (int64_t)kv_heads * group * 128;
    ATP_CHECK(check_matrix(qkv, tokens, ld_qkv, cols, "qkv"));
    ATP_CHECK(check_matrix(out, tokens, ld_out, ocols, "out"));
    if (tokens == 0 || docs->n_docs == 0) return ATP_OK;
    ATP_CHECK(check_vector(lse, "lse"));
    const Named to[] = {{buf(out, tokens, ld_out, ocols), "out"},
                        {vec(lse, tokens * kv_heads * group), "lse"}};
    const Named from[] = {{buf(qkv, tokens, ld_qkv, cols), "qkv"}};
    ATP_CHECK(check_apart(to, from));
    ATP_CHECK(check_lists_apart(to, docs, (int64_t)kv_heads * group));
    atp::DocsAttentionProblem p = {};
    p.docs = view(docs);
    p.tokens = tokens;
    p.kv_heads = kv_heads;
    p.group = group;
    p.qkv = bits(qkv); p.ldq = ld_qkv;
    p.out = bits(out); p.ldo = ld_out;
    p.lse = lse;
    hipStream_t s = stream_of(stream);
    // the documents' lengths are on the device: what the rows take alone
    return run_timed("attention_docs_fwd", 0.0, 2.0 * tokens * (cols + ocols), s,
                     [&] { return atp::launch_docs_attention(p, s); });
}

size_t atp_attention_docs_workspace_bytes(int64_t tokens, int32_t kv_heads, int32_t group) {
    if (tokens < 0 || tokens > kMaxTokens || kv_heads < 1 || group < 1 ||
        group > ATP_MAX_QUERY_GROUP || (int64_t)kv_heads * (group + 2) * 128 > kMaxLd)
        return 0;
    return sizeof(float) * (size_t)atp::docs_attention_ws_floats(tokens, kv_heads, group);
}

atp_status atp_attention_docs_bwd(int64_t tokens, int32_t kv_heads, int32_t group,
                                  const atp_attention_docs* docs, const void* qkv, int64_t ld_qkv,
                                  const void* out, int64_t ld_out, const float* lse,
                                  const void* d_out, int64_t ld_dout, void* d_qkv, int64_t ld_dqkv,
                                  void* workspace, size_t ws_bytes, void* stream) {
    ATP_CHECK(check_docs(docs, tokens, kv_heads, group));
    const int64_t cols = (int64_t)kv_heads * (group + 2) * 128;
    const int64_t ocols = (int64_t)kv_heads * group * 128;
    ATP_CHECK(check_matrix(qkv, tokens, ld_qkv, cols, "qkv"));
    ATP_CHECK(check_matrix(out, tokens, ld_out, ocols, "out"));
    ATP_CHECK(check_matrix(d_out, tokens, ld_dout, ocols, "d_out"));
    ATP_CHECK(check_matrix(d_qkv, tokens, ld_dqkv, cols, "d_qkv"));
    if (tokens == 0 || docs->n_docs == 0) return ATP_OK;
    ATP_CHECK(check_vector(lse, "lse"));
    const size_t need = atp_attention_docs_workspace_bytes(tokens, kv_heads, group);
    ATP_CHECK(check_workspace(workspace, ws_bytes, need));
    const Named to[] = {{buf(d_qkv, tokens, ld_dqkv, cols), "d_qkv"},
                        {vec(workspace, (int64_t)need, 1), "workspace"}};
    const Named from[] = {{buf(qkv, tokens, ld_qkv, cols), "qkv"},
                          {buf(out, tokens, ld_out, ocols), "out"},
                          {buf(d_out, tokens, ld_dout, ocols), "d_out"},
                          {vec(lse, tokens * kv_heads * group), "lse"}};
    ATP_CHECK(check_apart(to, from));
    ATP_CHECK(check_lists_apart(to, docs, (int64_t)kv_heads * group));
    atp::DocsAttentionBwdProblem p = {};
    p.docs = view(docs);
    p.tokens = tokens;
    p.kv_heads = kv_heads;
    p.group = group;
    p.qkv = bits(qkv); p.ldq = ld_qkv;
    p.out = bits(out); p.ldo = ld_out;
    p.lse = lse;
    p.dout = bits(d_out); p.lddo = ld_dout;
    p.dqkv = bits(d_qkv); p.lddq = ld_dqkv;
    p.ws = static_cast<float*>(workspace);
    hipStream_t s = stream_of(stream);
    return run_timed("attention_docs_bwd", 0.0, 4.0 * tokens * (cols + ocols), s,
                     [&] { return atp::launch_docs_attention_bwd(p, s); });
}

}  // extern "C"
