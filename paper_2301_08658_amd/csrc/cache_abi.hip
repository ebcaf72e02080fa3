// C ABI of the position, cache and cached-attention calls: argument checking and
// launches.  Declarations and contracts: include/atp.h.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/atp.h"
#include "abi_common.h"
#include "cache_kernels.h"
#include "errors.h"

namespace {

using atp::set_error;
using atp::abi::check_matrix;
using atp::abi::check_vector;
using atp::abi::run_timed;

#define ATP_CHECK(expr)                                   \
    do {                                                  \
        atp_status _s = (expr);                           \
        if (_s != ATP_OK) return _s;                      \
    } while (0)

constexpr int64_t kMaxTokens = 1 << 24;
constexpr int64_t kMaxPlaces = 1 << 30;    // tokens that a table row can hold
constexpr int32_t kMaxPool = 1 << 28;
constexpr int32_t kMaxCopies = 1 << 23;    // workgroups of 256 threads in a row of a grid
constexpr int32_t kMaxSeqs = 1 << 16;
constexpr int64_t kMaxLd = 1 << 22;

// Bytes [0, extent) that a matrix of these rows takes from its first element.
int64_t extent(int64_t rows, int64_t ld, int64_t cols) {
    return rows > 0 ? ((rows - 1) * ld + cols) * 2 : 0;
}
bool share_bytes(const void* a, int64_t na, const void* b, int64_t nb) {
    const uintptr_t a0 = reinterpret_cast<uintptr_t>(a), b0 = reinterpret_cast<uintptr_t>(b);
    return na > 0 && nb > 0 && a0 < b0 + (uintptr_t)nb && b0 < a0 + (uintptr_t)na;
}

atp_status check_heads(int64_t kv_heads, int32_t group) {
    if (kv_heads < 1 || group < 1)
        return set_error(ATP_ERR_INVALID_ARGUMENT, "kv_heads %lld and group %d must be positive",
                         (long long)kv_heads, group);
    if (group > ATP_MAX_QUERY_GROUP)
        return set_error(ATP_ERR_UNSUPPORTED, "group %d: at most %d query heads per key head",
                         group, ATP_MAX_QUERY_GROUP);
    if (kv_heads * (group + 2) * atp::kHead > kMaxLd)
        return set_error(ATP_ERR_UNSUPPORTED, "%lld heads of group %d: rows above 4M elements",
                         (long long)kv_heads, group);
    return ATP_OK;
}

atp_status check_tokens(int64_t tokens) {
    if (tokens < 0) return set_error(ATP_ERR_INVALID_ARGUMENT, "negative number of tokens");
    if (tokens > kMaxTokens)
        return set_error(ATP_ERR_UNSUPPORTED, "%lld tokens: at most 2^24", (long long)tokens);
    return ATP_OK;
}

// Aligned like every vector; NULL allowed.
atp_status check_optional(const void* p, const char* name) {
    return p ? check_vector(p, name) : ATP_OK;
}

atp_status check_params(const atp_qk_norm_rope* p) {
    if (!p) return set_error(ATP_ERR_INVALID_ARGUMENT, "params is NULL");
    if (p->norm != 0 && p->norm != 1)
        return set_error(ATP_ERR_INVALID_ARGUMENT, "norm %d is neither 0 nor 1", p->norm);
    if (p->interleaved != 0 && p->interleaved != 1)
        return set_error(ATP_ERR_INVALID_ARGUMENT, "interleaved %d is neither 0 nor 1",
                         p->interleaved);
    if (!(p->eps >= 0.f) || isinf(p->eps))
        return set_error(ATP_ERR_INVALID_ARGUMENT, "eps must be finite and not negative");
    if (!p->norm && (p->q_weight || p->k_weight))
        return set_error(ATP_ERR_INVALID_ARGUMENT, "norm weights without norm");
    if (p->rotary_dims < 0 || p->rotary_dims > atp::kHead)
        return set_error(ATP_ERR_INVALID_ARGUMENT, "rotary_dims %d outside [0, %d]",
                         p->rotary_dims, atp::kHead);
    if (p->rotary_dims % 8 != 0)
        return set_error(ATP_ERR_UNSUPPORTED, "rotary_dims %d is not a multiple of 8",
                         p->rotary_dims);
    if (p->rotary_dims > 0) ATP_CHECK(check_vector(p->inv_freq, "inv_freq"));
    ATP_CHECK(check_optional(p->q_weight, "q_weight"));
    return check_optional(p->k_weight, "k_weight");
}

atp::NormRope norm_rope(const atp_qk_norm_rope* p, const int32_t* positions) {
    atp::NormRope f;
    f.qw = static_cast<const uint16_t*>(p->q_weight);
    f.kw = static_cast<const uint16_t*>(p->k_weight);
    f.inv_freq = p->inv_freq;
    f.pos = positions;
    f.eps = p->eps;
    f.norm = p->norm != 0;
    f.interleaved = p->interleaved != 0;
    f.rot = p->rotary_dims;
    return f;
}

atp_status check_page_size(int32_t page) {
    if (page < 1) return set_error(ATP_ERR_INVALID_ARGUMENT, "page_size %d", page);
    if (page < 16 || page > 1024 || (page & (page - 1)) != 0)
        return set_error(ATP_ERR_UNSUPPORTED, "page_size %d is not a power of two in [16, 1024]",
                         page);
    return ATP_OK;
}

int shift_of(int32_t page) { return __builtin_ctz((unsigned)page); }

atp_status check_pool(int32_t n_pages, int32_t page) {
    if (n_pages < 1) return set_error(ATP_ERR_INVALID_ARGUMENT, "n_pages %d", n_pages);
    if (n_pages > kMaxPool)
        return set_error(ATP_ERR_UNSUPPORTED, "n_pages %d: at most 2^28", n_pages);
    return check_page_size(page);
}

atp_status check_cache(const atp_kv_cache* c) {
    if (!c) return set_error(ATP_ERR_INVALID_ARGUMENT, "cache is NULL");
    ATP_CHECK(check_pool(c->n_pages, c->page_size));
    ATP_CHECK(check_heads(c->kv_heads, 1));
    return check_vector(c->pages, "cache pages");
}

int64_t cache_bytes(const atp_kv_cache* c) {
    return (int64_t)c->n_pages * 2 * c->kv_heads * c->page_size * atp::kHead * 2;
}

// cu_needed, ctx_needed: the call reads the new tokens' rows / the lengths.
atp_status check_batch(const atp_kv_batch* b, int32_t page, bool ctx_needed, bool cu_needed) {
    if (!b) return set_error(ATP_ERR_INVALID_ARGUMENT, "batch is NULL");
    if (b->n_seqs < 0) return set_error(ATP_ERR_INVALID_ARGUMENT, "n_seqs %d", b->n_seqs);
    if (b->n_seqs > kMaxSeqs)
        return set_error(ATP_ERR_UNSUPPORTED, "n_seqs %d: at most %d", b->n_seqs, kMaxSeqs);
    if (b->max_pages < 1) return set_error(ATP_ERR_INVALID_ARGUMENT, "max_pages %d", b->max_pages);
    if ((int64_t)b->max_pages * page > kMaxPlaces)
        return set_error(ATP_ERR_UNSUPPORTED, "max_pages %d of %d tokens: at most 2^30 tokens",
                         b->max_pages, page);
    if (b->ld_table < b->max_pages)
        return set_error(ATP_ERR_INVALID_ARGUMENT, "ld_table %lld < max_pages %d",
                         (long long)b->ld_table, b->max_pages);
    if (b->n_seqs == 0) return ATP_OK;
    ATP_CHECK(check_vector(b->table, "table"));
    if (ctx_needed) ATP_CHECK(check_vector(b->ctx, "ctx"));
    if (cu_needed) ATP_CHECK(check_vector(b->cu_new, "cu_new"));
    return ATP_OK;
}

atp::CacheView view(const atp_kv_cache* c) {
    return atp::CacheView{static_cast<uint16_t*>(c->pages), c->n_pages, c->kv_heads,
                          shift_of(c->page_size)};
}
atp::BatchView view(const atp_kv_batch* b) {
    return atp::BatchView{b->table, b->ld_table, b->max_pages, b->n_seqs, b->ctx, b->cu_new};
}

atp_status check_workspace(const void* ws, size_t have, size_t need) {
    if (need == 0) return ATP_OK;
    ATP_CHECK(check_vector(ws, "workspace"));
    if (have < need)
        return set_error(ATP_ERR_INVALID_ARGUMENT, "workspace of %zu bytes: needs %zu", have, need);
    return ATP_OK;
}

const uint16_t* bits(const void* p) { return static_cast<const uint16_t*>(p); }
uint16_t* bits(void* p) { return static_cast<uint16_t*>(p); }
hipStream_t stream_of(void* s) { return static_cast<hipStream_t>(s); }

// A training call's sizes: rows and row width of its blocks.
atp_status check_block(int64_t batch, int64_t seq, int32_t kv_heads, int32_t group, int64_t* T,
                       int64_t* cols) {
    if (batch < 0 || seq < 0) return set_error(ATP_ERR_INVALID_ARGUMENT, "negative batch or seq");
    ATP_CHECK(check_heads(kv_heads, group));
    if (batch > kMaxTokens || seq > kMaxTokens)
        return set_error(ATP_ERR_UNSUPPORTED, "batch and seq must be at most 2^24");
    ATP_CHECK(check_tokens(batch * seq));
    *T = batch * seq;
    *cols = (int64_t)kv_heads * (group + 2) * atp::kHead;
    return ATP_OK;
}

}  // namespace

extern "C" {

atp_status atp_qk_norm_rope_fwd(int64_t batch, int64_t seq, int32_t kv_heads, int32_t group,
                                const atp_qk_norm_rope* params, const int32_t* positions,
                                const void* qkv, int64_t ld_qkv, void* out, int64_t ld_out,
                                void* stream) {
    int64_t T, cols;
    ATP_CHECK(check_block(batch, seq, kv_heads, group, &T, &cols));
    ATP_CHECK(check_params(params));
    ATP_CHECK(check_matrix(qkv, T, ld_qkv, cols, "qkv"));
    ATP_CHECK(check_matrix(out, T, ld_out, cols, "out"));
    ATP_CHECK(check_optional(positions, "positions"));
    if (T == 0) return ATP_OK;
    if (!(out == qkv && ld_out == ld_qkv) &&
        share_bytes(qkv, extent(T, ld_qkv, cols), out, extent(T, ld_out, cols)))
        return set_error(ATP_ERR_INVALID_ARGUMENT, "out must be qkv itself or not overlap it");
    atp::NormRopeProblem p = {};
    p.f = norm_rope(params, positions);
    p.x = bits(qkv); p.ldx = ld_qkv;
    p.y = bits(out); p.ldy = ld_out;
    p.tokens = T;
    p.seq = seq;
    p.kv_heads = kv_heads;
    p.group = group;
    const double heads = (double)T * kv_heads * (out == qkv ? group + 1 : group + 2);
    hipStream_t s = stream_of(stream);
    return run_timed("qk_norm_rope_fwd", 8.0 * heads * atp::kHead, 4.0 * heads * atp::kHead, s,
                     [&] { return atp::launch_norm_rope(p, s); });
}

size_t atp_qk_norm_rope_workspace_bytes(int64_t tokens) {
    return tokens < 0 ? 0 : sizeof(float) * (size_t)atp::norm_rope_ws_floats(tokens);
}

atp_status atp_qk_norm_rope_bwd(int64_t batch, int64_t seq, int32_t kv_heads, int32_t group,
                                const atp_qk_norm_rope* params, const int32_t* positions,
                                const void* qkv, int64_t ld_qkv, const void* d_out,
                                int64_t ld_dout, void* d_qkv, int64_t ld_dqkv, float* dq_weight,
                                float* dk_weight, void* workspace, size_t ws_bytes, void* stream) {
    int64_t T, cols;
    ATP_CHECK(check_block(batch, seq, kv_heads, group, &T, &cols));
    ATP_CHECK(check_params(params));
    ATP_CHECK(check_matrix(qkv, T, ld_qkv, cols, "qkv"));
    ATP_CHECK(check_matrix(d_out, T, ld_dout, cols, "d_out"));
    ATP_CHECK(check_matrix(d_qkv, T, ld_dqkv, cols, "d_qkv"));
    ATP_CHECK(check_optional(positions, "positions"));
    const bool weights = dq_weight || dk_weight;
    if (weights && !params->norm)
        return set_error(ATP_ERR_INVALID_ARGUMENT, "weight gradients without norm");
    ATP_CHECK(check_optional(dq_weight, "dq_weight"));
    ATP_CHECK(check_optional(dk_weight, "dk_weight"));
    if (T == 0 && !weights) return ATP_OK;
    if (weights)
        ATP_CHECK(check_workspace(workspace, ws_bytes, atp_qk_norm_rope_workspace_bytes(T)));
    const int64_t nd = extent(T, ld_dqkv, cols);
    if (share_bytes(d_qkv, nd, qkv, extent(T, ld_qkv, cols)))
        return set_error(ATP_ERR_INVALID_ARGUMENT, "d_qkv must not overlap qkv");
    if (!(d_qkv == d_out && ld_dqkv == ld_dout) &&
        share_bytes(d_qkv, nd, d_out, extent(T, ld_dout, cols)))
        return set_error(ATP_ERR_INVALID_ARGUMENT, "d_qkv must be d_out itself or not overlap it");
    atp::NormRopeBwdProblem p = {};
    p.f = norm_rope(params, positions);
    p.x = bits(qkv); p.ldx = ld_qkv;
    p.dy = bits(d_out); p.lddy = ld_dout;
    p.dx = bits(d_qkv); p.lddx = ld_dqkv;
    p.tokens = T;
    p.seq = seq;
    p.kv_heads = kv_heads;
    p.group = group;
    p.dqw = dq_weight;
    p.dkw = dk_weight;
    p.ws = static_cast<float*>(workspace);
    const double qk = (double)T * kv_heads * (group + 1) * atp::kHead;
    const double v = d_qkv == d_out ? 0.0 : (double)T * kv_heads * atp::kHead;
    hipStream_t s = stream_of(stream);
    return run_timed("qk_norm_rope_bwd", 16.0 * qk, 6.0 * qk + 4.0 * v, s,
                     [&] { return atp::launch_norm_rope_bwd(p, s); });
}

atp_status atp_qk_norm_rope_cache(const atp_kv_cache* cache, const atp_kv_batch* batch,
                                  int64_t tokens, int32_t group, const atp_qk_norm_rope* params,
                                  const int32_t* positions, const void* qkv, int64_t ld_qkv,
                                  void* q, int64_t ld_q, void* stream) {
    ATP_CHECK(check_cache(cache));
    ATP_CHECK(check_batch(batch, cache->page_size, true, true));
    ATP_CHECK(check_tokens(tokens));
    ATP_CHECK(check_heads(cache->kv_heads, group));
    ATP_CHECK(check_params(params));
    const int64_t cols = (int64_t)cache->kv_heads * (group + 2) * atp::kHead;
    const int64_t qcols = (int64_t)cache->kv_heads * group * atp::kHead;
    ATP_CHECK(check_matrix(qkv, tokens, ld_qkv, cols, "qkv"));
    ATP_CHECK(check_matrix(q, tokens, ld_q, qcols, "q"));
    ATP_CHECK(check_optional(positions, "positions"));
    if (tokens == 0 || batch->n_seqs == 0) return ATP_OK;
    const int64_t nx = extent(tokens, ld_qkv, cols), nq = extent(tokens, ld_q, qcols);
    const int64_t nc = cache_bytes(cache);
    if (share_bytes(qkv, nx, q, nq) || share_bytes(qkv, nx, cache->pages, nc) ||
        share_bytes(q, nq, cache->pages, nc))
        return set_error(ATP_ERR_INVALID_ARGUMENT, "qkv, q and the cache must not overlap");
    atp::NormRopeProblem p = {};
    p.f = norm_rope(params, positions);
    p.x = bits(qkv); p.ldx = ld_qkv;
    p.y = bits(q); p.ldy = ld_q;
    p.tokens = tokens;
    p.seq = 1;
    p.kv_heads = cache->kv_heads;
    p.group = group;
    p.cached = true;
    p.cache = view(cache);
    p.batch = view(batch);
    const double el = (double)tokens * cols;
    hipStream_t s = stream_of(stream);
    return run_timed("qk_norm_rope_cache", 8.0 * el, 4.0 * el, s,
                     [&] { return atp::launch_norm_rope(p, s); });
}

size_t atp_cache_workspace_bytes(int32_t n_pages, int32_t n_seqs) {
    if (n_pages < 1 || n_seqs < 0) return 0;
    return sizeof(int32_t) * ((size_t)n_pages + (size_t)n_seqs);
}

atp_status atp_cache_reserve(int32_t n_pages, int32_t page_size, int32_t* refs,
                             const atp_kv_batch* batch, int32_t* missing, int32_t* copy_src,
                             int32_t* copy_dst, int32_t* copy_rows, void* workspace,
                             size_t ws_bytes, void* stream) {
    ATP_CHECK(check_pool(n_pages, page_size));
    ATP_CHECK(check_batch(batch, page_size, true, true));
    ATP_CHECK(check_vector(refs, "refs"));
    if (batch->n_seqs == 0) return ATP_OK;
    ATP_CHECK(check_vector(missing, "missing"));
    ATP_CHECK(check_vector(copy_src, "copy_src"));
    ATP_CHECK(check_vector(copy_dst, "copy_dst"));
    ATP_CHECK(check_vector(copy_rows, "copy_rows"));
    ATP_CHECK(check_workspace(workspace, ws_bytes,
                              atp_cache_workspace_bytes(n_pages, batch->n_seqs)));
    hipStream_t s = stream_of(stream);
    return run_timed("cache_reserve", 0.0, 4.0 * n_pages, s, [&] {
        return atp::launch_cache_reserve(n_pages, shift_of(page_size), refs, view(batch), missing,
                                         copy_src, copy_dst, copy_rows,
                                         static_cast<int32_t*>(workspace), s);
    });
}

atp_status atp_cache_fork(int32_t n_pages, int32_t page_size, int32_t* refs,
                          const atp_kv_batch* batch, int32_t n_forks, const int32_t* parents,
                          const int32_t* children, int32_t* done, void* stream) {
    ATP_CHECK(check_pool(n_pages, page_size));
    ATP_CHECK(check_batch(batch, page_size, true, false));
    ATP_CHECK(check_vector(refs, "refs"));
    if (n_forks < 0) return set_error(ATP_ERR_INVALID_ARGUMENT, "n_forks %d", n_forks);
    if (n_forks > ATP_MAX_FORKS)
        return set_error(ATP_ERR_UNSUPPORTED, "n_forks %d: at most %d", n_forks, ATP_MAX_FORKS);
    if (n_forks == 0) return ATP_OK;
    ATP_CHECK(check_vector(parents, "parents"));
    ATP_CHECK(check_vector(children, "children"));
    ATP_CHECK(check_vector(done, "done"));
    hipStream_t s = stream_of(stream);
    return run_timed("cache_fork", 0.0, 12.0 * n_forks * batch->max_pages, s, [&] {
        return atp::launch_cache_fork(n_pages, shift_of(page_size), refs, view(batch), n_forks,
                                      parents, children, done, s);
    });
}

atp_status atp_cache_release(int32_t n_pages, int32_t page_size, int32_t* refs,
                             const atp_kv_batch* batch, const int32_t* keep, void* stream) {
    ATP_CHECK(check_pool(n_pages, page_size));
    ATP_CHECK(check_batch(batch, page_size, false, false));
    ATP_CHECK(check_vector(refs, "refs"));
    if (batch->n_seqs == 0) return ATP_OK;
    ATP_CHECK(check_vector(keep, "keep"));
    hipStream_t s = stream_of(stream);
    return run_timed("cache_release", 0.0, 8.0 * batch->n_seqs * batch->max_pages, s, [&] {
        return atp::launch_cache_release(n_pages, shift_of(page_size), refs, view(batch), keep, s);
    });
}

atp_status atp_cache_copy_pages(const atp_kv_cache* cache, int32_t n, const int32_t* src,
                                const int32_t* dst, const int32_t* rows, void* stream) {
    ATP_CHECK(check_cache(cache));
    if (n < 0) return set_error(ATP_ERR_INVALID_ARGUMENT, "n %d", n);
    if (n > kMaxCopies) return set_error(ATP_ERR_UNSUPPORTED, "n %d: at most 2^23", n);
    if (n == 0) return ATP_OK;
    ATP_CHECK(check_vector(src, "src"));
    ATP_CHECK(check_vector(dst, "dst"));
    ATP_CHECK(check_optional(rows, "rows"));
    const double bytes = 2.0 * n * (double)cache_bytes(cache) / cache->n_pages;
    hipStream_t s = stream_of(stream);
    return run_timed("cache_copy_pages", 0.0, bytes, s,
                     [&] { return atp::launch_cache_copy(view(cache), n, src, dst, rows, s); });
}

atp_status atp_cache_compact(const atp_kv_cache* cache, const atp_kv_batch* batch,
                             const int32_t* cu_keep, const int32_t* keep, int32_t n_keep,
                             int32_t* moved, void* stream) {
    ATP_CHECK(check_cache(cache));
    ATP_CHECK(check_batch(batch, cache->page_size, true, false));
    if (n_keep < 0) return set_error(ATP_ERR_INVALID_ARGUMENT, "n_keep %d", n_keep);
    if (batch->n_seqs == 0) return ATP_OK;
    ATP_CHECK(check_vector(cu_keep, "cu_keep"));
    if (n_keep > 0) ATP_CHECK(check_vector(keep, "keep"));
    ATP_CHECK(check_optional(moved, "moved"));
    const double bytes = 2.0 * n_keep * 2.0 * cache->kv_heads * atp::kHead * 2.0;
    hipStream_t s = stream_of(stream);
    return run_timed("cache_compact", 0.0, bytes, s, [&] {
        return atp::launch_cache_compact(view(cache), view(batch), cu_keep, keep, n_keep, moved, s);
    });
}

size_t atp_attention_cache_workspace_bytes(int32_t kv_heads, int32_t group, int32_t max_new) {
    if (kv_heads < 1 || group < 1 || group > ATP_MAX_QUERY_GROUP || max_new < 1) return 0;
    return sizeof(float) * (size_t)atp::cache_attention_ws_floats(group, max_new);
}

atp_status atp_attention_cache_fwd(const atp_kv_cache* cache, const atp_kv_batch* batch,
                                   int64_t tokens, int32_t group, int32_t max_new, const void* q,
                                   int64_t ld_q, const uint64_t* tree_mask, int32_t mask_words,
                                   void* out, int64_t ld_out, float* lse, void* workspace,
                                   size_t ws_bytes, void* stream) {
    ATP_CHECK(check_cache(cache));
    ATP_CHECK(check_batch(batch, cache->page_size, true, true));
    ATP_CHECK(check_tokens(tokens));
    ATP_CHECK(check_heads(cache->kv_heads, group));
    if (max_new < 1) return set_error(ATP_ERR_INVALID_ARGUMENT, "max_new %d", max_new);
    const int64_t cols = (int64_t)cache->kv_heads * group * atp::kHead;
    ATP_CHECK(check_matrix(q, tokens, ld_q, cols, "q"));
    ATP_CHECK(check_matrix(out, tokens, ld_out, cols, "out"));
    ATP_CHECK(check_optional(lse, "lse"));
    ATP_CHECK(check_optional(tree_mask, "tree_mask"));
    if (tree_mask && mask_words < 1)
        return set_error(ATP_ERR_INVALID_ARGUMENT, "mask_words %d", mask_words);
    if (tokens == 0 || batch->n_seqs == 0) return ATP_OK;
    ATP_CHECK(check_workspace(
        workspace, ws_bytes,
        atp_attention_cache_workspace_bytes(cache->kv_heads, group, max_new)));
    const int64_t nq = extent(tokens, ld_q, cols), no = extent(tokens, ld_out, cols);
    if (share_bytes(q, nq, out, no) || share_bytes(out, no, cache->pages, cache_bytes(cache)))
        return set_error(ATP_ERR_INVALID_ARGUMENT, "out must not overlap q or the cache");
    atp::CacheAttentionProblem p = {};
    p.cache = view(cache);
    p.batch = view(batch);
    p.tokens = tokens;
    p.group = group;
    p.max_new = max_new;
    p.q = bits(q); p.ldq = ld_q;
    p.mask = tree_mask; p.mask_words = mask_words;
    p.out = bits(out); p.ldo = ld_out;
    p.lse = lse;
    p.ws = static_cast<float*>(workspace);
    hipStream_t s = stream_of(stream);
    // the lengths are on the device: what the queries and outputs take alone
    return run_timed("attention_cache", 0.0, 4.0 * tokens * cols, s,
                     [&] { return atp::launch_cache_attention(p, s); });
}

}  // extern "C"
