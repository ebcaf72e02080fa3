// Internal launch interface of the position, cache and cached-attention
// kernels.  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace atp {

constexpr int kHead = 128;   // head dimension

// A layer's cache and a batch's pages, as the kernels take them.
struct CacheView {
    uint16_t* pages;         // [n_pages][2][kv_heads][page][128]
    int n_pages, kv_heads, page_shift;
};
struct BatchView {
    int32_t* table;          // [n_seqs][ld_table]
    int64_t ld_table;
    int max_pages, n_seqs;
    const int32_t* ctx;      // [n_seqs]
    const int32_t* cu;       // [n_seqs + 1]
};

struct NormRope {
    const uint16_t *qw, *kw;   // nullable: ones
    const float* inv_freq;
    const int32_t* pos;        // nullable
    float eps;
    bool norm, interleaved;
    int rot;
};

struct NormRopeProblem {
    NormRope f;
    const uint16_t* x; int64_t ldx;
    uint16_t* y; int64_t ldy;     // the block, or the queries when `cached`
    int64_t tokens, seq;
    int kv_heads, group;
    bool cached;
    CacheView cache;
    BatchView batch;
};
hipError_t launch_norm_rope(const NormRopeProblem& p, hipStream_t s);

struct NormRopeBwdProblem {
    NormRope f;
    const uint16_t* x; int64_t ldx;
    const uint16_t* dy; int64_t lddy;
    uint16_t* dx; int64_t lddx;
    int64_t tokens, seq;
    int kv_heads, group;
    float *dqw, *dkw;             // nullable
    float* ws;
};
hipError_t launch_norm_rope_bwd(const NormRopeBwdProblem& p, hipStream_t s);
int64_t norm_rope_ws_floats(int64_t tokens);

hipError_t launch_cache_reserve(int n_pages, int page_shift, int32_t* refs, const BatchView& b,
                                int32_t* missing, int32_t* src, int32_t* dst, int32_t* rows,
                                int32_t* ws, hipStream_t s);
hipError_t launch_cache_fork(int n_pages, int page_shift, int32_t* refs, const BatchView& b, int n,
                             const int32_t* parents, const int32_t* children, int32_t* done,
                             hipStream_t s);
hipError_t launch_cache_release(int n_pages, int page_shift, int32_t* refs, const BatchView& b,
                                const int32_t* keep, hipStream_t s);
hipError_t launch_cache_copy(const CacheView& c, int n, const int32_t* src, const int32_t* dst,
                             const int32_t* rows, hipStream_t s);
hipError_t launch_cache_compact(const CacheView& c, const BatchView& b, const int32_t* cu_keep,
                                const int32_t* keep, int n_keep, int32_t* moved, hipStream_t s);

struct CacheAttentionProblem {
    CacheView cache;
    BatchView batch;
    int64_t tokens;
    int group, max_new;
    const uint16_t* q; int64_t ldq;
    const uint64_t* mask; int mask_words;   // nullable: causal
    uint16_t* out; int64_t ldo;
    float* lse;                             // nullable
    float* ws;
};
hipError_t launch_cache_attention(const CacheAttentionProblem& p, hipStream_t s);
int64_t cache_attention_ws_floats(int group, int max_new);

}  // namespace atp
