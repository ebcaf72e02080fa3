// Internal launch interface of the kernels around the layers: embedding, layer
// norm, gradient norm and clipping, attention within documents.  Not part of the
// public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.h"

namespace atp {

// Threads of a launch are fewer than 2^32: HIP drops the rest of a larger one without an error.
constexpr int64_t kLaunchThreads = (int64_t)1 << 32;
inline bool fits_launch(int64_t groups, int64_t threads) {
    return groups < kLaunchThreads / threads;
}

struct EmbeddingProblem {
    const int32_t* ids;
    int64_t tokens, vocab, off, cols;    // rows of this device's table, its first token
    const uint16_t* table; int64_t ldt;
    float scale;
    void* out; int64_t ldo; bool out_f32;
};
bool embedding_fits(int64_t tokens, int64_t cols);       // one launch
hipError_t launch_embedding(const EmbeddingProblem& p, hipStream_t s);

struct EmbeddingBwdProblem {
    const int32_t* ids;
    int64_t tokens, vocab, off, cols;
    const uint16_t* dy; int64_t lddy;
    float scale;
    float* dtable; int64_t ldt;
    bool accumulate;
    void* ws;
};
hipError_t launch_embedding_bwd(const EmbeddingBwdProblem& p, hipStream_t s);
int64_t embedding_ws_bytes(int64_t tokens, int64_t vocab, int64_t cols);

constexpr int64_t kMaxNormCols = 32768;
// One call of the layer norm: statistics of the own columns alone (stats_out), the
// norm of whole rows, or the norm from the group's statistics (parts).
struct LayerNormProblem {
    int64_t tokens, cols;
    bool f32;                            // type of x and x_out
    const void* x; int64_t ldx;
    const uint16_t* add; int64_t ldadd;  // nullable
    void* x_out; int64_t ldxo;           // with add
    const uint16_t *weight, *bias;       // nullable
    float eps;
    float* stats_out;                    // [tokens][2]: mean, centred squares
    int nparts;
    const float* parts[kMaxParts];
    uint16_t* y; int64_t ldy;
    float *mean, *rstd;
};
bool layer_norm_fits(int64_t tokens, int64_t cols);      // one launch
hipError_t launch_layer_norm(const LayerNormProblem& p, hipStream_t s);

struct LayerNormBwdProblem {
    int64_t tokens, cols;
    bool f32;
    const void* x; int64_t ldx;
    const uint16_t* weight;
    const float *mean, *rstd;
    const uint16_t* dy; int64_t lddy;
    float* sums_out;                     // [tokens][2]; alone: nothing else is formed
    int nparts;
    const float* parts[kMaxParts];
    const void* dres; int64_t lddres;    // nullable
    void* dx; int64_t lddx;
    uint16_t* dadd; int64_t lddadd;      // nullable
    float *dw, *db;                      // nullable
    float* ws;
};
hipError_t launch_layer_norm_bwd(const LayerNormBwdProblem& p, hipStream_t s);
int64_t layer_norm_ws_floats(int64_t tokens, int64_t cols);

// Gradients, as the clipping kernels take them.
struct GradView {
    const void* src; void* dst;
    int64_t rows, cols, ld_src, ld_dst;
    bool src_f32, dst_f32;
};
int64_t grad_sum_blocks(int n, const GradView* g);
hipError_t launch_grad_sq_sum(int n, const GradView* g, double* sum, double* ws, hipStream_t s);
hipError_t launch_grad_clip(int n, const GradView* g, int nparts, const double* const* parts,
                            float scale, float max_norm, float* norm, hipStream_t s);

// Attention within documents of the packed rows.
struct DocsView {
    const int32_t* cu;
    const int32_t* prefix;               // nullable
    const float* slopes;                 // nullable
    int n_docs;
    float cap;                           // 0: none
};
struct DocsAttentionProblem {
    DocsView docs;
    int64_t tokens;
    int kv_heads, group;
    const uint16_t* qkv; int64_t ldq;
    uint16_t* out; int64_t ldo;
    float* lse;
};
hipError_t launch_docs_attention(const DocsAttentionProblem& p, hipStream_t s);

struct DocsAttentionBwdProblem {
    DocsView docs;
    int64_t tokens;
    int kv_heads, group;
    const uint16_t* qkv; int64_t ldq;
    const uint16_t* out; int64_t ldo;
    const float* lse;
    const uint16_t* dout; int64_t lddo;
    uint16_t* dqkv; int64_t lddq;
    float* ws;
};
hipError_t launch_docs_attention_bwd(const DocsAttentionBwdProblem& p, hipStream_t s);
int64_t docs_attention_ws_floats(int64_t tokens, int kv_heads, int group);

}  // namespace atp
