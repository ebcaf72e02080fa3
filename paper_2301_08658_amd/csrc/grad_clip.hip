// Norm over many gradients, and clipping by it.
//
//   S = sum over the tensors of g^2 (per device),  N = scale sqrt(sum of S over the
//   devices),  f = scale (N > max_norm ? max_norm / N : 1),  dst = f src.
//
// Squares and sums are formed in 64 bits: squares of 32-bit values neither overflow
// nor vanish there, and a sum of 10^9 of them keeps its digits.  A workgroup takes
// consecutive values of one tensor and leaves one partial sum; the partial sums are
// added in a fixed order.  Bound by memory: the gradients are read once
// for the norm, and once more, with one write, for the clipping, which cannot begin
// before the norm is known.  The list of tensors travels in the kernels' arguments,
// as many per launch as 4 KiB hold (250 for the sum, 160 for the clipping), so a call
// keeps nothing and can be captured; with one list of 72 entries for all uses 300
// tensors took 64 us, in 11 launches.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "train_kernels.h"
#include "wave_ops.h"

namespace atp {
namespace {

constexpr int kThreads = 256;
// Values of a workgroup, of the sum and of the clipping (629 M fp32 values: sums of 4096
// 381 us, of 16384 380, of bf16 values 394 and 381; clipping of 4096 857 us, of 8192 940,
// of 16384 990).
constexpr int kSumValues = 16384, kClipValues = 4096;
constexpr int64_t kMaxRun = 1 << 30;                 // values of a run; longer ones are cut
constexpr int64_t kMaxRowBlocks = 1 << 23;           // workgroups of rows with gaps, likewise
static_assert(kMaxRun / kClipValues <= kMaxRowBlocks && kClipValues <= kSumValues, "pieces");
// Gradients of more bytes go past the caches, which hold no value from the sum to the
// clipping then.  Sum and clipping into other memory, cached and past the caches: of
// 128 MiB 65 and 71 us, of 256 MiB 154 and 134, of 1 GiB 572 and 526.
constexpr int64_t kCachedBytes = 128 << 20;

// Tensors of a launch: runs of consecutive values (kRuns without a destination), or
// matrices with gaps between their rows.  Bit 0 of the pointers (16-byte aligned) says
// whether the values are fp32.
enum Kind { kRuns, kRunsTo, kRowsTo };
template <Kind K, int N>
struct List {
    static constexpr Kind kind = K;
    static constexpr int kMost = N;
    int32_t n;
    int32_t first[N];                                // first workgroup of each
    uint64_t src[N], dst[K == kRuns ? 1 : N];
    int64_t cols[K == kRowsTo ? N : 1];
    uint32_t run[K == kRowsTo ? 1 : N];
    int32_t rows[K == kRowsTo ? N : 1], ld_src[K == kRowsTo ? N : 1], ld_dst[K == kRowsTo ? N : 1];
};

// The tensor of a workgroup, the last one that begins at or before it: 64 entries at a
// time.
template <class L>
__device__ __forceinline__ int find(const L& list, int block) {
    const int lane = threadIdx.x & 63;
    int at = -1;
#pragma unroll
    for (int i = 0; i < (L::kMost + 63) / 64; ++i) {
        if (i * 64 >= list.n) break;
        const int k = i * 64 + lane;
        at += __popcll(__builtin_amdgcn_ballot_w64(k < list.n && list.first[k] <= block));
    }
    return __builtin_amdgcn_readfirstlane(at);
}

// Where the thread's vectors of W values lie, in workgroups of G values: vector i in row
// `row` from value `col`.
template <Kind K, int W, int G>
struct Places {
    int64_t cols, row0;
    int32_t rows, ld_src, ld_dst;
    uint32_t rem, per;                               // of the workgroup's first vector, per row
    template <class L>
    __device__ __forceinline__ Places(const L& list, int t, int block) {
        const int64_t vec0 = (int64_t)(block - list.first[t]) * (G / W);
        if constexpr (K == kRowsTo) {
            cols = list.cols[t];
            rows = list.rows[t];
            ld_src = list.ld_src[t];
            ld_dst = list.ld_dst[t];
            // a row with gaps has at most 2^22 values
            per = (uint32_t)((cols + 7) >> 3) * (8 / W);
            row0 = vec0 / per;
            rem = (uint32_t)(vec0 - row0 * per);
        } else {
            cols = list.run[t];
            row0 = vec0 * W;                         // the first value
        }
    }
    struct At {
        int64_t row, col;
        bool in;
    };
    __device__ __forceinline__ At at(int i) const {
        const uint32_t v = i * kThreads + threadIdx.x;
        if constexpr (K == kRowsTo) {
            const uint32_t down = (rem + v) / per;
            const int64_t row = row0 + down;
            return At{row, (int64_t)(rem + v - down * per) * W, row < rows};
        } else {
            const int64_t col = row0 + (int64_t)v * W;
            return At{0, col, col < cols};
        }
    }
};

// W values of a tensor, in the tensor's type.  fp32 values go four at a time, so that a
// wave's 16-byte accesses lie side by side.  PAST: past the caches.
template <class T, int W, bool PAST>
struct Values {
    typedef T Vec __attribute__((ext_vector_type(W)));
    Vec w;
    // values [c, c + W) of a row, zeros behind its end
    __device__ __forceinline__ void load(const T* row, int64_t c, int64_t cols) {
        if (c + W <= cols) {
            const Vec* from = reinterpret_cast<const Vec*>(row + c);
            if constexpr (PAST) w = __builtin_nontemporal_load(from);
            else w = *from;
            return;
        }
#pragma unroll
        for (int e = 0; e < W; ++e) w[e] = c + e < cols ? row[c + e] : T(0);
    }
    __device__ __forceinline__ void store(T* row, int64_t c, int64_t cols) const {
        if (c + W <= cols) {
            Vec* to = reinterpret_cast<Vec*>(row + c);
            if constexpr (PAST) __builtin_nontemporal_store(w, to);
            else *to = w;
            return;
        }
#pragma unroll
        for (int e = 0; e < W; ++e)
            if (c + e < cols) row[c + e] = w[e];
    }
    __device__ __forceinline__ float get(int e) const {
        if constexpr (sizeof(T) == 4) return w[e];
        else return __uint_as_float((uint32_t)w[e] << 16);
    }
    __device__ __forceinline__ void set(const float (&v)[W]) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int e = 0; e < W; ++e) w[e] = v[e];
        } else {
            uint32_t two[W / 2];
#pragma unroll
            for (int e = 0; e < W / 2; ++e) two[e] = wave::pack2(v[2 * e], v[2 * e + 1]);
            w = __builtin_bit_cast(Vec, two);
        }
    }
};

__device__ __forceinline__ double block_sum(double v, double* red) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    const int waves = blockDim.x >> 6;
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0;
    for (int i = 0; i < waves; ++i) v += red[i];
    return v;
}

template <bool PAST, class T, class L>
__device__ __forceinline__ double squares(const T* src, const L& list, int t) {
    constexpr int W = sizeof(T) == 4 ? 4 : 8, N = kSumValues / kThreads / W;
    constexpr Kind K = L::kind;
    const Places<K, W, kSumValues> p(list, t, blockIdx.x);
    Values<T, W, PAST> in[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const auto a = p.at(i);
        if (a.in) in[i].load(K == kRowsTo ? src + a.row * p.ld_src : src, a.col, p.cols);
        else in[i].w = {};
    }
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
#pragma unroll
        for (int e = 0; e < W; ++e) s += (double)in[i].get(e) * (double)in[i].get(e);
    }
    return s;
}

template <class T>
__device__ __forceinline__ T* pointer(uint64_t p) {
    return reinterpret_cast<T*>(p & ~(uint64_t)15);
}

template <bool PAST, class L>
__global__ __launch_bounds__(kThreads) void sq_sum_kernel(L list, double* part) {
    __shared__ double red[kThreads / 64];
    const int t = find(list, blockIdx.x);
    const uint64_t src = list.src[t];
    double s = src & 1 ? squares<PAST>(pointer<const float>(src), list, t)
                       : squares<PAST>(pointer<const uint16_t>(src), list, t);
    s = block_sum(s, red);
    if (threadIdx.x == 0) part[blockIdx.x] = s;
}

constexpr int kJoinThreads = 1024;
__global__ __launch_bounds__(kJoinThreads) void sq_join_kernel(const double* part, int64_t n,
                                                               double* sum) {
    __shared__ double red[kJoinThreads / 64];
    double s = 0.0;
#pragma unroll 4
    for (int64_t i = threadIdx.x; i < n; i += kJoinThreads) s += part[i];
    s = block_sum(s, red);
    if (threadIdx.x == 0) *sum = s;
}

template <int N>
struct Factor {
    const double* parts[N];
    int nparts;
    float scale, max_norm;
    float* norm;                                     // in the first launch: norm and factor
};

// The devices' sums, in group order, as norm and factor (by every workgroup).
template <int N>
__device__ __forceinline__ float factor_of(const Factor<N>& F) {
    double s = 0.0;
    for (int j = 0; j < F.nparts; ++j) s += *F.parts[j];
    const double norm = (double)F.scale * sqrt(s);
    const float f = (float)((double)F.scale *
                            (norm <= (double)F.max_norm ? 1.0 : (double)F.max_norm / norm));
    if (F.norm && blockIdx.x == 0 && threadIdx.x == 0) {
        F.norm[0] = (float)norm;
        F.norm[1] = f;
    }
    return f;
}

template <bool PAST, class S, class T, class L, int PARTS>
__device__ __forceinline__ void scaled(const S* src, T* dst, const L& list, int t,
                                       const Factor<PARTS>& F) {
    constexpr int W = sizeof(S) == 4 || sizeof(T) == 4 ? 4 : 8, N = kClipValues / kThreads / W;
    constexpr Kind K = L::kind;
    const Places<K, W, kClipValues> p(list, t, blockIdx.x);
    Values<S, W, PAST> in[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const auto a = p.at(i);
        if (a.in) in[i].load(K == kRowsTo ? src + a.row * p.ld_src : src, a.col, p.cols);
    }
    const float f = factor_of(F);                    // while the values come
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const auto a = p.at(i);
        if (!a.in) continue;
        float v[W];
#pragma unroll
        for (int e = 0; e < W; ++e) v[e] = f * in[i].get(e);
        Values<T, W, PAST> out;
        out.set(v);
        out.store(K == kRowsTo ? dst + a.row * p.ld_dst : dst, a.col, p.cols);
    }
}

template <bool PAST, class L, int N>
__global__ __launch_bounds__(kThreads) void clip_kernel(L list, Factor<N> F) {
    if (list.n == 0) {
        factor_of(F);
        return;
    }
    const int t = find(list, blockIdx.x);
    const uint64_t src = list.src[t], dst = list.dst[t];
    if (src == dst && factor_of(F) == 1.f) return;   // in place already
    if (src & 1) {
        const float* from = pointer<const float>(src);
        if (dst & 1) scaled<PAST>(from, pointer<float>(dst), list, t, F);
        else scaled<PAST>(from, pointer<uint16_t>(dst), list, t, F);
    } else {
        const uint16_t* from = pointer<const uint16_t>(src);
        if (dst & 1) scaled<PAST>(from, pointer<float>(dst), list, t, F);
        else scaled<PAST>(from, pointer<uint16_t>(dst), list, t, F);
    }
}

// Rows without gaps are one run.
bool is_run(const GradView& g, bool with_dst) {
    return g.rows <= 1 || (g.ld_src == g.cols && (!with_dst || g.ld_dst == g.cols));
}
int64_t row_blocks(int64_t rows, int64_t cols, int group) {
    return (rows * ((cols + 7) / 8) + group / 8 - 1) / (group / 8);
}
// Rows with gaps that one entry takes.
int64_t piece_rows(int64_t cols, int group) {
    return kMaxRowBlocks * (group / 8) / ((cols + 7) / 8);
}
int64_t blocks_of(const GradView& g) {
    if (g.rows == 0 || g.cols == 0) return 0;
    int64_t blocks = 0;
    if (!is_run(g, false)) {
        const int64_t most = piece_rows(g.cols, kSumValues);
        for (int64_t left = g.rows; left > 0; left -= most)
            blocks += row_blocks(std::min(left, most), g.cols, kSumValues);
        return blocks;
    }
    for (int64_t left = g.rows * g.cols; left > 0; left -= kMaxRun)
        blocks += row_blocks(1, std::min(left, kMaxRun), kSumValues);
    return blocks;
}

bool past_caches(int n, const GradView* g) {
    int64_t bytes = 0;
    for (int i = 0; i < n; ++i) bytes += g[i].rows * g[i].cols * (g[i].src_f32 ? 4 : 2);
    return bytes > kCachedBytes;
}

// Collects entries of one kind and calls f(list, workgroups) for every full one, or one that
// fills a launch.
template <class L, class F>
struct Launches {
    L list;
    int64_t blocks = 0;
    F f;
    hipError_t e = hipSuccess;
    explicit Launches(F f_) : f(f_) { list.n = 0; }
    void flush() {
        if (list.n && e == hipSuccess) e = f(list, blocks);
        list.n = 0;
        blocks = 0;
    }
    // the next entry's place; b: its workgroups
    int next(int64_t b) {
        if (list.n == L::kMost || !fits_launch(blocks + b, kThreads)) flush();
        list.first[list.n] = (int32_t)blocks;
        blocks += b;
        return list.n++;
    }
};

template <class Runs, class Rows, class F>
hipError_t in_launches(int n, const GradView* g, bool with_dst, F f) {
    Launches<Runs, F> runs(f);
    Launches<Rows, F> rows(f);
    const int group = with_dst ? kClipValues : kSumValues;
    for (int i = 0; i < n; ++i) {
        if (g[i].rows == 0 || g[i].cols == 0) continue;
        const uint64_t src = reinterpret_cast<uint64_t>(g[i].src);
        const uint64_t dst = reinterpret_cast<uint64_t>(g[i].dst);
        if (is_run(g[i], with_dst)) {
            const int64_t total = g[i].rows * g[i].cols;
            for (int64_t at = 0; at < total; at += kMaxRun) {
                const int64_t len = std::min(total - at, kMaxRun);
                const int t = runs.next(row_blocks(1, len, group));
                runs.list.src[t] = (src + at * (g[i].src_f32 ? 4 : 2)) | (g[i].src_f32 ? 1 : 0);
                if (with_dst)
                    runs.list.dst[t] = (dst + at * (g[i].dst_f32 ? 4 : 2)) | (g[i].dst_f32 ? 1 : 0);
                runs.list.run[t] = (uint32_t)len;
            }
            continue;
        }
        const int64_t most = piece_rows(g[i].cols, group);
        for (int64_t at = 0; at < g[i].rows; at += most) {
            const int64_t n_rows = std::min(g[i].rows - at, most);
            const int t = rows.next(row_blocks(n_rows, g[i].cols, group));
            rows.list.src[t] =
                (src + at * g[i].ld_src * (g[i].src_f32 ? 4 : 2)) | (g[i].src_f32 ? 1 : 0);
            if (with_dst)
                rows.list.dst[t] =
                    (dst + at * g[i].ld_dst * (g[i].dst_f32 ? 4 : 2)) | (g[i].dst_f32 ? 1 : 0);
            rows.list.cols[t] = g[i].cols;
            rows.list.rows[t] = (int32_t)n_rows;
            rows.list.ld_src[t] = (int32_t)g[i].ld_src;
            rows.list.ld_dst[t] = (int32_t)g[i].ld_dst;
        }
    }
    runs.flush();
    if (runs.e != hipSuccess) return runs.e;
    rows.flush();
    return rows.e;
}

template <int RUNS, int ROWS, int PARTS>
hipError_t clip(int n, const GradView* g, int nparts, const double* const* parts, float scale,
                float max_norm, float* norm, hipStream_t s) {
    Factor<PARTS> F = {};
    std::copy(parts, parts + nparts, F.parts);
    F.nparts = nparts;
    F.scale = scale;
    F.max_norm = max_norm;
    F.norm = norm;
    typedef List<kRunsTo, RUNS> Runs;
    typedef List<kRowsTo, ROWS> Rows;
    static_assert(sizeof(Runs) + sizeof(F) <= 4096 && sizeof(Rows) + sizeof(F) <= 4096,
                  "kernel arguments");
    const bool past = past_caches(n, g);
    const hipError_t e = in_launches<Runs, Rows>(n, g, true, [&](const auto& L, int64_t blocks) {
        const dim3 grid((unsigned)blocks);
        if (past) clip_kernel<true><<<grid, kThreads, 0, s>>>(L, F);
        else clip_kernel<false><<<grid, kThreads, 0, s>>>(L, F);
        F.norm = nullptr;
        return hipGetLastError();
    });
    if (e != hipSuccess || !F.norm) return e;
    Runs none;                                       // nothing to scale: the norm alone
    none.n = 0;
    clip_kernel<false><<<1, 64, 0, s>>>(none, F);
    return hipGetLastError();
}

}  // namespace

int64_t grad_sum_blocks(int n, const GradView* g) {
    int64_t blocks = 0;
    for (int i = 0; i < n; ++i) blocks += blocks_of(g[i]);
    return blocks;
}

hipError_t launch_grad_sq_sum(int n, const GradView* g, double* sum, double* ws, hipStream_t s) {
    int64_t done = 0;
    typedef List<kRuns, 250> Runs;
    typedef List<kRowsTo, 80> Rows;
    static_assert(sizeof(Runs) + 8 <= 4096 && sizeof(Rows) + 8 <= 4096, "kernel arguments");
    const bool past = past_caches(n, g);
    const hipError_t e = in_launches<Runs, Rows>(n, g, false, [&](const auto& L, int64_t blocks) {
        const dim3 grid((unsigned)blocks);
        if (past) sq_sum_kernel<true><<<grid, kThreads, 0, s>>>(L, ws + done);
        else sq_sum_kernel<false><<<grid, kThreads, 0, s>>>(L, ws + done);
        done += blocks;
        return hipGetLastError();
    });
    if (e != hipSuccess) return e;
    sq_join_kernel<<<1, kJoinThreads, 0, s>>>(ws, done, sum);
    return hipGetLastError();
}

hipError_t launch_grad_clip(int n, const GradView* g, int nparts, const double* const* parts,
                            float scale, float max_norm, float* norm, hipStream_t s) {
    if (nparts <= 8) return clip<160, 80, 8>(n, g, nparts, parts, scale, max_norm, norm, s);
    return clip<140, 80, kMaxParts>(n, g, nparts, parts, scale, max_norm, norm, s);
}

}  // namespace atp
