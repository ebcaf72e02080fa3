// Norm over many gradients, and clipping by it.
//
//   S = sum over the tensors of g^2 (per device),  N = scale sqrt(sum of S over the
//   devices),  f = scale (N > max_norm ? max_norm / N : 1),  dst = f src.
//
// Squares and sums are formed in 64 bits: squares of 32-bit values neither overflow
// nor vanish there, and a sum of 10^9 of them keeps its digits.  A workgroup takes
// 16384 consecutive values of one tensor and leaves one partial sum; the partial
// sums are added in a fixed order.  Bound by memory: the gradients are read once
// for the norm, and once more, with one write, for the clipping, which cannot begin
// before the norm is known.  The list of tensors travels in the kernels' arguments
// (a launch takes as many tensors as fit 4 KiB), so a call keeps nothing and can be
// captured.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "train_kernels.h"
#include "wave_ops.h"

namespace atp {
namespace {

using wave::Eight;

constexpr int kThreads = 256;
constexpr int kVecs = 8;                             // vectors of eight values per thread
constexpr int64_t kSpan = (int64_t)kThreads * kVecs * 8;

// One tensor of a launch: rows of `cols` values, or one run of them.  Bit 0 of the
// pointers (16-byte aligned) says whether the values are fp32.
struct Item {
    uint64_t src, dst;
    int64_t cols;
    int32_t ld_src, ld_dst, rows, first;             // first: its first workgroup in the launch
};
constexpr int kItems = 72;
struct Items {
    Item t[kItems];
    int n;
};

// Item and span of this workgroup.
__device__ __forceinline__ int find(const Items& L, int block) {
    int lo = 0, hi = L.n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (L.t[mid].first <= block) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// Values [c, c + 8) of a row, zeros behind its end.
template <class T>
__device__ __forceinline__ Eight<T> load8(const T* row, int64_t c, int64_t cols) {
    Eight<T> v;
    if (c + 8 <= cols) {
        v.load(row + c);
    } else {
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            f[e] = 0.f;
            if (c + e < cols) {
                if constexpr (sizeof(T) == 4) f[e] = row[c + e];
                else f[e] = __uint_as_float((uint32_t)row[c + e] << 16);
            }
        }
        v.set(f);
    }
    return v;
}
template <class T>
__device__ __forceinline__ void store8(T* row, int64_t c, int64_t cols, const float* f) {
    Eight<T> v;
    v.set(f);
    if (c + 8 <= cols) {
        v.store(row + c);
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (c + e < cols) {
            if constexpr (sizeof(T) == 4) row[c + e] = f[e];
            else row[c + e] = (uint16_t)(wave::pack2(f[e], 0.f) & 0xffffu);
        }
}

// Row and column of vector i of the workgroup's span `at` (in vectors): a run of
// vectors for one row, rows one behind the other for several.
struct Place {
    int64_t row, col;
    bool in;
};
__device__ __forceinline__ Place place(const Item& it, int64_t vec) {
    const int64_t per = (it.cols + 7) >> 3;
    Place p;
    p.row = it.rows == 1 ? 0 : vec / per;
    p.col = (vec - p.row * per) * 8;
    p.in = p.row < it.rows && p.col < it.cols;
    return p;
}

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

template <class T>
__device__ __forceinline__ double squares(const Item& it, int64_t vec0) {
    const T* src = reinterpret_cast<const T*>(it.src & ~(uint64_t)15);
    Eight<T> in[kVecs];
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        const Place p = place(it, vec0 + i * kThreads + threadIdx.x);
        float z[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (p.in) in[i] = load8(src + p.row * it.ld_src, p.col, it.cols);
        else in[i].set(z);
    }
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        float f[8];
        in[i].get(f);
#pragma unroll
        for (int e = 0; e < 8; ++e) s += (double)f[e] * (double)f[e];
    }
    return s;
}

__global__ __launch_bounds__(kThreads) void sq_sum_kernel(Items L, double* part) {
    __shared__ double red[kThreads / 64];
    const Item& it = L.t[find(L, blockIdx.x)];
    const int64_t vec0 = (int64_t)((int)blockIdx.x - it.first) * (kThreads * kVecs);
    double s = it.src & 1 ? squares<float>(it, vec0) : squares<uint16_t>(it, vec0);
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

struct Factor {
    const double* parts[kMaxParts];
    int nparts;
    float scale, max_norm;
};
struct ClipArgs {
    Items L;
    float* norm;                                     // in the first launch: norm and factor
};
static_assert(sizeof(ClipArgs) + sizeof(Factor) <= 4096, "kernel arguments");

template <class S, class T>
__device__ __forceinline__ void scaled(const Item& it, int64_t vec0, float f) {
    const S* src = reinterpret_cast<const S*>(it.src & ~(uint64_t)15);
    T* dst = reinterpret_cast<T*>(it.dst & ~(uint64_t)15);
    Eight<S> in[kVecs];
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        const Place p = place(it, vec0 + i * kThreads + threadIdx.x);
        if (p.in) in[i] = load8(src + p.row * it.ld_src, p.col, it.cols);
    }
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        const Place p = place(it, vec0 + i * kThreads + threadIdx.x);
        if (!p.in) continue;
        float v[8];
        in[i].get(v);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= f;
        store8(dst + p.row * it.ld_dst, p.col, it.cols, v);
    }
}

__global__ __launch_bounds__(kThreads) void clip_kernel(ClipArgs A, Factor F) {
    // every workgroup adds the devices' sums, in group order
    double s = 0.0;
    for (int j = 0; j < F.nparts; ++j) s += *F.parts[j];
    const double norm = (double)F.scale * sqrt(s);
    const float f = (float)((double)F.scale *
                            (norm <= (double)F.max_norm ? 1.0 : (double)F.max_norm / norm));
    if (A.norm && blockIdx.x == 0 && threadIdx.x == 0) {
        A.norm[0] = (float)norm;
        A.norm[1] = f;
    }
    if (A.L.n == 0) return;
    const Item& it = A.L.t[find(A.L, blockIdx.x)];
    if (f == 1.f && it.src == it.dst && it.ld_src == it.ld_dst) return;    // in place already
    const int64_t vec0 = (int64_t)((int)blockIdx.x - it.first) * (kThreads * kVecs);
    if (it.src & 1) {
        if (it.dst & 1) scaled<float, float>(it, vec0, f);
        else scaled<float, uint16_t>(it, vec0, f);
    } else {
        if (it.dst & 1) scaled<uint16_t, float>(it, vec0, f);
        else scaled<uint16_t, uint16_t>(it, vec0, f);
    }
}

// The tensors as items: rows without gaps are one run.
struct Run {
    int64_t rows, cols, ld_src, ld_dst;
};
Run run_of(const GradView& g, bool with_dst) {
    const bool flat = g.rows <= 1 || (g.ld_src == g.cols && (!with_dst || g.ld_dst == g.cols));
    return flat ? Run{g.rows > 0 ? 1 : 0, g.rows * g.cols, 0, 0}
                : Run{g.rows, g.cols, g.ld_src, g.ld_dst};
}
int64_t blocks_of(const Run& r) {
    if (r.rows == 0 || r.cols == 0) return 0;
    return (r.rows * ((r.cols + 7) / 8) * 8 + kSpan - 1) / kSpan;
}

// Calls f(items, workgroups) for every launch.
template <class F>
hipError_t in_launches(int n, const GradView* g, bool with_dst, F&& f) {
    Items L;
    L.n = 0;
    int64_t blocks = 0;
    for (int i = 0; i < n; ++i) {
        const Run r = run_of(g[i], with_dst);
        const int64_t b = blocks_of(r);
        if (b == 0) continue;
        if (L.n == kItems || blocks + b > 0x7fffffff) {
            const hipError_t e = f(L, blocks);
            if (e != hipSuccess) return e;
            L.n = 0;
            blocks = 0;
        }
        Item& t = L.t[L.n++];
        t.src = reinterpret_cast<uint64_t>(g[i].src) | (g[i].src_f32 ? 1 : 0);
        t.dst = reinterpret_cast<uint64_t>(g[i].dst) | (g[i].dst_f32 ? 1 : 0);
        t.cols = r.cols;
        t.ld_src = (int32_t)r.ld_src;
        t.ld_dst = (int32_t)r.ld_dst;
        t.rows = (int32_t)r.rows;
        t.first = (int32_t)blocks;
        blocks += b;
    }
    return L.n ? f(L, blocks) : hipSuccess;
}

}  // namespace

int64_t grad_sum_blocks(int n, const GradView* g) {
    int64_t blocks = 0;
    for (int i = 0; i < n; ++i) blocks += blocks_of(run_of(g[i], false));
    return blocks;
}

hipError_t launch_grad_sq_sum(int n, const GradView* g, double* sum, double* ws, hipStream_t s) {
    int64_t done = 0;
    const hipError_t e = in_launches(n, g, false, [&](const Items& L, int64_t blocks) {
        sq_sum_kernel<<<dim3((unsigned)blocks), kThreads, 0, s>>>(L, ws + done);
        done += blocks;
        return hipGetLastError();
    });
    if (e != hipSuccess) return e;
    sq_join_kernel<<<1, kJoinThreads, 0, s>>>(ws, done, sum);
    return hipGetLastError();
}

hipError_t launch_grad_clip(int n, const GradView* g, int nparts, const double* const* parts,
                            float scale, float max_norm, float* norm, hipStream_t s) {
    Factor F = {};
    std::copy(parts, parts + nparts, F.parts);
    F.nparts = nparts;
    F.scale = scale;
    F.max_norm = max_norm;
    bool first = true;
    ClipArgs a;
    const hipError_t e = in_launches(n, g, true, [&](const Items& L, int64_t blocks) {
        a.L = L;
        a.norm = first ? norm : nullptr;
        first = false;
        clip_kernel<<<dim3((unsigned)blocks), kThreads, 0, s>>>(a, F);
        return hipGetLastError();
    });
    if (e != hipSuccess || !first) return e;
    a.L.n = 0;                                       // nothing to scale: the norm alone
    a.norm = norm;
    clip_kernel<<<1, 64, 0, s>>>(a, F);
    return hipGetLastError();
}

}  // namespace atp
