// Layer norm of rows, with the sum that feeds it, and its gradient.
//
//   s = x + add,  mu = mean(s),  r = 1 / sqrt(mean((s - mu)^2) + eps),
//   y = (s - mu) r w + b;
//   g = w dy,  xh = (s - mu) r,  dx = r (g - mean(g) - xh mean(g xh)) + d_res,
//   dw = sum over rows of dy xh,  db = sum over rows of dy.
//
// A row stays in registers between its two passes (mean, then centred squares: no
// difference of large sums), so every value is read and written once: the calls
// are bound by memory (4096 rows of 20480 columns with the sum: 120 us forward, 5.6
// TB/s, 155 backward, 4.3).  Up to 2048 columns a wave holds a row, eight consecutive
// values per lane and vector; wider rows take a workgroup of just as many waves as hold
// them, joined through LDS.
//
// Rows whose columns lie on several devices: each device gives the mean and the
// centred squares of its own columns (a row's two sums, in the backward), and
// the join walks the devices in group order, so all of them get the same bits.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "lds_dma.h"
#include "train_kernels.h"
#include "wave_ops.h"

namespace atp {
namespace {

using wave::Eight;
using wave::sum64;

constexpr int kRowsPerGroup = 4;         // rows of a workgroup whose waves hold one each
constexpr size_t kStageBytes = 160 * 1024 - 512;   // LDS beside the row sums

// How a row of `cols` is held: threads * nv lanes of eight values.  Backward of 4096 rows:
// of 2048 columns by waves 20.7 us, by workgroups 22.9; of 8192 with two vectors per lane
// 44, with four 66, which only the widest rows take.
struct Shape {
    bool one;                            // a wave per row
    int nv, threads;                     // vectors of a lane, threads of a row
};
Shape shape_of(int64_t cols) {
    const int64_t vecs = cols / 8;
    if (vecs <= 256) return Shape{true, vecs <= 64 ? 1 : vecs <= 128 ? 2 : 4, 64};
    const int nv = vecs <= 1280 ? 2 : 4;
    return Shape{false, nv, (int)((vecs + 64 * nv - 1) / (64 * nv)) * 64};
}

struct Args {
    int64_t tokens;
    int cols, nparts;
    float inv_total, eps, part_cols;
    const void* x; int64_t ldx;
    const uint16_t* add; int64_t ldadd;
    void* x_out; int64_t ldxo;
    const uint16_t *w, *b;
    float* stats;
    uint16_t* y; int64_t ldy;
    float *mean, *rstd;
    const float* parts[kMaxParts];
};

// Sum over the row's lanes.  red: 16 floats of LDS that no other sum of the same
// round uses.
template <bool ONE>
__device__ __forceinline__ float row_sum(float v, float* red, int waves) {
    v = sum64(v);
    if constexpr (ONE) return v;
    const int lane = threadIdx.x & 63;
    if (lane == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    const int i = lane & 15;
    float t = i < waves ? red[i] : 0.f;
    t = wave::dpp_add<0xb1>(t);
    t = wave::dpp_add<0x4e>(t);
    t = wave::dpp_add<0x141>(t);
    return wave::dpp_add<0x140>(t);
}

// A row's entry of every device's table: lane j holds device j's.
struct Pair {
    float a, b;
};
__device__ __forceinline__ Pair part_of(const float* const* parts, int n, int64_t row) {
    Pair p = {0.f, 0.f};
    const int j = threadIdx.x & 63;
    if (j < n) {
        const wave::f32x2 v = *reinterpret_cast<const wave::f32x2*>(parts[j] + 2 * row);
        p.a = v[0];
        p.b = v[1];
    }
    return p;
}
__device__ __forceinline__ float of_lane(float v, int j) {
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), j));
}

template <class T, int NV, bool ONE>
__global__ __launch_bounds__(ONE ? 64 * kRowsPerGroup : 1024) void norm_fwd_kernel(Args A) {
    __shared__ float red[2][16];
    const int l = ONE ? (int)(threadIdx.x & 63) : (int)threadIdx.x;
    const int per = ONE ? 64 : (int)blockDim.x, waves = per >> 6;
    const int64_t row = ONE ? (int64_t)blockIdx.x * kRowsPerGroup + (threadIdx.x >> 6)
                            : (int64_t)blockIdx.x;
    if (row >= A.tokens) return;         // whole waves, and no barrier follows for them
    const T* x = static_cast<const T*>(A.x) + row * A.ldx;
    const Pair part = part_of(A.parts, A.nparts, row);
    Eight<T> in[NV];
    float v[NV][8];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * per + l) * 8;
        if (c < A.cols) in[i].load(x + c);
    }
    if (A.add) {
        const uint16_t* add = A.add + row * A.ldadd;
        T* xo = static_cast<T*>(A.x_out) + row * A.ldxo;
        Eight<uint16_t> more[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * per + l) * 8;
            if (c < A.cols) more[i].load(add + c);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * per + l) * 8;
            if (c >= A.cols) continue;
            float a[8], b[8];
            in[i].get(a);
            more[i].get(b);
#pragma unroll
            for (int e = 0; e < 8; ++e) a[e] += b[e];
            in[i].set(a);                // what is normed is the sum as it is stored
            in[i].store(xo + c);
        }
    }
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if ((i * per + l) * 8 < A.cols) {
            in[i].get(v[i]);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += v[i][e];
        }
    }
    float mean = 0.f, m2 = 0.f;
    if (A.nparts == 0) {
        // divided, not by a rounded reciprocal: rows of one value have it as their mean
        mean = row_sum<ONE>(sum, red[0], waves) / A.part_cols;
        float sq = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if ((i * per + l) * 8 < A.cols) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float d = v[i][e] - mean;
                    sq += d * d;
                }
            }
        }
        m2 = row_sum<ONE>(sq, red[1], waves);
        if (A.stats) {
            if (l == 0) {
                A.stats[2 * row] = mean;
                A.stats[2 * row + 1] = m2;
            }
            return;
        }
    } else {
        // equal shards: the mean of the means; the squares about it
        for (int j = 0; j < A.nparts; ++j) mean += of_lane(part.a, j);
        mean /= (float)A.nparts;
        for (int j = 0; j < A.nparts; ++j) {
            const float d = of_lane(part.a, j) - mean;
            m2 += of_lane(part.b, j) + A.part_cols * d * d;
        }
    }
    const float r = 1.f / sqrtf(m2 * A.inv_total + A.eps);
    if (l == 0) {
        A.mean[row] = mean;
        A.rstd[row] = r;
    }
    uint16_t* y = A.y + row * A.ldy;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * per + l) * 8;
        if (c >= A.cols) continue;
        float w[8], b[8];
        Eight<uint16_t> t;
        if (A.w) {
            t.load(A.w + c);
            t.get(w);
        }
        if (A.b) {
            t.load(A.b + c);
            t.get(b);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float o = (v[i][e] - mean) * r;
            if (A.w) o *= w[e];
            if (A.b) o += b[e];
            v[i][e] = o;
        }
        t.set(v[i]);
        t.store(y + c);
    }
}

__device__ __forceinline__ void hold(Eight<uint16_t>& v) { asm volatile("" : "+v"(v.w)); }
__device__ __forceinline__ void hold(Eight<float>& v) { asm volatile("" : "+v"(v.a), "+v"(v.b)); }

struct BwdArgs {
    int64_t tokens;
    int cols, nparts;
    float inv_total;
    const void* x; int64_t ldx;
    const uint16_t* w;
    const float *mean, *rstd;
    const uint16_t* dy; int64_t lddy;
    float* sums;
    const void* dres; int64_t lddres;
    void* dx; int64_t lddx;
    uint16_t* dadd; int64_t lddadd;
    float* part;                         // [workgroups][2][cols], nullable
    const float* parts[kMaxParts];
};

// A workgroup walks rows gridDim.x apart and keeps its lanes' share of both
// column sums in registers; it leaves one row of partial sums, which
// column_sum_kernel adds in order.  The grid is a function of the sizes alone, so
// the sums are too.  A row's values come while the row before is worked on: into
// registers where a wave holds a row, else (STAGED) by copies into LDS, where each
// wave reads back what it copied itself, because the registers of one or two
// workgroups per CU do not hold two wide rows beside the column sums.  The copies of
// x and dy are begun as soon as the row before is in registers and waited for
// before its results are stored, so that nothing waits for the stores; d_res is
// read from LDS where it is added, and its next copy begun behind that.
template <class T, int NV, bool ONE, int THREADS, bool STAGED>
__global__ __launch_bounds__(THREADS) void norm_bwd_kernel(BwdArgs A) {
    constexpr bool kAhead = ONE && (sizeof(T) == 2 || NV <= 2);
    constexpr int kPlanes = sizeof(T) / 2;           // 16-byte pieces of eight values
    // the weights stay in registers where there are some for them, else come from L2
    constexpr bool kHoldW = NV <= 2 || ONE || (sizeof(T) == 2 && THREADS <= 640);
    __shared__ float red[2][2][16];
    extern __shared__ float join[];      // ONE: [3 waves][cols]; STAGED: planes of the row
    const int l = ONE ? (int)(threadIdx.x & 63) : (int)threadIdx.x;
    const int per = ONE ? 64 : (int)blockDim.x, waves = per >> 6;
    const int mine = ONE ? (int)(threadIdx.x >> 6) : 0;
    const int64_t step = (int64_t)gridDim.x * (ONE ? kRowsPerGroup : 1);
    float dw[NV][8], db[NV][8];
    Eight<uint16_t> w[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * per + l) * 8;
        if (kHoldW && A.w && c < A.cols) w[i].load(A.w + c);
        else w[i].w = wave::u32x4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};   // ones
#pragma unroll
        for (int e = 0; e < 8; ++e) dw[i][e] = db[i][e] = 0.f;
    }
    auto weight = [&](int i, float* v) {
        if constexpr (!kHoldW) {
            if (A.w) {
                Eight<uint16_t> t;
                t.load(A.w + (i * per + l) * 8);
                t.get(v);
                return;
            }
        }
        w[i].get(v);
    };
    Eight<T> xs[NV], xn[NV], res[NV];
    Eight<uint16_t> gs[NV], gn[NV];
    auto load = [&](int64_t row, Eight<T> (&x)[NV], Eight<uint16_t> (&g)[NV]) {
        const T* xr = static_cast<const T*>(A.x) + row * A.ldx;
        const uint16_t* gr = A.dy + row * A.lddy;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * per + l) * 8;
            if (c < A.cols) {
                x[i].load(xr + c);
                g[i].load(gr + c);
            }
        }
    };
    auto load_res = [&](int64_t row) {
        const T* dr = static_cast<const T*>(A.dres) + row * A.lddres;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * per + l) * 8;
            if (c < A.cols) res[i].load(dr + c);
        }
    };
    // plane p of vector i: a wave's 64 lanes one behind the other; x, dy, then d_res
    uint16_t* slots = reinterpret_cast<uint16_t*>(join);
    const int w0 = __builtin_amdgcn_readfirstlane(l & ~63);
    auto slot = [&](int p, int i) { return slots + ((p * NV + i) * per + w0) * 8; };
    auto words = [](const void* base, int64_t bytes) {   // the same in every lane
        dma::u32x4 r = dma::rsrc_words(base, bytes);
#pragma unroll
        for (int k = 0; k < 4; ++k) r[k] = (uint32_t)__builtin_amdgcn_readfirstlane((int)r[k]);
        return r;
    };
    auto stage = [&](int64_t row) {
        const dma::u32x4 rx =
            words(static_cast<const T*>(A.x) + row * A.ldx, A.cols * sizeof(T));
        const dma::u32x4 rg = words(A.dy + row * A.lddy, A.cols * 2);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const uint32_t at = (uint32_t)(i * per + l) * 16;     // beyond the row: zeros
#pragma unroll
            for (int p = 0; p < kPlanes; ++p)
                dma::lds_dma16(rx, slot(p, i), at * kPlanes + 16 * p, 0u);
            dma::lds_dma16(rg, slot(kPlanes, i), at, 0u);
        }
    };
    auto stage_res = [&](int64_t row) {
        const dma::u32x4 rr =
            words(static_cast<const T*>(A.dres) + row * A.lddres, A.cols * sizeof(T));
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int p = 0; p < kPlanes; ++p)
                dma::lds_dma16(rr, slot(kPlanes + 1 + p, i),
                               (uint32_t)(i * per + l) * 16 * kPlanes + 16 * p, 0u);
    };
    auto piece = [&](int p, int i) {
        return *reinterpret_cast<const wave::u32x4*>(slot(p, i) + (l & 63) * 8);
    };
    auto staged = [&](int p, int i, Eight<T>& v) {
        if constexpr (sizeof(T) == 2) {
            v.w = piece(p, i);
        } else {
            v.a = __builtin_bit_cast(wave::f32x4, piece(p, i));
            v.b = __builtin_bit_cast(wave::f32x4, piece(p + 1, i));
        }
    };
    int64_t row = (int64_t)blockIdx.x * (ONE ? kRowsPerGroup : 1) + mine;
    if (kAhead && row < A.tokens) load(row, xs, gs);
    if (STAGED && row < A.tokens) {
        stage(row);
        if (A.dres) stage_res(row);
        dma::wait_vmcnt<0>();
    }
    for (int turn = 0; row < A.tokens; row += step, turn ^= 1) {
        if constexpr (STAGED) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                staged(0, i, xs[i]);
                gs[i].w = piece(kPlanes, i);
            }
            // read before the next row's copies may land
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            if (row + step < A.tokens) stage(row + step);
        } else {
            if (!kAhead) load(row, xs, gs);
            if (A.dres) load_res(row);
        }
        const float mean = A.mean[row], r = A.rstd[row];
        const Pair part = part_of(A.parts, A.nparts, row);
        float c1 = 0.f, c2 = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if ((i * per + l) * 8 >= A.cols) continue;
            float v[8], g[8], wv[8];
            xs[i].get(v);
            gs[i].get(g);
            weight(i, wv);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float xh = (v[e] - mean) * r;
                dw[i][e] += g[e] * xh;
                db[i][e] += g[e];
                const float gw = g[e] * wv[e];
                c1 += gw;
                c2 += gw * xh;
            }
            if constexpr (!ONE) __builtin_amdgcn_sched_barrier(0);   // one vector at a time
        }
        if (kAhead && row + step < A.tokens) load(row + step, xn, gn);
        // the packed values alone live on: what was unpacked above is unpacked again below
        // (kept, it would take twice the registers)
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            hold(xs[i]);
            hold(gs[i]);
            if constexpr (kHoldW) hold(w[i]);
        }
        if (A.nparts == 0) {
            // both sums under one barrier
            c1 = sum64(c1);
            c2 = sum64(c2);
            if constexpr (!ONE) {
                const int lane = threadIdx.x & 63;
                if (lane == 0) {
                    red[turn][0][threadIdx.x >> 6] = c1;
                    red[turn][1][threadIdx.x >> 6] = c2;
                }
                // for LDS alone: the row's loads and copies go on
                asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
                const int k = lane & 15;
                c1 = k < waves ? red[turn][0][k] : 0.f;
                c2 = k < waves ? red[turn][1][k] : 0.f;
                c1 = wave::dpp_add<0xb1>(c1);
                c2 = wave::dpp_add<0xb1>(c2);
                c1 = wave::dpp_add<0x4e>(c1);
                c2 = wave::dpp_add<0x4e>(c2);
                c1 = wave::dpp_add<0x141>(c1);
                c2 = wave::dpp_add<0x141>(c2);
                c1 = wave::dpp_add<0x140>(c1);
                c2 = wave::dpp_add<0x140>(c2);
            }
            if (A.sums && l == 0) {
                A.sums[2 * row] = c1;
                A.sums[2 * row + 1] = c2;
            }
        } else {
            c1 = c2 = 0.f;
            for (int j = 0; j < A.nparts; ++j) {
                c1 += of_lane(part.a, j);
                c2 += of_lane(part.b, j);
            }
        }
        c1 *= A.inv_total;
        c2 *= A.inv_total;
        auto gradient = [&](int i, float* g) {
            float v[8], wv[8];
            xs[i].get(v);
            gs[i].get(g);
            weight(i, wv);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                g[e] = r * (g[e] * wv[e] - c1 - (v[e] - mean) * r * c2);
            if (A.dres) {
                if constexpr (STAGED) {
                    Eight<T> t;
                    staged(kPlanes + 1, i, t);
                    t.get(v);
                } else {
                    res[i].get(v);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) g[e] += v[e];
            }
        };
        if constexpr (STAGED) dma::wait_vmcnt<0>();
        if (!A.sums) {
            T* dx = static_cast<T*>(A.dx) + row * A.lddx;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (i * per + l) * 8;
                if (c >= A.cols) continue;
                float g[8];
                gradient(i, g);
                Eight<T> o;
                o.set(g);
                o.store(dx + c);
                if (A.dadd) {
                    Eight<uint16_t> o16;
                    o16.set(g);
                    o16.store(A.dadd + row * A.lddadd + c);
                }
                if constexpr (!ONE) __builtin_amdgcn_sched_barrier(0);
            }
        }
        if constexpr (STAGED) {
            if (A.dres && row + step < A.tokens) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                stage_res(row + step);
            }
        }
        if (kAhead) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                xs[i] = xn[i];
                gs[i] = gn[i];
            }
        }
    }
    if (!A.part) return;
    float* out = A.part + (int64_t)blockIdx.x * 2 * A.cols;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        if constexpr (ONE) {
            // the waves' sums, in order
            if (which) __syncthreads();
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (i * per + l) * 8;
                if (mine && c < A.cols) {
                    Eight<float> t;
                    t.set(which ? db[i] : dw[i]);
                    t.store(join + (mine - 1) * A.cols + c);
                }
            }
            __syncthreads();
        }
        if (mine) continue;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * per + l) * 8;
            if (c >= A.cols) continue;
            float s[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) s[e] = which ? db[i][e] : dw[i][e];
            if constexpr (ONE) {
#pragma unroll
                for (int k = 0; k < kRowsPerGroup - 1; ++k) {
                    Eight<float> t;
                    t.load(join + k * A.cols + c);
                    float u[8];
                    t.get(u);
#pragma unroll
                    for (int e = 0; e < 8; ++e) s[e] += u[e];
                }
            }
            Eight<float> t;
            t.set(s);
            t.store(out + which * A.cols + c);
        }
    }
}

// Column sums of n rows of 2 cols partials: C columns per workgroup, 1024 / C runs of
// rows (every 1024 / C-th), joined in order.  16 columns where 64 would leave CUs idle:
// 626 rows of 2048 columns 3.9 us, 5.3 with 64.
constexpr int kSumThreads = 1024;
template <int C>
__global__ __launch_bounds__(kSumThreads) void column_sum_kernel(const float* part, int n,
                                                                 int cols, float* dw, float* db) {
    constexpr int G = kSumThreads / C;
    __shared__ float red[G][C + 1];
    const int c = threadIdx.x % C, g = threadIdx.x / C;
    const int64_t col = (int64_t)blockIdx.x * C + c;
    float sum = 0.f;
    if (col < 2 * (int64_t)cols) {
#pragma unroll 8
        for (int i = g; i < n; i += G) sum += part[(int64_t)i * 2 * cols + col];
    }
    red[g][c] = sum;
    __syncthreads();
    if (g != 0 || col >= 2 * (int64_t)cols) return;
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < G; ++i) sum += red[i][c];
    if (col < cols) {
        if (dw) dw[col] = sum;
    } else if (db) {
        db[col - cols] = sum;
    }
}

// Workgroups of the backward: enough to fill the chip, each with four rows at least (eight
// where its waves hold one each), since it leaves a row of partial sums, 8 bytes a
// column against the 8 to 14 of a row, and all with the same number of visits.
struct Groups {
    int64_t rows, most, visits;          // rows at a time, workgroups at most, visits at least
};
Groups groups_of(int64_t cols) {
    const Shape sh = shape_of(cols);
    return Groups{sh.one ? kRowsPerGroup : 1,
                  256 * (sh.one ? 4 : std::max(1, 1024 / sh.threads)), sh.one ? 2 : 4};
}
int64_t bwd_groups(int64_t tokens, int64_t cols) {
    const Groups g = groups_of(cols);
    const int64_t visits =
        std::max((tokens + g.most * g.rows - 1) / (g.most * g.rows), g.visits);
    return (tokens + visits * g.rows - 1) / (visits * g.rows);
}

template <class T, int NV, bool ONE>
void fwd(const Args& a, int64_t grid, int threads, hipStream_t s) {
    norm_fwd_kernel<T, NV, ONE><<<dim3((unsigned)grid), threads, 0, s>>>(a);
}
template <class T, int NV, bool ONE, int THREADS>
void bwd(const BwdArgs& a, int64_t grid, int threads, hipStream_t s) {
    if constexpr (ONE) {
        const size_t lds = a.part ? sizeof(float) * (kRowsPerGroup - 1) * a.cols : 0;
        norm_bwd_kernel<T, NV, true, THREADS, false>
            <<<dim3((unsigned)grid), threads, lds, s>>>(a);
    } else {
        const size_t lds = (size_t)threads * NV * (8 * (a.dres ? 2 : 1) * sizeof(T) + 16);
        if (lds <= kStageBytes)
            norm_bwd_kernel<T, NV, false, THREADS, true>
                <<<dim3((unsigned)grid), threads, lds, s>>>(a);
        else
            norm_bwd_kernel<T, NV, false, THREADS, false>
                <<<dim3((unsigned)grid), threads, 0, s>>>(a);
    }
}

template <class T>
void fwd_of(const Shape& sh, const Args& a, hipStream_t s) {
    const int64_t rows = sh.one ? kRowsPerGroup : 1;
    const int64_t grid = (a.tokens + rows - 1) / rows;
    const int thr = sh.one ? 64 * kRowsPerGroup : sh.threads;
    if (sh.one) {
        if (sh.nv == 1) fwd<T, 1, true>(a, grid, thr, s);
        else if (sh.nv == 2) fwd<T, 2, true>(a, grid, thr, s);
        else fwd<T, 4, true>(a, grid, thr, s);
    } else if (sh.nv == 2) {
        fwd<T, 2, false>(a, grid, thr, s);
    } else {
        fwd<T, 4, false>(a, grid, thr, s);
    }
}
template <class T>
void bwd_of(const Shape& sh, const BwdArgs& a, int64_t grid, hipStream_t s) {
    const int thr = sh.one ? 64 * kRowsPerGroup : sh.threads;
    if (sh.one) {
        if (sh.nv == 1) bwd<T, 1, true, 256>(a, grid, thr, s);
        else if (sh.nv == 2) bwd<T, 2, true, 256>(a, grid, thr, s);
        else bwd<T, 4, true, 256>(a, grid, thr, s);
    } else if (sh.nv == 2) {
        bwd<T, 2, false, 640>(a, grid, thr, s);
    } else if (sh.threads <= 640) {
        bwd<T, 4, false, 640>(a, grid, thr, s);
    } else {
        bwd<T, 4, false, 1024>(a, grid, thr, s);
    }
}

}  // namespace

// Enough for every smaller number of tokens too: one visit more for all leaves fewer
// workgroups, so what counts is the most that there are with the fewest visits.
int64_t layer_norm_ws_floats(int64_t tokens, int64_t cols) {
    const Groups g = groups_of(cols);
    return std::min(g.most, (tokens + g.visits * g.rows - 1) / (g.visits * g.rows)) * 2 * cols;
}

bool layer_norm_fits(int64_t tokens, int64_t cols) {
    return fits_launch(tokens, shape_of(cols).threads);
}

hipError_t launch_layer_norm(const LayerNormProblem& p, hipStream_t s) {
    if (p.tokens == 0) return hipSuccess;
    Args a = {};
    a.tokens = p.tokens;
    a.cols = (int)p.cols;
    a.nparts = p.nparts;
    a.inv_total = 1.f / (float)(p.cols * std::max(1, p.nparts));
    a.part_cols = (float)p.cols;
    a.eps = p.eps;
    a.x = p.x; a.ldx = p.ldx;
    a.add = p.add; a.ldadd = p.ldadd;
    a.x_out = p.x_out; a.ldxo = p.ldxo;
    a.w = p.weight;
    a.b = p.bias;
    a.stats = p.stats_out;
    a.y = p.y; a.ldy = p.ldy;
    a.mean = p.mean;
    a.rstd = p.rstd;
    std::copy(p.parts, p.parts + p.nparts, a.parts);
    const Shape sh = shape_of(p.cols);
    if (p.f32) fwd_of<float>(sh, a, s);
    else fwd_of<uint16_t>(sh, a, s);
    return hipGetLastError();
}

hipError_t launch_layer_norm_bwd(const LayerNormBwdProblem& p, hipStream_t s) {
    const bool weights = p.dw || p.db;
    int64_t grid = 0;
    if (p.tokens > 0) {
        BwdArgs a = {};
        a.tokens = p.tokens;
        a.cols = (int)p.cols;
        a.nparts = p.nparts;
        a.inv_total = 1.f / (float)(p.cols * std::max(1, p.nparts));
        a.x = p.x; a.ldx = p.ldx;
        a.w = p.weight;
        a.mean = p.mean;
        a.rstd = p.rstd;
        a.dy = p.dy; a.lddy = p.lddy;
        a.sums = p.sums_out;
        a.dres = p.dres; a.lddres = p.lddres;
        a.dx = p.dx; a.lddx = p.lddx;
        a.dadd = p.dadd; a.lddadd = p.lddadd;
        a.part = weights ? p.ws : nullptr;
        std::copy(p.parts, p.parts + p.nparts, a.parts);
        grid = bwd_groups(p.tokens, p.cols);
        const Shape sh = shape_of(p.cols);
        if (p.f32) bwd_of<float>(sh, a, grid, s);
        else bwd_of<uint16_t>(sh, a, grid, s);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (!weights) return hipSuccess;
    const int cols = (int)p.cols;
    if (2 * cols < 64 * 256)
        column_sum_kernel<16><<<dim3((unsigned)((2 * cols + 15) / 16)), kSumThreads, 0, s>>>(
            p.ws, (int)grid, cols, p.dw, p.db);
    else
        column_sum_kernel<64><<<dim3((unsigned)((2 * cols + 63) / 64)), kSumThreads, 0, s>>>(
            p.ws, (int)grid, cols, p.dw, p.db);
    return hipGetLastError();
}

}  // namespace atp
