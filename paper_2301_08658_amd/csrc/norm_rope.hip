// Norms of queries and keys for each head with the position rotation in the
// same pass: y = R(p) (w o x r), r = 1 / sqrt(mean(x^2) + eps), its gradient,
// and the form that writes keys and values of new tokens into a paged cache.
//
// Sixteen lanes (a "worker", four per wave) hold one head row of 128 values,
// eight each, so the sum of squares is four row rotations within the lanes and
// nothing passes through LDS.  A rotation's pairs (i, i + rot / 2) are kept
// inside one lane: lane l < rot / 8 holds values [4 l, 4 l + 4) and [rot / 2 +
// 4 l, ..), the other lanes 8 consecutive ones, and with interleaved pairs all
// lanes do.  Every lane of a worker then needs the same four angles 4 l .. 4 l
// + 3 of its token for every head, and they are formed once per worker.
//
// Angles: position * inv_freq is formed in 64 bits and reduced to a fraction
// of a turn there; 32 bits would lose 0.06 radians at position 10^6.  The hardware's
// sine and cosine take turns and are off by 1.3e-7 at most (measured over half a turn
// either way; the library's sincospi by 5e-8, at ten times the instructions, which
// is what bounded the kernels).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "cache_kernels.h"
#include "epilogue_math.h"

namespace atp {
namespace {

constexpr int kThreads = 256;
constexpr int kWorkers = kThreads / 16;      // workers of a workgroup

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

struct Args {
    const uint16_t *x, *dy;
    uint16_t* y;
    int64_t ldx, lddy, ldy;
    const uint16_t *qw, *kw;
    const float* inv_freq;
    const int32_t* pos;
    int64_t tokens, seq;
    float eps;
    int norm, rot, heads, per_kv, group;   // heads: kv_heads * per_kv, per_kv = group + 2
    int parts, step_kv, step_r;            // a worker's next head: parts = step_kv * per_kv + step_r
    int copy_v;
    int64_t stride;                        // tokens between a worker's visits (backward)
    float* part;                           // weight-gradient partials, nullable
    CacheView cache;
    BatchView batch;
};

// The sum over the 16 lanes of a worker, the same bits in each: every step adds
// the value of the lane 8, 4, 2, 1 places on, and both partners add the same two.
__device__ __forceinline__ float sum16(float v) {
    auto ror = [](float f, auto ctrl) {
        const int i = __builtin_bit_cast(int, f);
        return __builtin_bit_cast(float,
                                  __builtin_amdgcn_update_dpp(i, i, decltype(ctrl)::value, 0xf, 0xf,
                                                              false));
    };
    v += ror(v, std::integral_constant<int, 0x128>{});   // row_ror:8
    v += ror(v, std::integral_constant<int, 0x124>{});
    v += ror(v, std::integral_constant<int, 0x122>{});
    v += ror(v, std::integral_constant<int, 0x121>{});
    return v;
}

__device__ __forceinline__ void widen(u32x2 a, float* f) {
    f[0] = __uint_as_float(a[0] << 16);
    f[1] = __uint_as_float(a[0] & 0xffff0000u);
    f[2] = __uint_as_float(a[1] << 16);
    f[3] = __uint_as_float(a[1] & 0xffff0000u);
}
__device__ __forceinline__ u32x2 narrow(const float* f) {   // round to nearest even
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const f32x2 a = {f[0], f[1]}, b = {f[2], f[3]};
    return u32x2{__builtin_bit_cast(uint32_t, __builtin_convertvector(a, bf16x2)),
                 __builtin_bit_cast(uint32_t, __builtin_convertvector(b, bf16x2))};
}

// A lane's place in a head row and the cosines and sines of its four angles.
template <bool INTER>
struct Lane {
    int a, b;          // first value of its two runs of four
    bool turned;       // its values are rotated
    float c[4], s[4];
    __device__ __forceinline__ void place(int l, int rot) {
        turned = l < rot / 8;
        const bool split = !INTER && turned;
        a = split ? 4 * l : 8 * l;
        b = split ? rot / 2 + 4 * l : 8 * l + 4;
    }
    __device__ __forceinline__ void angles(int l, const float* inv_freq, int position) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            c[e] = 1.f;
            s[e] = 0.f;
            if (turned) {
                const double t = (double)position * ((double)inv_freq[4 * l + e] *
                                                     0.15915494309189533577);   // 1 / (2 pi)
                const float f = (float)(t - rint(t));
                s[e] = __builtin_amdgcn_sinf(f);
                c[e] = __builtin_amdgcn_cosf(f);
            }
        }
    }
    // v[0..3] and v[4..7]: the two runs; sign -1 turns back
    __device__ __forceinline__ void turn(float* v, float sign) const {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = INTER ? 2 * e : e, j = INTER ? 2 * e + 1 : e + 4;
            const float p = v[i], q = v[j], sn = sign * s[e];
            v[i] = p * c[e] - q * sn;
            v[j] = q * c[e] + p * sn;
        }
    }
    __device__ __forceinline__ void load(const uint16_t* row, u32x2& ra, u32x2& rb) const {
        ra = *reinterpret_cast<const u32x2*>(row + a);
        rb = *reinterpret_cast<const u32x2*>(row + b);
    }
    __device__ __forceinline__ void store(uint16_t* row, const u32x2& ra, const u32x2& rb) const {
        *reinterpret_cast<u32x2*>(row + a) = ra;
        *reinterpret_cast<u32x2*>(row + b) = rb;
    }
    __device__ __forceinline__ void weight(const uint16_t* w, float* f) const {
        if (w) {
            u32x2 ra, rb;
            load(w, ra, rb);
            widen(ra, f);
            widen(rb, f + 4);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = 1.f;
        }
    }
};

__device__ __forceinline__ int position_of(const Args& A, int64_t t) {
    if (!A.rot) return 0;
    return A.pos ? A.pos[t] : (int)(t % A.seq);
}

// The number of entries of the ascending list v[0 .. n) that are <= t: a search
// in sixteenths by the lanes of a worker (two steps for up to 256 entries).
// Every step shrinks len, whatever the list holds.
__device__ __forceinline__ int count_upto(const int32_t* v, int n, int64_t t, int lane) {
    const int l = lane & 15;
    int lo = 0, len = n;
    while (len > 0) {
        const int step = (len + 15) >> 4;
        const bool in = l * step < len;
        const bool le = in && v[lo + min((l + 1) * step, len) - 1] <= t;
        const uint64_t votes = __builtin_amdgcn_ballot_w64(le);
        const int c = __popcll((votes >> (lane & 48)) & 0xffffull);
        const int adv = min(c * step, len);
        lo += adv;
        if (step == 1) break;
        len = min(step, len - adv) - 1;     // the next sixteenth's last entry is above t
    }
    return lo;
}

// A worker takes heads part, part + parts, .. of one token, four loads in
// flight; it runs at the rate of a copy (reads the row once, writes it once).
template <bool INTER, bool CACHED>
__global__ __launch_bounds__(kThreads) void norm_rope_kernel(Args A) {
    const int lane = threadIdx.x & 63, l = lane & 15;
    const int64_t w = (int64_t)blockIdx.x * kWorkers + threadIdx.x / 16;
    const int64_t t = w / A.parts;
    const int part = (int)(w - t * A.parts);
    if (t >= A.tokens) return;

    // the first heads are asked for before the token's place is looked up
    Lane<INTER> ln;
    ln.place(l, A.rot);
    const uint16_t* xrow = A.x + t * A.ldx;
    uint16_t* yrow = A.y + t * A.ldy;
    constexpr int U = 4;
    u32x2 ra[U], rb[U];
    auto load = [&](int h0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int h = h0 + u * A.parts;
            if (h < A.heads) ln.load(xrow + (int64_t)h * kHead, ra[u], rb[u]);
        }
    };
    load(part);

    int position = 0;
    uint16_t *kdst = nullptr, *vdst = nullptr;      // the token's place of key head 0
    if constexpr (CACHED) {
        const int s = count_upto(A.batch.cu, A.batch.n_seqs + 1, t, lane) - 1;
        if (s < 0 || s >= A.batch.n_seqs) return;    // a padding row
        const int64_t at = (int64_t)max(A.batch.ctx[s], 0) + (t - A.batch.cu[s]);
        position = A.pos ? A.pos[t] : (int)at;
        // (a list that does not ascend can put a token before its sequence)
        const int64_t col = at >> A.cache.page_shift;
        const int page = col >= 0 && col < A.batch.max_pages
                             ? A.batch.table[s * A.batch.ld_table + col] : -1;
        if (page >= 0 && page < A.cache.n_pages) {
            const int64_t slot = at & ((1 << A.cache.page_shift) - 1);
            const int64_t half = (int64_t)A.cache.kv_heads << A.cache.page_shift;
            kdst = A.cache.pages + ((int64_t)page * 2 * half + slot) * kHead;
            vdst = kdst + half * kHead;
        }
    } else {
        position = position_of(A, t);
    }
    float wq[8], wk[8];
    ln.weight(A.qw, wq);
    ln.weight(A.kw, wk);
    ln.angles(l, A.inv_freq, position);

    int kv = part / A.per_kv, r = part - kv * A.per_kv;
    for (int h0 = part; h0 < A.heads; h0 += U * A.parts) {
        if (h0 != part) load(h0);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int h = h0 + u * A.parts;
            if (h >= A.heads) break;
            if (r <= A.group) {
                float v[8];
                widen(ra[u], v);
                widen(rb[u], v + 4);
                if (A.norm) {
                    float ss = 0.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) ss += v[e] * v[e];
                    const float rs = 1.f / sqrtf(sum16(ss) * (1.f / kHead) + A.eps);
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = v[e] * rs * (r < A.group ? wq[e] : wk[e]);
                }
                if (ln.turned) ln.turn(v, 1.f);
                ra[u] = narrow(v);
                rb[u] = narrow(v + 4);
            }
            if constexpr (CACHED) {
                const int64_t row = ((int64_t)kv << A.cache.page_shift) * kHead;
                if (r < A.group)
                    ln.store(yrow + ((int64_t)kv * A.group + r) * kHead, ra[u], rb[u]);
                else if (kdst)
                    ln.store((r == A.group ? kdst : vdst) + row, ra[u], rb[u]);
            } else if (r <= A.group || A.copy_v) {
                ln.store(yrow + (int64_t)h * kHead, ra[u], rb[u]);
            }
            kv += A.step_kv;
            r += A.step_r;
            if (r >= A.per_kv) {
                r -= A.per_kv;
                ++kv;
            }
        }
    }
}

// dx = r (g - x r mean(g o x r)), g = w o (dy turned back); dw = sum of
// (dy turned back) o x r.  A worker walks tokens `stride` apart and keeps its lanes'
// share of both weight gradients in registers;
// the workgroup adds its workers in order and leaves 256 partial sums, which
// weight_sum_kernel adds in order.  The grid is a function of the sizes alone,
// so the sums are too.
template <bool INTER>
__global__ __launch_bounds__(kThreads) void norm_rope_bwd_kernel(Args A) {
    __shared__ float red[kWorkers][2 * kHead];
    const int lane = threadIdx.x & 63, l = lane & 15;
    const int64_t w = (int64_t)blockIdx.x * kWorkers + threadIdx.x / 16;
    const int part = (int)(w % A.parts);
    Lane<INTER> ln;
    ln.place(l, A.rot);
    float wq[8], wk[8], gq[8], gk[8];
    ln.weight(A.qw, wq);
    ln.weight(A.kw, wk);
#pragma unroll
    for (int e = 0; e < 8; ++e) gq[e] = gk[e] = 0.f;

    // workers past the last whole token slot have nothing
    for (int64_t t = w / A.parts; t < A.tokens && w / A.parts < A.stride; t += A.stride) {
        ln.angles(l, A.inv_freq, position_of(A, t));
        const uint16_t* xrow = A.x + t * A.ldx;
        const uint16_t* grow = A.dy + t * A.lddy;
        uint16_t* drow = A.y + t * A.ldy;
        int r = part % A.per_kv;
        constexpr int U = 2;
        for (int h0 = part; h0 < A.heads; h0 += U * A.parts) {
            u32x2 xa[U], xb[U], da[U], db[U];
            int ru[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int h = h0 + u * A.parts;
                ru[u] = r;
                r += A.step_r;
                if (r >= A.per_kv) r -= A.per_kv;
                if (h >= A.heads) continue;
                if (A.norm && ru[u] <= A.group) ln.load(xrow + (int64_t)h * kHead, xa[u], xb[u]);
                if (ru[u] <= A.group || A.copy_v)
                    ln.load(grow + (int64_t)h * kHead, da[u], db[u]);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int h = h0 + u * A.parts;
                if (h >= A.heads) break;
                const bool key = ru[u] == A.group;
                if (ru[u] <= A.group) {
                    float g[8];
                    widen(da[u], g);
                    widen(db[u], g + 4);
                    if (ln.turned) ln.turn(g, -1.f);
                    if (A.norm) {
                        float v[8];
                        widen(xa[u], v);
                        widen(xb[u], v + 4);
                        float ss = 0.f;
#pragma unroll
                        for (int e = 0; e < 8; ++e) ss += v[e] * v[e];
                        const float rs = 1.f / sqrtf(sum16(ss) * (1.f / kHead) + A.eps);
                        float dot = 0.f;
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            v[e] *= rs;
                            const float gv = g[e] * v[e];
                            if (key) gk[e] += gv;
                            else gq[e] += gv;
                            g[e] *= key ? wk[e] : wq[e];
                            dot += g[e] * v[e];
                        }
                        dot = sum16(dot) * (1.f / kHead);
#pragma unroll
                        for (int e = 0; e < 8; ++e) g[e] = rs * (g[e] - v[e] * dot);
                    }
                    da[u] = narrow(g);
                    db[u] = narrow(g + 4);
                }
                if (ru[u] <= A.group || A.copy_v)
                    ln.store(drow + (int64_t)h * kHead, da[u], db[u]);
            }
        }
    }
    if (!A.part) return;
    const int wk_ = threadIdx.x / 16;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int d = e < 4 ? ln.a + e : ln.b + e - 4;
        red[wk_][d] = gq[e];
        red[wk_][kHead + d] = gk[e];
    }
    __syncthreads();
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < kWorkers; ++i) sum += red[i][threadIdx.x];
    A.part[(int64_t)blockIdx.x * 2 * kHead + threadIdx.x] = sum;
}

// Column sums of n rows of 256 partials: 16 columns per workgroup, 64 runs of rows
// (every 64th), joined in order.  16 runs and one load under way took 20 us for
// 1024 rows.
constexpr int kSumThreads = 1024;
__global__ __launch_bounds__(kSumThreads) void weight_sum_kernel(const float* part, int n,
                                                                 float* dqw, float* dkw) {
    constexpr int G = kSumThreads / 16;
    __shared__ float red[G][17];
    const int c = threadIdx.x & 15, g = threadIdx.x / 16;
    const int col = blockIdx.x * 16 + c;
    float sum = 0.f;
#pragma unroll 8
    for (int i = g; i < n; i += G) sum += part[(int64_t)i * 2 * kHead + col];
    red[g][c] = sum;
    __syncthreads();
    if (g != 0) return;
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < G; ++i) sum += red[i][c];
    if (col < kHead) {
        if (dqw) dqw[col] = sum;
    } else if (dkw) {
        dkw[col - kHead] = sum;
    }
}

// Workers of one token: as many as it takes to fill the chip, in fours so that a
// wave reads consecutive heads.  A worker looks its token up and forms its angles
// before the first head, so more of them cost: 16 waves per CU take 52 us for 8192 tokens
// of 60 heads (4.8 TB/s) and 15.8 for 1700 tokens of 48 into a cache, 8 waves 57 and
// 15.0, 32 waves 52 and 16.7, 64 waves 56 and 22.
int token_parts(int64_t tokens, int heads, int64_t want) {
    const int64_t need = (want + tokens - 1) / tokens;
    const int64_t p = need <= 1 ? 1 : (need + 3) / 4 * 4;
    return (int)std::min<int64_t>(p, heads);
}

constexpr int64_t kFwdWorkers = 256 * 16 * 4;
// Most groups of the backward: four workgroups per CU (8192 tokens of 60 heads take 77 us,
// 4.9 TB/s; 512 groups 104, 768 94, 1536 79, 2048 80).
constexpr int kBwdGroups = 1024;

Args common(const NormRope& f, const uint16_t* x, int64_t ldx, uint16_t* y, int64_t ldy,
            int64_t tokens, int64_t seq, int kv_heads, int group, int parts) {
    Args a = {};
    a.x = x; a.ldx = ldx;
    a.y = y; a.ldy = ldy;
    a.qw = f.qw; a.kw = f.kw;
    a.inv_freq = f.inv_freq;
    a.pos = f.pos;
    a.tokens = tokens;
    a.seq = seq;
    a.eps = f.eps;
    a.norm = f.norm;
    a.rot = f.rot;
    a.group = group;
    a.per_kv = group + 2;
    a.heads = kv_heads * a.per_kv;
    a.parts = parts;
    a.step_kv = parts / a.per_kv;
    a.step_r = parts % a.per_kv;
    return a;
}

// The backward's grid: parts of a token's heads (in fours, so that a wave reads
// consecutive heads) and the tokens between a worker's visits.  A visit costs about two
// heads beside its heads (the angles), and all workers get the same number of visits:
// 5001 tokens of 45 heads from memory take 67 us, 75 where a fifth of the workers had
// a second token.
struct BwdPlan {
    int parts;
    int64_t stride, groups;
};
int64_t most_groups(int64_t tokens) { return std::min<int64_t>(kBwdGroups, tokens); }
BwdPlan bwd_plan(int64_t tokens, int heads) {
    const int64_t workers = most_groups(tokens) * kWorkers;
    BwdPlan best = {1, 1, 1};
    int64_t least = INT64_MAX;
    for (int p = std::min(4, heads); p <= heads && p <= workers; p += 4) {
        const int64_t at_once = workers / p, visits = (tokens + at_once - 1) / at_once;
        const int64_t cost = visits * ((heads + p - 1) / p + 2);
        if (cost < least) {
            least = cost;
            best.parts = p;
            best.stride = (tokens + visits - 1) / visits;
        }
    }
    best.groups = (best.stride * best.parts + kWorkers - 1) / kWorkers;
    return best;
}

}  // namespace

int64_t norm_rope_ws_floats(int64_t tokens) { return most_groups(tokens) * 2 * kHead; }

hipError_t launch_norm_rope(const NormRopeProblem& p, hipStream_t s) {
    const int parts = token_parts(p.tokens, p.kv_heads * (p.group + 2), kFwdWorkers);
    Args a = common(p.f, p.x, p.ldx, p.y, p.ldy, p.tokens, p.seq, p.kv_heads, p.group, parts);
    a.copy_v = p.x != p.y;
    a.cache = p.cache;
    a.batch = p.batch;
    const int64_t grid = (p.tokens * parts + kWorkers - 1) / kWorkers;
    void (*k)(Args) = p.cached ? (p.f.interleaved ? norm_rope_kernel<true, true>
                                                  : norm_rope_kernel<false, true>)
                               : (p.f.interleaved ? norm_rope_kernel<true, false>
                                                  : norm_rope_kernel<false, false>);
    k<<<dim3((unsigned)grid), kThreads, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_norm_rope_bwd(const NormRopeBwdProblem& p, hipStream_t s) {
    if (p.tokens == 0) {      // sums of nothing
        weight_sum_kernel<<<16, kSumThreads, 0, s>>>(nullptr, 0, p.dqw, p.dkw);
        return hipGetLastError();
    }
    const BwdPlan plan = bwd_plan(p.tokens, p.kv_heads * (p.group + 2));
    const int64_t grid = plan.groups;
    Args a = common(p.f, p.x, p.ldx, p.dx, p.lddx, p.tokens, p.seq, p.kv_heads, p.group,
                    plan.parts);
    a.stride = plan.stride;
    a.dy = p.dy;
    a.lddy = p.lddy;
    a.copy_v = p.dy != p.dx;
    a.part = p.dqw || p.dkw ? p.ws : nullptr;
    void (*k)(Args) = p.f.interleaved ? norm_rope_bwd_kernel<true> : norm_rope_bwd_kernel<false>;
    k<<<dim3((unsigned)grid), kThreads, 0, s>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !a.part) return e;
    weight_sum_kernel<<<16, kSumThreads, 0, s>>>(p.ws, (int)grid, p.dqw, p.dkw);
    return hipGetLastError();
}

}  // namespace atp
