// Attention of new tokens over a paged cache: o = softmax(q K^T / sqrt(128)) V
// over the cached tokens and the new ones that each row sees (causal, or the bits
// of a drafted tree).  Head dimension 128, key/value heads shared by `group`
// query heads.
//
// A unit is 16 RT rows (tokens' query heads of one key/value head) against a
// sequence's keys; workgroup w takes an equal share of all units' steps of 128
// keys (cache_plan.h).  A unit that lies inside one share is finished there; one
// that is cut leaves its pieces' maxima, sums and outputs in the workspace, and
// join_kernel adds them in order.
//
// Inside a workgroup the four waves take 32 keys of every step each, with their
// own running maximum, sum and output, and meet only at the end of a piece: no
// barrier stands in the key loop.  A wave's K and V tiles (8 KB each) go straight
// to LDS; K's next tile is asked for as soon as the score products have read this
// one and V's after the second products, so 8 to 16 KB per wave are under way at
// any time, 64 to 128 KB per CU.  With few rows the time is the cache's bytes.
//
// Products (layouts as in attention.hip): a lane of S^T = K Q^T holds row lane %
// 16 and keys 4 (lane / 16) + e of two 16-key tiles, its probabilities are the
// right operand of O^T += V^T P^T as they are, and V^T's fragments are transposing
// LDS reads in the same key order.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "cache_kernels.h"
#include "cache_plan.h"
#include "lds_dma.h"

namespace atp {
namespace {

constexpr int D = kHead;
constexpr int NWAVE = 4;
constexpr int NTHR = 64 * NWAVE;
constexpr int KT = 32;                 // keys of a wave's tile
constexpr int kGroups = 512;           // shares: two workgroups per CU on 256 CUs
constexpr int kLeastSteps = 1;
constexpr int kXcds = 8;
// largest base-2 gain of a row maximum absorbed without rescaling (weights stay
// below 2^8, exact in bf16's range)
constexpr float kSlack = 8.f;
constexpr float kLn2 = 0.69314718055994530942f;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef short i16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
// lists that the kernel never writes: uniform reads go through the scalar cache
typedef const __attribute__((address_space(4))) int32_t* const_ints;

// 16-byte chunk c of tile row n is kept at these places (distinct banks for the
// fragment reads and for the transposing reads)
__device__ __forceinline__ int kpos(int n, int c) { return c ^ (n & 15); }
__device__ __forceinline__ int vpos(int n, int c) { return c ^ (2 * (n & 3) + 8 * ((n >> 2) & 1)); }

// maximum and sum over the four lanes l, l ^ 16, l ^ 32, l ^ 48, the same bits in each
__device__ __forceinline__ float row_max4(float x) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                    false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                    false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float row_sum4(float x) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                    false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                    false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
__device__ __forceinline__ uint32_t pack_bf16x2(float a, float b) {   // round to nearest even
    const f32x2 v = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}
__device__ __forceinline__ float weight_of(float m, float top) {   // exp2(m - top), 0 for m = -inf
    return m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
}

// A value that is the same in every lane, kept in scalar registers.
__device__ __forceinline__ int64_t uniform(int64_t v) {
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v);
    const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)v >> 32));
    return (int64_t)((uint64_t)hi << 32 | lo);
}

struct Args {
    CacheView cache;
    BatchView batch;
    const uint16_t* q; int64_t ldq;
    const uint64_t* mask; int words;
    uint16_t* out; int64_t ldo;
    float* lse;
    float* ws;
    int tokens, group, rows;     // rows: tokens of a row block
    int64_t cap;                 // max_pages * page size
    float scale_log2;
};

__device__ __forceinline__ plan::Seq seq_of(const Args& a, int s) {
    const const_ints cu = (const_ints)(uintptr_t)a.batch.cu;
    return plan::make_seq(((const_ints)(uintptr_t)a.batch.ctx)[s], cu[s], cu[s + 1], a.tokens,
                          a.cap, a.rows);
}
__device__ __forceinline__ int64_t seq_steps(const Args& a, const plan::Seq& q) {
    return plan::steps_before(q, q.blocks, a.rows, a.mask == nullptr) * a.cache.kv_heads;
}

// Steps of the whole batch and, for thread t, of the sequences before its run of
// them (runs of `run` consecutive sequences).
struct Line {
    int64_t total, before, mine;
    int run;
};
__device__ __forceinline__ Line lay_out(const Args& a, int64_t* sums) {
    Line ln;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = a.batch.n_seqs;
    ln.run = (n + NTHR - 1) / NTHR;
    ln.mine = 0;
    for (int i = 0; i < ln.run; ++i) {
        const int s = tid * ln.run + i;
        if (s < n)
            ln.mine += seq_steps(a, plan::make_seq(a.batch.ctx[s], a.batch.cu[s], a.batch.cu[s + 1],
                                                   a.tokens, a.cap, a.rows));
    }
    int64_t inc = ln.mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t up = __shfl_up(inc, d);
        if (lane >= d) inc += up;
    }
    if (lane == 63) sums[wave] = inc;
    __syncthreads();
    ln.total = 0;
    ln.before = inc - ln.mine;
#pragma unroll
    for (int w = 0; w < NWAVE; ++w) {
        if (w < wave) ln.before += sums[w];
        ln.total += sums[w];
    }
    ln.total = uniform(ln.total);
    return ln;
}
// The sequence of step `at` (0 <= at < total) and the step it starts at, for the
// whole workgroup.
__device__ __forceinline__ void find_seq(const Args& a, const Line& ln, int64_t at, int64_t* found,
                                         int* s, int64_t* start) {
    if (ln.mine > 0 && ln.before <= at && at < ln.before + ln.mine) {
        int64_t p = ln.before;
        int i = threadIdx.x * ln.run;
        for (;; ++i) {
            const int64_t n = seq_steps(a, plan::make_seq(a.batch.ctx[i], a.batch.cu[i],
                                                          a.batch.cu[i + 1], a.tokens, a.cap,
                                                          a.rows));
            if (at < p + n || i + 1 >= a.batch.n_seqs) break;
            p += n;
        }
        found[0] = i;
        found[1] = p;
    }
    __syncthreads();
    *s = (int)uniform(found[0]);
    *start = uniform(found[1]);
    __syncthreads();
}

// One row block of one head of one sequence, and its steps [u0, u1) of the line.
struct Unit {
    plan::Seq q;
    int s, head, block;
    int64_t u0, u1;
};
__device__ __forceinline__ Unit unit_at(const Args& a, int s, int64_t start, int64_t at) {
    Unit u;
    const bool causal = a.mask == nullptr;
    u.s = s;
    u.q = seq_of(a, s);
    const int64_t head = plan::steps_before(u.q, u.q.blocks, a.rows, causal);
    u.head = __builtin_amdgcn_readfirstlane((int)((at - start) / head));
    const int64_t h0 = start + u.head * head;
    u.block = __builtin_amdgcn_readfirstlane(plan::block_of(u.q, at - h0, a.rows, causal));
    u.u0 = uniform(h0 + plan::steps_before(u.q, u.block, a.rows, causal));
    u.u1 = uniform(h0 + plan::steps_before(u.q, u.block + 1, a.rows, causal));
    return u;
}

// Shares are numbered so that consecutive ones run on one XCD (workgroups go
// round the eight dies): the row blocks of a head share its keys in that L2.
__device__ __forceinline__ int64_t share_index(int bid, int64_t used) {
    const int64_t base = used / kXcds, rem = used % kXcds;
    const int x = bid % kXcds;
    return x * base + (x < rem ? x : rem) + bid / kXcds;
}

// A piece's results in the workspace: BM rows of 128 sums, BM maxima (base 2),
// BM sums of weights; slot 0 of a share for a unit that began before it, 1 for one
// that goes on behind it.
template <int BM>
__device__ __forceinline__ float* slot_of(float* ws, int64_t share, int slot) {
    return ws + (share * 2 + slot) * (int64_t)(BM * (D + 2));
}

template <int RT>
__global__ __launch_bounds__(NTHR, 2) void attention_cache_kernel(Args a) {
    constexpr int BM = 16 * RT;
    constexpr int kRed = D + 4;      // padded row of the merge
    __shared__ __attribute__((aligned(16))) uint16_t tiles[NWAVE][2][KT * D];
    __shared__ float wm[NWAVE][BM], wl[NWAVE][BM];
    __shared__ int64_t sums[NWAVE], found[2];
    const int lane = threadIdx.x & 63, g = lane >> 4, l16 = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool causal = a.mask == nullptr;

    const Line ln = lay_out(a, sums);
    if (ln.total == 0) return;
    const int64_t per = uniform(plan::share(ln.total, kGroups, kLeastSteps));
    const int64_t used = uniform((ln.total + per - 1) / per);
    if (blockIdx.x >= used) return;
    const int64_t share = share_index(blockIdx.x, used);
    const int64_t begin = share * per, end = min(begin + per, ln.total);
    int s;
    int64_t start;
    find_seq(a, ln, begin, found, &s, &start);

    uint16_t* kt = tiles[wave][0];
    uint16_t* vt = tiles[wave][1];
    // copy instruction i fills tile rows 4 i + lane / 16, place lane % 16
    uint32_t koffs[4], voffs[2];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        koffs[i] = (uint32_t)((4 * i + g) * D * 2 + kpos(4 * i + g, l16) * 16);
#pragma unroll
    for (int i = 0; i < 2; ++i)
        voffs[i] = (uint32_t)((4 * i + g) * D * 2 + vpos(4 * i + g, l16) * 16);
    int kread[4], vread[8];
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) kread[ks] = l16 * D + kpos(l16, 4 * ks + g) * 8;
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) {
        const int r = 4 * g + (l16 >> 2), col = 16 * dt + 4 * (l16 & 3);
        vread[dt] = r * D + vpos(r, col >> 3) * 8 + (col & 7);
    }
    const int shift = a.cache.page_shift;
    const int64_t half = ((int64_t)a.cache.kv_heads << shift) * D;   // K to V of a page

    for (int64_t at = begin; at < end;) {
        if (seq_of(a, s).blocks == 0) {        // no new tokens: no steps either
            ++s;
            continue;
        }
        const Unit u = unit_at(a, s, start, at);
        const int t0 = (int)(at - u.u0), t1 = (int)(min(end, u.u1) - u.u0);
        const int lim = plan::block_keys(u.q, u.block, a.rows, causal);
        const const_ints table =
            (const_ints)(uintptr_t)(a.batch.table + (int64_t)u.s * a.batch.ld_table);
        const int64_t head0 = ((int64_t)u.head << shift) * D;
        auto page_at = [&](int key) {          // uniform
            const int col = key >> shift;
            const int e = col < a.batch.max_pages ? table[col] : -1;
            return e >= 0 && e < a.cache.n_pages ? e : -1;
        };

        // rows: token block * rows + r / group of the sequence, query head r % group
        int tok[RT];
        const uint16_t* qrow[RT];
        bf16x8 qf[RT][4];
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const int row = 16 * r + l16;
            const int j = row / a.group, hq = u.head * a.group + row - j * a.group;
            tok[r] = u.block * a.rows + j;
            const bool on = j < a.rows && tok[r] < u.q.fresh;
            if (!on) tok[r] = -1;
            qrow[r] = a.q + (int64_t)(u.q.first + tok[r]) * a.ldq + (int64_t)hq * D;
#pragma unroll
            for (int ks = 0; ks < 4; ++ks)
                qf[r][ks] = on ? *reinterpret_cast<const bf16x8*>(qrow[r] + 32 * ks + 8 * g)
                               : __builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0});
        }
        f32x4 o[RT][8];
        float mrun[RT], lrun[RT];
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            mrun[r] = -INFINITY;
            lrun[r] = 0.f;
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) o[r][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
        }

        // the wave's tiles: keys [base, base + 32) of every step
        auto base_of = [&](int t) { return t * plan::kStep + KT * wave; };
        struct Tile {
            int page[2];
        };
        auto pages_of = [&](int base) {
            Tile p;
            p.page[0] = base < lim ? page_at(base) : -1;
            p.page[1] = base + 16 < lim ? page_at(base + 16) : -1;
            return p;
        };
        // half h of a tile: 16 rows of one page; rows at and behind lim, and those of an
        // empty place, are past the range and read zeros
        auto copy = [&](const Tile& p, int base, int64_t kv, uint16_t* dst, bool keys) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int key = base + 16 * h;
                const int page = max(p.page[h], 0);
                const int left = __builtin_amdgcn_readfirstlane(
                    p.page[h] < 0 ? 0 : min(max(lim - key, 0), 16));
                const uint16_t* src = a.cache.pages + (int64_t)page * 2 * half + kv + head0 +
                                      (int64_t)(key & ((1 << shift) - 1)) * D;
                const dma::u32x4 rs = dma::rsrc_words(src, (int64_t)left * D * 2);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    dma::lds_dma16(rs, dst + (16 * h + 4 * i) * D,
                                   keys ? koffs[i] : voffs[i & 1] + (uint32_t)((i >> 1) * 8 * D * 2),
                                   0u);
            }
        };
        int t = t0;
        bool more = t < t1 && base_of(t) < lim;
        Tile cur = {{-1, -1}};
        if (more) {
            cur = pages_of(base_of(t));
            copy(cur, base_of(t), 0, kt, true);
            copy(cur, base_of(t), half, vt, false);
        }
        while (more) {
            const int base = base_of(t);
            const bool next = t + 1 < t1 && base_of(t + 1) < lim;
            Tile nxt = {{-1, -1}};
            if (next) nxt = pages_of(base_of(t + 1));
            dma::wait_vmcnt<8>();                       // K has landed, V may be under way
            f32x4 sc[RT][2];
#pragma unroll
            for (int r = 0; r < RT; ++r) sc[r][0] = sc[r][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < 4; ++ks)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const bf16x8 kf =
                        *reinterpret_cast<const bf16x8*>(kt + 16 * j * D + kread[ks]);
#pragma unroll
                    for (int r = 0; r < RT; ++r)
                        sc[r][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[r][ks], sc[r][j],
                                                                           0, 0, 0);
                }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // K's tile has been read
            if (next) copy(nxt, base_of(t + 1), 0, kt, true);

            // what the rows see of these 32 keys, where that is not everything
            const bool masked = base + KT > u.q.ctx || base + KT > lim || cur.page[0] < 0 ||
                                cur.page[1] < 0;
            uint32_t sees[RT];
            if (masked) {
                uint32_t there = (cur.page[0] < 0 ? 0u : 0xffffu) |
                                 (cur.page[1] < 0 ? 0u : 0xffff0000u);
                if (lim - base < KT) there &= (1u << (lim - base)) - 1;
                const int d0 = base - u.q.ctx;      // new token at the tile's first place
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    uint32_t w = 0;
                    if (tok[r] >= 0 && causal) {
                        const int n = tok[r] + 1 - d0;
                        w = n >= KT ? ~0u : (n <= 0 ? 0u : (1u << n) - 1);
                    } else if (tok[r] >= 0) {
                        const uint64_t* bits =
                            a.mask + (int64_t)(u.q.first + tok[r]) * a.words;
                        if (d0 < 0) {               // cached tokens, then new ones
                            w = d0 <= -KT ? ~0u
                                          : ((uint32_t)bits[0] << -d0) | ((1u << -d0) - 1);
                        } else {
                            const int i = d0 >> 6, sh = d0 & 63;
                            uint64_t v = i < a.words ? bits[i] >> sh : 0;
                            if (sh > 32 && i + 1 < a.words) v |= bits[i + 1] << (64 - sh);
                            w = (uint32_t)v;
                        }
                    }
                    sees[r] = w & there;
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (!(sees[r] >> (16 * j + 4 * g + e) & 1)) sc[r][j][e] = -INFINITY;
                }
            }
            bf16x8 pf[RT];
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                float mx = fmaxf(fmaxf(fmaxf(sc[r][0][0], sc[r][0][1]),
                                       fmaxf(sc[r][0][2], sc[r][0][3])),
                                 fmaxf(fmaxf(sc[r][1][0], sc[r][1][1]),
                                       fmaxf(sc[r][1][2], sc[r][1][3])));
                mx = row_max4(mx);
                const float mnew = fmaxf(mrun[r], mx * a.scale_log2);
                // the exponentials' reference moves when a row gains more than
                // kSlack on it; results differ by rounding only
                if (__builtin_amdgcn_ballot_w64(mnew > mrun[r] + kSlack) != 0) {
                    const float alpha = weight_of(mrun[r], mnew);
                    lrun[r] *= alpha;
#pragma unroll
                    for (int dt = 0; dt < 8; ++dt) o[r][dt] *= alpha;
                    mrun[r] = mnew;
                }
                const float msub = mrun[r] == -INFINITY ? 0.f : mrun[r];
                float p[2][4], rs = 0.f;
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        p[j][e] = __builtin_amdgcn_exp2f(
                            __builtin_fmaf(sc[r][j][e], a.scale_log2, -msub));
                        rs += p[j][e];
                    }
                lrun[r] += rs;             // the lane's own keys; joined at the end
                // the weights are rounded to bf16 for the matrix product (half a step
                // is 2^-9 of a weight, as in attention.hip); their sum is not
                const u32x4 pw = {pack_bf16x2(p[0][0], p[0][1]), pack_bf16x2(p[0][2], p[0][3]),
                                  pack_bf16x2(p[1][0], p[1][1]), pack_bf16x2(p[1][2], p[1][3])};
                pf[r] = __builtin_bit_cast(bf16x8, pw);
            }
            if (next) dma::wait_vmcnt<8>();             // V has landed, the next K may not have
            else dma::wait_vmcnt<0>();
            // a masked place may hold anything; 0 times an infinity or NaN would still
            // reach the sums, so such values take another way
            bool odd = false;
            if (masked) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const u32x4 v = *reinterpret_cast<const u32x4*>(vt + (i * 64 + lane) * 8);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        odd |= (v[e] & 0x7f80u) == 0x7f80u || (v[e] & 0x7f800000u) == 0x7f800000u;
                }
                odd = __builtin_amdgcn_ballot_w64(odd) != 0;
            }
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) {
                const uint16_t* p0 = vt + vread[dt];
                i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)p0);
                i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(p0 + 16 * D));
                if (odd) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if ((lo[e] & 0x7f80) == 0x7f80) lo[e] = 0;
                        if ((hi[e] & 0x7f80) == 0x7f80) hi[e] = 0;
                    }
                }
                const i16x8 vv = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
                const bf16x8 vf = __builtin_bit_cast(bf16x8, vv);
#pragma unroll
                for (int r = 0; r < RT; ++r)
                    o[r][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[r], o[r][dt], 0, 0, 0);
            }
            if (odd) {
                // the infinities and NaN that a row does see: o(row l16, value 16 dt +
                // 4 g + e) += p(row, key) v(key, value), key by key
                for (int key = 0; key < KT; ++key) {
                    const int from = 16 * ((key & 15) >> 2) + l16;    // the lane with p(row, key)
#pragma unroll
                    for (int r = 0; r < RT; ++r) {
                        const u32x4 pw = __builtin_bit_cast(u32x4, pf[r]);
                        const int i = 4 * (key >> 4) + (key & 3);      // of the lane's eight
                        uint32_t word = i < 4 ? (i < 2 ? pw[0] : pw[1]) : (i < 6 ? pw[2] : pw[3]);
                        word = __shfl(word, from);
                        const float p = __uint_as_float(i & 1 ? word & 0xffff0000u : word << 16);
                        if (!(sees[r] >> key & 1)) continue;
#pragma unroll
                        for (int dt = 0; dt < 8; ++dt)
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const int col = 16 * dt + 4 * g + e;
                                const uint32_t b =
                                    vt[key * D + vpos(key, col >> 3) * 8 + (col & 7)];
                                if ((b & 0x7f80u) == 0x7f80u)
                                    o[r][dt][e] += p * __uint_as_float(b << 16);
                            }
                    }
                }
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // V's tile has been read
            if (next) copy(nxt, base_of(t + 1), half, vt, false);
            cur = nxt;
            more = next;
            ++t;
        }

        // the four waves' results of this piece, row block by row block
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            lrun[r] = row_sum4(lrun[r]);
            if (g == 0) {
                wm[wave][16 * r + l16] = mrun[r];
                wl[wave][16 * r + l16] = lrun[r];
            }
        }
        const bool whole = t0 == 0 && u.u1 <= end;
        float* slot = slot_of<BM>(a.ws, share, t0 > 0 ? 0 : 1);
        float* red = reinterpret_cast<float*>(&tiles[wave][0][0]);     // 16 rows of kRed
        const int orow = threadIdx.x >> 4, ocol = (threadIdx.x & 15) * 8;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            float top = -INFINITY;
#pragma unroll
            for (int w = 0; w < NWAVE; ++w) top = fmaxf(top, wm[w][16 * r + l16]);
            const float f = weight_of(mrun[r], top);
#pragma unroll
            for (int dt = 0; dt < 8; ++dt)
                *reinterpret_cast<f32x4*>(red + l16 * kRed + 16 * dt + 4 * g) = o[r][dt] * f;
            __syncthreads();
            const int row = 16 * r + orow;
            float m = -INFINITY, l = 0.f, v[8];
#pragma unroll
            for (int w = 0; w < NWAVE; ++w) m = fmaxf(m, wm[w][row]);
#pragma unroll
            for (int w = 0; w < NWAVE; ++w) l += wl[w][row] * weight_of(wm[w][row], m);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = 0.f;
#pragma unroll
            for (int w = 0; w < NWAVE; ++w) {
                const float* p = reinterpret_cast<const float*>(&tiles[w][0][0]) + orow * kRed + ocol;
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] += p[e];
            }
            const int j = row / a.group, tk = u.block * a.rows + j;
            if (j < a.rows && tk < u.q.fresh) {
                const int hq = u.head * a.group + row - j * a.group;
                const int64_t token = u.q.first + tk;
                if (whole) {
                    const float inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);   // NaN stays
                    const u32x4 w = {pack_bf16x2(v[0] * inv, v[1] * inv),
                                     pack_bf16x2(v[2] * inv, v[3] * inv),
                                     pack_bf16x2(v[4] * inv, v[5] * inv),
                                     pack_bf16x2(v[6] * inv, v[7] * inv)};
                    *reinterpret_cast<u32x4*>(a.out + token * a.ldo + (int64_t)hq * D + ocol) = w;
                    if (a.lse && ocol == 0)
                        a.lse[(int64_t)hq * a.tokens + token] =
                            l == 0.f ? -INFINITY : kLn2 * m + logf(l);
                } else {
                    float* p = slot + row * D + ocol;
                    *reinterpret_cast<f32x4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
                    *reinterpret_cast<f32x4*>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
                    if (ocol == 0) {
                        slot[BM * D + row] = m;
                        slot[BM * D + BM + row] = l;
                    }
                }
            }
            __syncthreads();
        }
        at = u.u0 + t1;
        // the next unit of the line: another block or head, or a later sequence
        const int64_t all = uniform(seq_steps(a, u.q));
        if (at >= start + all) {
            start += all;
            ++s;
        }
    }
}

// The unit that is cut at the end of share blockIdx.x, if it began there: its
// pieces are slot 1 of that share and slot 0 of the following ones.  A wave joins
// one row.
template <int RT>
__global__ __launch_bounds__(NTHR) void join_kernel(Args a) {
    constexpr int BM = 16 * RT;
    __shared__ int64_t sums[NWAVE], found[2];
    const int lane = threadIdx.x & 63;
    const Line ln = lay_out(a, sums);
    if (ln.total == 0) return;
    const int64_t per = plan::share(ln.total, kGroups, kLeastSteps);
    const int64_t share = blockIdx.x;
    const int64_t begin = share * per, end = begin + per;
    if (end >= ln.total) return;                    // nothing follows
    int s;
    int64_t start;
    find_seq(a, ln, end - 1, found, &s, &start);
    const Unit u = unit_at(a, s, start, end - 1);
    if (u.u1 <= end || u.u0 < begin) return;
    const int64_t last = (u.u1 - 1) / per;          // share of its last step
    const int row = blockIdx.y * NWAVE + (threadIdx.x >> 6);
    const int j = row / a.group, tk = u.block * a.rows + j;
    if (j >= a.rows || tk >= u.q.fresh) return;

    float top = -INFINITY;
    for (int64_t w = share + lane; w <= last; w += 64)
        top = fmaxf(top, slot_of<BM>(a.ws, w, w == share)[BM * D + row]);
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    f32x2 sum = {0.f, 0.f};
    float l = 0.f;
#pragma unroll 4
    for (int64_t w = share; w <= last; ++w) {
        const float* p = slot_of<BM>(a.ws, w, w == share);
        const float f = weight_of(p[BM * D + row], top);
        l += f * p[BM * D + BM + row];
        const f32x2 v = *reinterpret_cast<const f32x2*>(p + row * D + 2 * lane);
        sum[0] += f * v[0];
        sum[1] += f * v[1];
    }
    const float inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);
    const int hq = u.head * a.group + row - j * a.group;
    const int64_t token = u.q.first + tk;
    *reinterpret_cast<uint32_t*>(a.out + token * a.ldo + (int64_t)hq * D + 2 * lane) =
        pack_bf16x2(sum[0] * inv, sum[1] * inv);
    if (a.lse && lane == 0)
        a.lse[(int64_t)hq * a.tokens + token] = l == 0.f ? -INFINITY : kLn2 * top + logf(l);
}

// 16-row tiles of a unit: as few as hold a sequence's rows, at most four.
int row_tiles(int group, int max_new) {
    const int64_t rows = (int64_t)group * max_new;
    const int need = rows <= 16 ? 1 : (rows <= 32 ? 2 : 4);
    const int least = group <= 16 ? 1 : (group <= 32 ? 2 : 4);   // a token's heads stay together
    return std::max(need, least);
}

template <int RT>
hipError_t launch(const Args& a, unsigned grid, hipStream_t s) {
    attention_cache_kernel<RT><<<grid, NTHR, 0, s>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || grid <= 1) return e;
    join_kernel<RT><<<dim3(grid, 16 * RT / NWAVE), NTHR, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

int64_t cache_attention_ws_floats(int group, int max_new) {
    return (int64_t)kGroups * 2 * 16 * row_tiles(group, max_new) * (D + 2);
}

hipError_t launch_cache_attention(const CacheAttentionProblem& p, hipStream_t s) {
    const int rt = row_tiles(p.group, p.max_new);
    Args a = {};
    a.cache = p.cache;
    a.batch = p.batch;
    a.q = p.q; a.ldq = p.ldq;
    a.mask = p.mask; a.words = p.mask_words;
    a.out = p.out; a.ldo = p.ldo;
    a.lse = p.lse;
    a.ws = p.ws;
    a.tokens = (int)p.tokens;
    a.group = p.group;
    a.rows = 16 * rt / p.group;
    a.cap = (int64_t)p.batch.max_pages << p.cache.page_shift;
    a.scale_log2 = 1.4426950408889634f / sqrtf((float)D);
    // no batch of these sizes has more steps than this
    const int64_t units = std::min<int64_t>(p.batch.n_seqs, p.tokens) + p.tokens / a.rows;
    const int64_t steps = 2 * ((a.cap + plan::kStep - 1) / plan::kStep) + 3;
    const int64_t most = std::min<int64_t>(units * p.cache.kv_heads, 1 << 20) * steps;
    const unsigned grid = (unsigned)std::min<int64_t>(kGroups, most);
    switch (rt) {
        case 1: return launch<1>(a, grid, s);
        case 2: return launch<2>(a, grid, s);
        default: return launch<4>(a, grid, s);
    }
}

}  // namespace atp
