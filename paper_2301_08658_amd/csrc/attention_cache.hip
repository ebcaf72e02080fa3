// Attention of new tokens over a paged cache: o = softmax(q K^T / sqrt(128)) V
// over the cached tokens and the new ones that each row sees (causal, or the bits
// of a drafted tree).  Head dimension 128, key/value heads shared by `group`
// query heads.
//
// A unit is 16 RT rows (tokens' query heads of one key/value head) against a
// sequence's keys; workgroup w takes an equal share of all units' keys
// (cache_plan.h).  A unit that lies inside one share is finished there; one
// that is cut leaves its pieces' maxima, sums and outputs in the workspace, and
// join_kernel adds them in order.
//
// Few rows (up to 32): the four waves take 32 keys of every 128 each, with their
// own reference (a running maximum), sum and output, and meet only at the end of a
// piece: no barrier stands in the key loop.  A wave's K and V tiles (8 KB each) go straight
// to LDS; K's next tile is asked for as soon as the score products have read this
// one and V's after the second products, so 8 to 16 KB per wave are under way at
// any time, 64 to 128 KB per CU.  The time is the cache's bytes: one token of each of
// 64 sequences, 20 heads, 2.67 GB of keys and values take 450 us, 5.9 TB/s (a copy on
// this chip moves 5.2).
//
// Many rows (128 per unit): the waves take 32 rows each and share double-buffered
// tiles of 64 keys, so every fragment read from LDS feeds two products.  Prompt chunks of
// 500 to 1024 tokens, 49 GFLOP, take 81 us with the joining (604 TFLOP/s), 4096 tokens
// behind 4000 860 TFLOP/s.  Two waves on a SIMD take 5900 cycles for a tile each, one wave
// alone 3500; 1024 of a wave's are products and about 900 vector instructions.  What
// bounds it is that these hardly overlap: left out one by one, weights, copies and second
// product shorten a tile by 15, 21 and 20%, while more waves, fewer LDS reads per product
// or keys that are all in L2 (trees 104 -> 97 us, chunks 82 -> 81) change little.
//
// Products (layouts as in attention.hip): a lane of S^T = K Q^T holds row lane %
// 16 and keys 4 (lane / 16) + e of 16-key tiles, its probabilities are the right
// operand of O^T += V^T P^T as they are, and V^T's fragments are transposing LDS
// reads in the same key order.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "cache_kernels.h"
#include "cache_plan.h"
#include "lds_dma.h"

namespace atp {
namespace {

constexpr int D = kHead;
constexpr int NWAVE = 4;
constexpr int NTHR = 64 * NWAVE;
constexpr int KT = 32;                 // keys of a wave's tile
using plan::kGroups;
using plan::kLeast;
constexpr int kXcds = 8;
constexpr float kLn2 = 0.69314718055994530942f;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef short i16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
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

// a / b for a >= 0, b > 0: 64-bit division takes its time
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
    if (((a | b) >> 32) == 0) return (uint32_t)a / (uint32_t)b;
    return a / b;
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
    int extra;                   // of a unit (plan::Seq)
    int64_t cap;                 // max_pages * page size
    float scale_log2;
};

__device__ __forceinline__ plan::Seq seq_of(const Args& a, int s) {
    const const_ints cu = (const_ints)(uintptr_t)a.batch.cu;
    return plan::make_seq(((const_ints)(uintptr_t)a.batch.ctx)[s], cu[s], cu[s + 1], a.tokens,
                          a.cap, a.rows, a.extra);
}
__device__ __forceinline__ int64_t seq_line(const Args& a, const plan::Seq& q) {
    return plan::line_of(q, q.blocks, a.rows, a.mask == nullptr) * a.cache.kv_heads;
}

// A workgroup's share of the line: keys [begin, end), the sequence of key `begin`
// and the key that sequence starts at.  None: begin == end.
struct Share {
    int64_t index, per, begin, end, start;
    int s;
    plan::Seq q;
};
// Shares are numbered so that consecutive ones run on one XCD (workgroups go
// round the eight dies): the row blocks of a head share its keys in that L2.
__device__ __forceinline__ bool take_share(int64_t total, Share& sh) {
    sh.per = uniform(plan::share(total, kGroups, kLeast));
    const int64_t used = uniform(quotient(total + sh.per - 1, sh.per));
    const int bid = blockIdx.x;
    if (bid >= used) {
        sh.index = bid;
        sh.begin = sh.end = 0;
        return false;
    }
    const int64_t base = used / kXcds, rem = used % kXcds;
    const int x = bid % kXcds;
    sh.index = x * base + (x < rem ? x : rem) + bid / kXcds;
    sh.begin = sh.index * sh.per;
    sh.end = min(sh.begin + sh.per, total);
    return true;
}

// Inclusive prefix sum over the wave (rows of 16 lanes, then across them).
__device__ __forceinline__ uint32_t wave_prefix(uint32_t v) {
    auto add = [&](auto ctrl, auto rows) {
        v += __builtin_amdgcn_update_dpp(0u, v, decltype(ctrl)::value, decltype(rows)::value, 0xf,
                                         false);
    };
    add(std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xf>{});   // row_shr:1
    add(std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xf>{});
    add(std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xf>{});
    add(std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xf>{});
    add(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});   // row_bcast:15
    add(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});   // row_bcast:31
    return v;
}

__device__ __forceinline__ plan::Seq load_seq(const Args& a, int s) {
    return plan::make_seq(a.batch.ctx[s], a.batch.cu[s], a.batch.cu[s + 1], a.tokens, a.cap, a.rows,
                          a.extra);
}

// Every workgroup lays out the batch for itself: reading a few lengths costs less
// than a launch that would do it once.  Up to 64 sequences: one per lane, each wave by
// itself, nothing but registers (8.7 -> 7.6 us for one sequence's token).  More: runs of
// consecutive sequences per thread, added up through LDS.
__device__ __forceinline__ Share find_share(const Args& a, int64_t* lds) {
    Share sh;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = a.batch.n_seqs;
    if (n <= 64) {
        plan::Seq q = {};
        if (lane < n) q = load_seq(a, lane);
        const int64_t mine = lane < n ? seq_line(a, q) : 0;
        if (__builtin_amdgcn_ballot_w64(mine >> 26 != 0) == 0) {
            const uint32_t upto = wave_prefix((uint32_t)mine);
            const uint32_t total = __builtin_amdgcn_readlane(upto, 63);
            if (!take_share(total, sh)) return sh;
            // no lane behind the last sequence counts: its prefix is the total
            sh.s = __popcll(__builtin_amdgcn_ballot_w64(upto <= (uint32_t)sh.begin));
            sh.start = (uint32_t)__builtin_amdgcn_readlane(upto - (uint32_t)mine, sh.s);
            sh.q.first = __builtin_amdgcn_readlane(q.first, sh.s);
            sh.q.fresh = __builtin_amdgcn_readlane(q.fresh, sh.s);
            sh.q.ctx = __builtin_amdgcn_readlane(q.ctx, sh.s);
            sh.q.keys = __builtin_amdgcn_readlane(q.keys, sh.s);
            sh.q.blocks = __builtin_amdgcn_readlane(q.blocks, sh.s);
            sh.q.extra = a.extra;
            return sh;
        }
    }
    const int run = (n + NTHR - 1) / NTHR;
    int64_t mine = 0;
    for (int i = tid * run; i < min((tid + 1) * run, n); ++i) mine += seq_line(a, load_seq(a, i));
    int64_t inc = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t up = __shfl_up(inc, d);
        if (lane >= d) inc += up;
    }
    if (lane == 63) lds[wave] = inc;
    __syncthreads();
    int64_t total = 0, before = inc - mine;
#pragma unroll
    for (int w = 0; w < NWAVE; ++w) {
        if (w < wave) before += lds[w];
        total += lds[w];
    }
    if (!take_share(uniform(total), sh)) return sh;
    if (mine > 0 && before <= sh.begin && sh.begin < before + mine) {
        int i = tid * run;
        for (;; ++i) {
            const int64_t m = seq_line(a, load_seq(a, i));
            if (sh.begin < before + m || i + 1 >= n) break;
            before += m;
        }
        lds[NWAVE] = i;
        lds[NWAVE + 1] = before;
    }
    __syncthreads();
    sh.s = (int)uniform(lds[NWAVE]);
    sh.start = uniform(lds[NWAVE + 1]);
    sh.q = seq_of(a, sh.s);
    return sh;
}

// One row block of one head of one sequence, and its keys [u0, u1) of the line.
struct Unit {
    plan::Seq q;
    int s, head, block;
    int64_t u0, u1;
};
__device__ __forceinline__ Unit unit_at(const Args& a, const plan::Seq& q, int s, int64_t start,
                                        int64_t at) {
    Unit u;
    const bool causal = a.mask == nullptr;
    u.s = s;
    u.q = q;
    const int64_t head = plan::line_of(q, q.blocks, a.rows, causal);
    u.head = __builtin_amdgcn_readfirstlane((int)quotient(at - start, head));
    const int64_t h0 = start + u.head * head;
    u.block = __builtin_amdgcn_readfirstlane(plan::block_of(q, at - h0, a.rows, causal));
    u.u0 = uniform(h0 + plan::line_of(q, u.block, a.rows, causal));
    u.u1 = uniform(h0 + plan::line_of(q, u.block + 1, a.rows, causal));
    return u;
}

// Moves a share on to the sequence of key `at`.  Sequences without new tokens have
// none; they are stepped over one by one, a dependent trip to memory each.
__device__ __forceinline__ void next_seq(const Args& a, Share& sh, int64_t at) {
    const int64_t line = uniform(seq_line(a, sh.q));
    if (at < sh.start + line) return;
    sh.start += line;
    if (at >= sh.end) return;
    // lengths that change under a running kernel must not lead it astray
    while (sh.s + 1 < a.batch.n_seqs) {
        sh.q = seq_of(a, ++sh.s);
        if (sh.q.blocks > 0) return;
    }
    sh.end = at;
}

// The workspace: a record of every share, then two slots per share.  The record
// tells join_kernel of the unit that begins in the share and goes on behind it (last:
// the share of its last keys, -1 for no such unit).  A slot holds a piece's
// results, BM rows of 128 sums, BM maxima (base 2), BM sums of weights: slot 0 for a
// unit that began before the share, 1 for the one that goes on behind it.
struct Record {
    int last, token, tokens, head;    // token: its first row of the step's buffers
};
constexpr int kRecordFloats = kGroups * (int)sizeof(Record) / 4;
template <int BM>
__device__ __forceinline__ float* slot_of(float* ws, int64_t share, int slot) {
    return ws + kRecordFloats + (share * 2 + slot) * (int64_t)(BM * (D + 2));
}
__device__ __forceinline__ void leave_record(const Args& a, int64_t share, const Record& r) {
    if (threadIdx.x == 0) reinterpret_cast<Record*>(a.ws)[share] = r;
}
__device__ __forceinline__ Record record_of(const Args& a, const Unit& u, int64_t per, int lim,
                                            int tile) {
    const int tok = u.block * a.rows;
    return Record{(int)plan::last_share(u.u0, u.u1, per, a.extra, lim, tile), u.q.first + tok,
                  min(a.rows, u.q.fresh - tok), u.head};
}

// Where a unit's keys are: the table row, and a head's place in a page.
struct Keys {
    const_ints table;
    int64_t head0, half;       // elements: the head in a page, and from keys to values
    int lim, end, shift, max_pages, n_pages;   // keys that rows see; that the piece reads
    const uint16_t* pages;
    // the page of a key of the piece, -1 for none
    __device__ __forceinline__ int page_at(int key) const {
        const int col = key >> shift;
        const int e = key < end && col < max_pages ? table[col] : -1;
        return e >= 0 && e < n_pages ? e : -1;
    }
    // N keys of one page from `key` on, as buffer resources of keys and values: rows at
    // and behind lim, and all of a missing page, are past the range and read zeros
    template <int N>
    __device__ __forceinline__ void source(int page, int key, dma::u32x4& k, dma::u32x4& v) const {
        const int left =
            __builtin_amdgcn_readfirstlane(page < 0 ? 0 : min(max(lim - key, 0), N)) * D * 2;
        const int64_t at = (int64_t)max(page, 0) * 2 * half + head0 +
                           (int64_t)(key & ((1 << shift) - 1)) * D;
        const uint64_t a = reinterpret_cast<uint64_t>(pages + at), b = a + (uint64_t)half * 2;
        k = dma::u32x4{(uint32_t)a, (uint32_t)(a >> 32) & 0xffffu, (uint32_t)left,
                       dma::kRsrcWord3};
        v = dma::u32x4{(uint32_t)b, (uint32_t)(b >> 32) & 0xffffu, (uint32_t)left,
                       dma::kRsrcWord3};
    }
};
__device__ __forceinline__ Keys keys_of(const Args& a, const Unit& u, int lim, int end) {
    Keys k;
    k.shift = a.cache.page_shift;
    k.table = (const_ints)(uintptr_t)(a.batch.table + (int64_t)u.s * a.batch.ld_table);
    k.head0 = ((int64_t)u.head << k.shift) * D;
    k.half = ((int64_t)a.cache.kv_heads << k.shift) * D;
    k.lim = lim;
    k.end = end;
    k.max_pages = a.batch.max_pages;
    k.n_pages = a.cache.n_pages;
    k.pages = a.cache.pages;
    return k;
}

// Rows [row0, row1) of a unit: keys below `all` are seen by every one of them, keys from
// `none` on by none (no row there: 0).
struct Sight {
    int all, none;
};
__device__ __forceinline__ Sight sight_of(const Args& a, const Unit& u, int row0, int row1,
                                          int lim) {
    const int tok = u.block * a.rows;
    const int first = row0 / a.group;
    const int last = min(min((row1 - 1) / a.group, a.rows - 1), u.q.fresh - tok - 1);
    if (first > last) return Sight{0, 0};
    if (a.mask != nullptr) return Sight{u.q.ctx, lim};
    return Sight{u.q.ctx + tok + first + 1, min(u.q.ctx + tok + last + 1, lim)};
}

// Bit i: new token `tok` of the unit's sequence (-1: no row) sees key base + i.
__device__ __forceinline__ uint64_t sees_keys(const Args& a, const Unit& u, int tok, int base) {
    if (tok < 0) return 0;
    const int d0 = base - u.q.ctx;              // new token at the first place
    if (a.mask == nullptr) {
        const int n = tok + 1 - d0;
        return n >= 64 ? ~0ull : (n <= 0 ? 0ull : (1ull << n) - 1);
    }
    if (d0 <= -64) return ~0ull;
    const uint64_t* bits = a.mask + (int64_t)(u.q.first + tok) * a.words;
    if (d0 < 0) return bits[0] << -d0 | ((1ull << -d0) - 1);   // cached tokens, then new ones
    const int i = d0 >> 6, sh = d0 & 63;
    uint64_t v = i < a.words ? bits[i] >> sh : 0;
    if (sh > 0 && i + 1 < a.words) v |= bits[i + 1] << (64 - sh);
    return v;
}

// Scores of keys that a row does not see become -inf; a lane's are keys 16 j + 4 g + e.
template <int N>
__device__ __forceinline__ void hide(uint64_t sees, int g, f32x4 (&sc)[N]) {
    const uint64_t mine = sees >> (4 * g);       // once; then bits at fixed places
    const uint32_t half[2] = {(uint32_t)mine, (uint32_t)(mine >> 32)};
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (!(half[j >> 1] & (1u << (16 * (j & 1) + e)))) sc[j][e] = -INFINITY;
}

// Infinities and NaN among bf16 values (their exponent is all ones, and one more carries
// into the sign's place): seen = 0 to begin with, has_odd at the end.
__device__ __forceinline__ void look_for_odd(const u32x4& v, uint32_t& seen) {
#pragma unroll
    for (int e = 0; e < 4; ++e) seen |= (v[e] & 0x7f807f80u) + 0x00800080u;
}
__device__ __forceinline__ bool has_odd(uint32_t seen) {    // in any lane
    return __builtin_amdgcn_ballot_w64((seen & 0x80008000u) != 0) != 0;
}

// V^T's fragment of a 32-key slice: two transposing reads 16 rows apart.
__device__ __forceinline__ bf16x8 v_fragment(const uint16_t* p) {
    const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)p);
    const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(p + 16 * D));
    const i16x8 vv = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    return __builtin_bit_cast(bf16x8, vv);
}
// Infinities and NaN of a 32-key slice of V where not every row sees them: 0 times them
// would reach the other rows' sums in a matrix product, so what the rows do see is
// added here, key by key, o(row lane % 16, value 16 dt + 4 g + e) += p(row, key) v(key,
// value), and the slice is cleared of them (clear_odd) before the product.  pf: the
// lane's weights, sees: bits of its row.
__device__ __forceinline__ float odd_value(uint32_t b) {   // of the low half; else 0
    return (b & 0x7f80u) == 0x7f80u ? __uint_as_float(b << 16) : 0.f;
}
__device__ __forceinline__ void add_odd(const uint16_t* vt, const bf16x8& pf, uint32_t sees,
                                        f32x4 (&o)[8]) {
    const int lane = threadIdx.x & 63, g = lane >> 4, l16 = lane & 15;
    const u32x4 pw = __builtin_bit_cast(u32x4, pf);
#pragma unroll 1
    for (int key = 0; key < 32; ++key) {
        const int i = 4 * (key >> 4) + (key & 3);          // of the holding lane's eight
        uint32_t word = i < 4 ? (i < 2 ? pw[0] : pw[1]) : (i < 6 ? pw[2] : pw[3]);
        word = __shfl(word, 16 * ((key & 15) >> 2) + l16);
        const float p = __uint_as_float(i & 1 ? word & 0xffff0000u : word << 16);
        if (!(sees >> key & 1)) continue;
        int g_ = g;
        asm volatile("" : "+v"(g_));      // addresses are formed here, not kept in registers
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) {
            const u32x2 b = *reinterpret_cast<const u32x2*>(
                vt + key * D + vpos(key, 2 * dt + (g_ >> 1)) * 8 + 4 * (g_ & 1));
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t v = e & 1 ? b[e >> 1] >> 16 : b[e >> 1];
                if (odd_value(v) != 0.f) o[dt][e] += p * odd_value(v);   // NaN != 0 too
            }
        }
    }
}
__device__ __forceinline__ void clear_odd(bf16x8& chunk) {
    u32x4 v = __builtin_bit_cast(u32x4, chunk);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if ((v[e] & 0x7f80u) == 0x7f80u) v[e] &= 0xffff0000u;
        if ((v[e] & 0x7f800000u) == 0x7f800000u) v[e] &= 0xffffu;
    }
    chunk = __builtin_bit_cast(bf16x8, v);
}

// Softmax of a row's new scores (N 16-key tiles): weights exp2(scale x - m) in sc,
// running reference m, sum l (the lane's own keys; joined at the end) and output
// moved.  The reference lies kRise above a maximum of earlier scores and stays while it does:
// the weights are formed first, and only where a lane's sum leaves 1 (a score kRise above
// all before it; or a row without a reference yet) does the wave look for maxima, move O and
// l and form them again.  O / l and m + log2 l do not depend on the reference.  A maximum in
// every step took a fifth of the kernel's vector instructions.  No weight is above 1, so the
// sums hold whatever values the sums of a softmax with its true maximum would.
constexpr float kRise = 10.f;
template <int N>
__device__ __forceinline__ void softmax_step(f32x4 (&sc)[N], float scale, float& m, float& l,
                                             f32x4 (&o)[8]) {
    f32x4 p[N];
    float rs;
    auto weights = [&] {
        const float msub = m == -INFINITY ? 0.f : m;
        rs = 0.f;
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                p[j][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[j][e], scale, -msub));
                rs += p[j][e];
            }
    };
    weights();
    if (__builtin_amdgcn_ballot_w64(!(rs <= 1.f) || m == -INFINITY) != 0) {
        float mx = -INFINITY;
#pragma unroll
        for (int j = 0; j < N; ++j)
            mx = fmaxf(mx, fmaxf(fmaxf(sc[j][0], sc[j][1]), fmaxf(sc[j][2], sc[j][3])));
        const float mnew = fmaxf(m, __builtin_fmaf(row_max4(mx), scale, kRise));
        const float alpha = weight_of(m, mnew);
        l *= alpha;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) o[dt] *= alpha;
        m = mnew;
        weights();
    }
    l += rs;
#pragma unroll
    for (int j = 0; j < N; ++j) sc[j] = p[j];
}

// Weights of a 32-key slice as the products' operand, rounded to bf16 (by at most 2^-8 of
// a weight, as in attention.hip; their sum is not rounded): the matrix cores take 16
// bits, and with many rows a second product for the rest would cost a quarter.
__device__ __forceinline__ bf16x8 round_weights(const f32x4& a, const f32x4& b) {
    return __builtin_bit_cast(bf16x8, u32x4{pack_bf16x2(a[0], a[1]), pack_bf16x2(a[2], a[3]),
                                            pack_bf16x2(b[0], b[1]), pack_bf16x2(b[2], b[3])});
}
// What that rounding left, rounded in turn: with both products a weight keeps 16
// bits.
__device__ __forceinline__ bf16x8 weights_left(const f32x4& a, const f32x4& b, const bf16x8& r) {
    const u32x4 w = __builtin_bit_cast(u32x4, r);
    f32x4 x, y;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t p = w[e >> 1], q = w[2 + (e >> 1)];
        x[e] = a[e] - __uint_as_float(e & 1 ? p & 0xffff0000u : p << 16);
        y[e] = b[e] - __uint_as_float(e & 1 ? q & 0xffff0000u : q << 16);
    }
    return round_weights(x, y);
}

__device__ __forceinline__ float inverse_sum(float l) {   // 0 for a row that saw nothing
    return l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);       // NaN stays
}
__device__ __forceinline__ float log_sum(float m, float l) {
    constexpr float kUp = 1 << (int)kRise;      // l is about 1 / kUp: both terms small again
    return l == 0.f ? -INFINITY : kLn2 * (m - kRise) + logf(l * kUp);
}

// SMALL: pages of 16 tokens, so that a wave's tile of 32 keys spans two.
template <int RT, bool SMALL>
__global__ __launch_bounds__(NTHR, 2) void attention_cache_kernel(Args a) {
    constexpr int BM = 16 * RT, TILE = plan::kFewTile;
    static_assert(TILE == NWAVE * KT, "a tile of every wave");
    constexpr int kRed = D + 4;      // padded row of the merge
    __shared__ __attribute__((aligned(16))) uint16_t tiles[NWAVE][2][KT * D];
    __shared__ float wm[NWAVE][BM], wl[NWAVE][BM];
    __shared__ int wnan[NWAVE];
    __shared__ int64_t lds[NWAVE + 2];
    const int lane = threadIdx.x & 63, g = lane >> 4, l16 = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool causal = a.mask == nullptr;

    Share sh = find_share(a, lds);
    Record record = {-1, 0, 0, 0};

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
    bool careful = false;            // every tile is taken as if it had a masked place
    for (int64_t at = sh.begin; at < sh.end;) {
        const Unit u = unit_at(a, sh.q, sh.s, sh.start, at);
        if (u.u1 <= at || u.u0 > at) break;     // lengths that changed: see next_seq
        const int lim = plan::block_keys(u.q, u.block, a.rows, causal);
        const int all = careful ? 0 : sight_of(a, u, 0, BM, lim).all;
        const int64_t upto = min(sh.end, u.u1);
        const plan::Piece piece =
            plan::piece_keys(at - u.u0, upto - u.u0, a.extra, upto == u.u1, lim, TILE);
        if (piece.first >= piece.last) {        // a cut that leaves nothing here
            at = upto;
            next_seq(a, sh, at);
            continue;
        }
        const Keys src = keys_of(a, u, lim, piece.last);

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

        // the wave's tiles: 32 keys of every 128
        constexpr int STEP = TILE;
        constexpr int P = SMALL ? 2 : 1, PK = KT / P;     // pages of a tile, keys of each
        struct Tile {
            int page[P];
            dma::u32x4 k[P], v[P];
        };
        auto look_up = [&](int base, int (&page)[P]) {
#pragma unroll
            for (int h = 0; h < P; ++h) page[h] = src.page_at(base + PK * h);
        };
        auto aim = [&](int base, const int (&page)[P]) {
            Tile tl;
#pragma unroll
            for (int h = 0; h < P; ++h) {
                tl.page[h] = page[h];
                src.source<PK>(page[h], base + PK * h, tl.k[h], tl.v[h]);
            }
            return tl;
        };
        auto copy_keys = [&](const Tile& tl) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                dma::lds_dma16(tl.k[i * P / 8], kt + 4 * i * D,
                               koffs[i & 3] + (SMALL ? 0u : (uint32_t)((i >> 2) * 16 * D * 2)), 0u);
        };
        auto copy_values = [&](const Tile& tl) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                dma::lds_dma16(tl.v[i * P / 8], vt + 4 * i * D,
                               voffs[i & 1] +
                                   (uint32_t)(((SMALL ? i & 3 : i) >> 1) * 8 * D * 2), 0u);
        };
        int base = piece.first + KT * wave;
        bool more = base < piece.last;
        Tile cur;
        int ahead[P];                              // pages of the tile after the next copy
        look_up(base, ahead);
        if (more) {
            cur = aim(base, ahead);
            copy_keys(cur);
            copy_values(cur);
        }
        look_up(base + STEP, ahead);
        while (more) {
            const bool next = base + STEP < piece.last;
            Tile nxt = cur;
            if (next) nxt = aim(base + STEP, ahead);
            look_up(base + 2 * STEP, ahead);
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
            if (next) copy_keys(nxt);

            // what the rows see of these 32 keys, where that is not everything
            const bool masked =
                base + KT > all || base + KT > lim || cur.page[0] < 0 || cur.page[P - 1] < 0;
            uint32_t sees[RT];
            if (masked) {
                uint32_t there = (cur.page[0] < 0 ? 0u : 0xffffu) |
                                 (cur.page[P - 1] < 0 ? 0u : 0xffff0000u);
                if (lim - base < KT) there &= (1u << (lim - base)) - 1;
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    sees[r] = (uint32_t)sees_keys(a, u, tok[r], base) & there;
                    hide<2>(sees[r], g, sc[r]);
                }
            }
            // the bytes bound this kernel and the products have time to spare: the weights'
            // second halves too (2.3e-3 -> 1.7e-3 from the 64-bit result, the output's own
            // rounding)
            bf16x8 pf[RT], pl[RT];
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                softmax_step(sc[r], a.scale_log2, mrun[r], lrun[r], o[r]);
                pf[r] = round_weights(sc[r][0], sc[r][1]);
                pl[r] = weights_left(sc[r][0], sc[r][1], pf[r]);
            }
            if (next) dma::wait_vmcnt<8>();             // V has landed, the next K may not have
            else dma::wait_vmcnt<0>();
            // a masked place may hold anything
            bool odd = false;
            if (masked) {
                uint32_t seen = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    look_for_odd(*reinterpret_cast<const u32x4*>(vt + (i * 64 + lane) * 8), seen);
                odd = has_odd(seen);
            }
            if (odd) {
#pragma unroll
                for (int r = 0; r < RT; ++r) add_odd(vt, pf[r], sees[r], o[r]);
                for (int i = 0; i < 8; ++i)
                    clear_odd(*reinterpret_cast<bf16x8*>(vt + (i * 64 + lane) * 8));
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            }
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) {
                const bf16x8 vf = v_fragment(vt + vread[dt]);
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    o[r][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[r], o[r][dt], 0, 0, 0);
                    o[r][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pl[r], o[r][dt], 0, 0, 0);
                }
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // V's tile has been read
            if (next) copy_values(nxt);
            cur = nxt;
            more = next;
            base += STEP;
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
        // Where every row sees a whole tile, nothing looks for infinities and NaN among its
        // values: one that stands there leaves NaN in a wave's sums (a weight's second part,
        // above, is zero or negative for most of them), and then the piece is taken once more
        // with the values of every tile looked through.  32 or 64 additions per piece; looking
        // at every tile at once would cost 64 vector instructions and 8 KB of LDS reads each.
        f32x4 of4 = o[0][0];
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int dt = r == 0; dt < 8; ++dt) of4 += o[r][dt];
        const float of_all = (of4[0] + of4[1]) + (of4[2] + of4[3]);
        const bool nan = __builtin_amdgcn_ballot_w64(of_all != of_all) != 0;
        if (lane == 0) wnan[wave] = nan;
        const bool begins = piece.first == 0, whole = begins && piece.last == lim;
        if (begins && !whole) record = record_of(a, u, sh.per, lim, TILE);
        float* slot = slot_of<BM>(a.ws, sh.index, begins ? 1 : 0);
        float* red = reinterpret_cast<float*>(&tiles[wave][0][0]);     // 16 rows of kRed
        const int orow = threadIdx.x >> 4, ocol = (threadIdx.x & 15) * 8;
        __syncthreads();
        if (!careful &&
            __builtin_amdgcn_readfirstlane(wnan[0] | wnan[1] | wnan[2] | wnan[3]) != 0) {
            careful = true;
            __syncthreads();                 // wm, wl and wnan have been read
            continue;
        }
        careful = false;
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
                    const float inv = inverse_sum(l);
                    const u32x4 w = {pack_bf16x2(v[0] * inv, v[1] * inv),
                                     pack_bf16x2(v[2] * inv, v[3] * inv),
                                     pack_bf16x2(v[4] * inv, v[5] * inv),
                                     pack_bf16x2(v[6] * inv, v[7] * inv)};
                    *reinterpret_cast<u32x4*>(a.out + token * a.ldo + (int64_t)hq * D + ocol) = w;
                    if (a.lse && ocol == 0)
                        a.lse[(int64_t)hq * a.tokens + token] = log_sum(m, l);
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
        at = upto;
        next_seq(a, sh, at);
    }
    leave_record(a, sh.index, record);
}

// Many rows: BM = 128, four waves of two 16-row blocks, keys in tiles of 64 that the
// waves copy together, two buffers, one barrier per tile.  The copies of the next
// tile are issued between the score products, a quarter (16 keys: one page) at a
// time.  Other shapes tried on prompt chunks (92 us then): eight waves of 256 rows on a
// ring of four buffers, half of them half a tile behind (135); keys copied two tiles
// ahead behind a second barrier (94); values lagging a tile behind so that their product
// and the next weights share the time (97: 26 registers spilled).  Beside the present 82:
// 32-key tiles (86), also with three waves per SIMD (90), with 192 rows (96), with 256 rows
// and one wave per SIMD (128); the row blocks apart, one's products beside the other's
// weights (92).
constexpr int kWideRows = 128;
constexpr int WT = plan::kWideTile;    // keys of a tile
// SMALL: pages of fewer than 64 tokens; a tile's quarters are looked up one by one.
template <bool SMALL>
__global__ __launch_bounds__(NTHR, 2) void attention_cache_wide_kernel(Args a) {
    constexpr int RB = 2, TILE = WT;
    __shared__ __attribute__((aligned(16))) uint16_t tiles[2][2][WT * D];
    __shared__ int64_t lds[NWAVE + 2];
    const int lane = threadIdx.x & 63, g = lane >> 4, l16 = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool causal = a.mask == nullptr;

    Share sh = find_share(a, lds);
    Record record = {-1, 0, 0, 0};

    // copy round r fills tile rows 16 r + 4 wave + lane / 16, place lane % 16
    const int crow = 4 * wave + g;
    const uint32_t koff = (uint32_t)(crow * D * 2 + kpos(crow, l16) * 16);
    const uint32_t voff = (uint32_t)(crow * D * 2 + vpos(crow, l16) * 16);
    int kread[4], vread[8];
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) kread[ks] = l16 * D + kpos(l16, 4 * ks + g) * 8;
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) {
        const int r = 4 * g + (l16 >> 2), col = 16 * dt + 4 * (l16 & 3);
        vread[dt] = r * D + vpos(r, col >> 3) * 8 + (col & 7);
    }
    for (int64_t at = sh.begin; at < sh.end;) {
        const Unit u = unit_at(a, sh.q, sh.s, sh.start, at);
        if (u.u1 <= at || u.u0 > at) break;     // lengths that changed: see next_seq
        const int lim = plan::block_keys(u.q, u.block, a.rows, causal);
        const Sight sight = sight_of(a, u, 32 * wave, 32 * wave + 32, lim);
        const int64_t upto = min(sh.end, u.u1);
        const plan::Piece piece =
            plan::piece_keys(at - u.u0, upto - u.u0, a.extra, upto == u.u1, lim, TILE);
        if (piece.first >= piece.last) {        // a cut that leaves nothing here
            at = upto;
            next_seq(a, sh, at);
            continue;
        }
        const int first = piece.first, last = piece.last;
        const Keys src = keys_of(a, u, lim, last);
        constexpr int P = SMALL ? 4 : 1, PK = WT / P;     // pages of a tile, keys of each
        auto look_up = [&](int base, int (&page)[P]) {
#pragma unroll
            for (int h = 0; h < P; ++h) page[h] = src.page_at(base + PK * h);
        };
        // quarter r (16 keys) of the tile at `base` into a buffer
        dma::u32x4 rk, rv;
        auto copy = [&](int base, const int (&page)[P], int buf, int r) {
            if (SMALL || r == 0) src.source<PK>(page[r * P / 4], base + PK * (r * P / 4), rk, rv);
            uint16_t* dst = tiles[buf][0] + (16 * r + 4 * wave) * D;
            const uint32_t down = SMALL ? 0u : (uint32_t)(r * 16 * D * 2);
            dma::lds_dma16(rk, dst, koff + down, 0u);
            dma::lds_dma16(rv, dst + WT * D, voff + down, 0u);
        };

        // the first tile is on its way while the rows are read
        int page[P], ahead[P];            // of the tile at hand, of the one to be copied
        look_up(first, page);
        if (first < last) {
#pragma unroll
            for (int r = 0; r < 4; ++r) copy(first, page, 0, r);
        }
        look_up(first + WT, ahead);
        int tok[RB], hq[RB];
        bf16x8 qf[RB][4];
        f32x4 o[RB][8];
        float mrun[RB], lrun[RB];
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            const int row = 32 * wave + 16 * r + l16;
            const int j = row / a.group;
            hq[r] = u.head * a.group + row - j * a.group;
            tok[r] = u.block * a.rows + j;
            const bool on = j < a.rows && tok[r] < u.q.fresh;
            if (!on) tok[r] = -1;
            const uint16_t* q = a.q + (int64_t)(u.q.first + tok[r]) * a.ldq + (int64_t)hq[r] * D;
#pragma unroll
            for (int ks = 0; ks < 4; ++ks)
                qf[r][ks] = on ? *reinterpret_cast<const bf16x8*>(q + 32 * ks + 8 * g)
                               : __builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0});
            mrun[r] = -INFINITY;
            lrun[r] = 0.f;
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) o[r][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
        }

        dma::wait_vmcnt<0>();
        __syncthreads();
        auto advance = [&](int base) {
#pragma unroll
            for (int h = 0; h < P; ++h) page[h] = ahead[h];
            look_up(base + 2 * WT, ahead);
            dma::wait_vmcnt<0>();
            __syncthreads();
        };
        int buf = 0;
        for (int base = first; base < last; base += WT, buf ^= 1) {
            const uint16_t* kt = tiles[buf][0];
            const uint16_t* vt = tiles[buf][1];
            if (base >= sight.none) {     // nothing here for this wave's rows: it only copies
#pragma unroll
                for (int r = 0; r < 4; ++r) copy(base + WT, ahead, buf ^ 1, r);
                advance(base);
                continue;
            }
            f32x4 sc[RB][4];
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int r = 0; r < RB; ++r) sc[r][j] = f32x4{0.f, 0.f, 0.f, 0.f};
            // Fragments are asked for one slice of the head dimension ahead of their
            // products; as built, slices 0 and 1 are read so, and 2 and 3 two fragments at a
            // time, because no read passes a copy issued before it.  The next tile's copies
            // go into the other buffer, which was last read before the last barrier; behind
            // the piece's end they find no page and fill zeros, which costs less than
            // branches around them.
            bf16x8 kf[2][4];
            auto read = [&](int ks) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    kf[ks & 1][j] = *reinterpret_cast<const bf16x8*>(kt + 16 * j * D + kread[ks]);
            };
            read(0);
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) {
                if (ks < 3) read(ks + 1);
                copy(base + WT, ahead, buf ^ 1, ks);
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int r = 0; r < RB; ++r)
                        sc[r][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[ks & 1][j], qf[r][ks],
                                                                           sc[r][j], 0, 0, 0);
            }
            bool masked = base + WT > sight.all || base + WT > lim;
#pragma unroll
            for (int h = 0; h < P; ++h) masked |= page[h] < 0;
            uint64_t sees[RB];
            bool odd = false;
            if (masked) {
                uint64_t on = 0;
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (page[r * P / 4] >= 0) on |= 0xffffull << (16 * r);
                if (lim - base < WT) on &= (1ull << (lim - base)) - 1;
#pragma unroll
                for (int r = 0; r < RB; ++r) {
                    sees[r] = sees_keys(a, u, tok[r], base) & on;
                    hide<4>(sees[r], g, sc[r]);
                }
                // a masked place may hold anything
                uint32_t seen = 0;
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    look_for_odd(*reinterpret_cast<const u32x4*>(vt + (i * 64 + lane) * 8), seen);
                odd = has_odd(seen);
            }
            // V^T's fragments in four groups of four, read a group ahead of their products (a
            // product pair takes 32 cycles, a read four times that; read a pair ahead, trees
            // took 129.5 us and prompt chunks 94.4 instead of 126 and 92).
            bf16x8 vf[2][4], pf[2][RB];
            auto read_values = [&](int i) {
#pragma unroll
                for (int d = 0; d < 4; ++d)
                    vf[i & 1][d] =
                        v_fragment(vt + 32 * (i >> 1) * D + vread[4 * (i & 1) + d]);
            };
#pragma unroll
            for (int r = 0; r < RB; ++r) {
                softmax_step(sc[r], a.scale_log2, mrun[r], lrun[r], o[r]);
#pragma unroll
                for (int sl = 0; sl < 2; ++sl)
                    pf[sl][r] = round_weights(sc[r][2 * sl], sc[r][2 * sl + 1]);
            }
            if (odd) {
#pragma unroll
                for (int sl = 0; sl < 2; ++sl)
#pragma unroll
                    for (int r = 0; r < RB; ++r)
                        add_odd(vt + 32 * sl * D, pf[sl][r], (uint32_t)(sees[r] >> (32 * sl)),
                                o[r]);
            }
            read_values(0);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (i < 3) read_values(i + 1);
                if (odd) {
#pragma unroll
                    for (int d = 0; d < 4; ++d) clear_odd(vf[i & 1][d]);
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int d = 0; d < 4; ++d)
#pragma unroll
                    for (int r = 0; r < RB; ++r) {
                        f32x4& acc = o[r][4 * (i & 1) + d];
                        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[i & 1][d], pf[i >> 1][r],
                                                                      acc, 0, 0, 0);
                    }
                __builtin_amdgcn_sched_barrier(0);
            }
            advance(base);
        }

        const bool begins = piece.first == 0, whole = begins && piece.last == lim;
        if (begins && !whole) record = record_of(a, u, sh.per, lim, TILE);
        float* slot = slot_of<kWideRows>(a.ws, sh.index, begins ? 1 : 0);
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            const float l = row_sum4(lrun[r]);
            if (tok[r] < 0) continue;
            const int64_t token = u.q.first + tok[r];
            if (whole) {
                const float inv = inverse_sum(l);
                uint16_t* p = a.out + token * a.ldo + (int64_t)hq[r] * D + 4 * g;
#pragma unroll
                for (int dt = 0; dt < 8; ++dt)
                    *reinterpret_cast<u32x2*>(p + 16 * dt) =
                        u32x2{pack_bf16x2(o[r][dt][0] * inv, o[r][dt][1] * inv),
                              pack_bf16x2(o[r][dt][2] * inv, o[r][dt][3] * inv)};
                if (a.lse && g == 0) a.lse[(int64_t)hq[r] * a.tokens + token] = log_sum(mrun[r], l);
            } else {
                const int row = 32 * wave + 16 * r + l16;
#pragma unroll
                for (int dt = 0; dt < 8; ++dt)
                    *reinterpret_cast<f32x4*>(slot + row * D + 16 * dt + 4 * g) = o[r][dt];
                if (g == 0) {
                    slot[kWideRows * D + row] = mrun[r];
                    slot[kWideRows * D + kWideRows + row] = l;
                }
            }
        }
        at = upto;
        next_seq(a, sh, at);
    }
    leave_record(a, sh.index, record);
}

// The unit that begins in share blockIdx.x and goes on behind it: its pieces are
// slot 1 of that share and slot 0 of the following ones, added in order with a
// running maximum.  A half wave holds a row, four values per lane.  Few pieces, or a row
// for every half wave: it takes a row's pieces by itself (66 tokens of two sequences, 25
// pieces per unit of 126 rows: 39 us with the attention, 87 where the workgroup took the
// rows one by one).  Many pieces of few rows (a long context): the workgroup takes its R
// rows one by one, its half waves every H-th piece each.  128-row units never do: one unit
// over 131000 keys (8 drafts of 16 heads) is cut into some 500 pieces, each half wave adds its
// row's alone, and the joining takes 109 us, the attention 27.
constexpr int kManyPieces = 16;
struct Joined {
    float m, l;
    f32x4 v;
    __device__ __forceinline__ void clear() {
        m = -INFINITY;
        l = 0.f;
        v = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    __device__ __forceinline__ void add(float m2, float l2, const f32x4& v2) {
        const float top = fmaxf(m, m2), f = weight_of(m, top), f2 = weight_of(m2, top);
        m = top;
        l = l * f + l2 * f2;
        v = v * f + v2 * f2;
    }
};
template <int BM, int R, int NT>
__global__ __launch_bounds__(NT) void join_kernel(Args a) {
    constexpr int H = NT / 32;
    __shared__ float parts[H][D + 4];
    const int64_t share = blockIdx.x;
    const Record rec = reinterpret_cast<const Record*>(a.ws)[share];
    if (rec.last < 0) return;
    const int hw = threadIdx.x / 32, l32 = threadIdx.x & 31;
    const int n = min(rec.tokens * a.group, BM);      // rows of the unit
    const int pieces = rec.last - (int)share + 1;
    auto add_piece = [&](Joined& j, int i, int row) {
        const float* p = slot_of<BM>(a.ws, share + i, i == 0);
        j.add(p[BM * D + row], p[BM * D + BM + row],
              *reinterpret_cast<const f32x4*>(p + row * D + 4 * l32));
    };
    auto finish = [&](const Joined& r, int row) {
        const int j = row / a.group, hq = rec.head * a.group + row - j * a.group;
        const int64_t token = rec.token + j;
        const float inv = inverse_sum(r.l);
        *reinterpret_cast<u32x2*>(a.out + token * a.ldo + (int64_t)hq * D + 4 * l32) =
            u32x2{pack_bf16x2(r.v[0] * inv, r.v[1] * inv), pack_bf16x2(r.v[2] * inv, r.v[3] * inv)};
        if (a.lse && l32 == 0) a.lse[(int64_t)hq * a.tokens + token] = log_sum(r.m, r.l);
    };
    for (int row0 = blockIdx.y * R; row0 < n; row0 += gridDim.y * R) {
        const int row1 = min(row0 + R, n);
        Joined j;
        if (R >= H || pieces <= kManyPieces) {
            for (int row = row0 + hw; row < row1; row += H) {
                j.clear();
#pragma unroll 4
                for (int i = 0; i < pieces; ++i) add_piece(j, i, row);
                finish(j, row);
            }
            continue;
        }
        for (int row = row0; row < row1; ++row) {
            j.clear();
#pragma unroll 4
            for (int i = hw; i < pieces; i += H) add_piece(j, i, row);
            *reinterpret_cast<f32x4*>(&parts[hw][4 * l32]) = j.v;
            if (l32 == 0) {
                parts[hw][D] = j.m;
                parts[hw][D + 1] = j.l;
            }
            __syncthreads();
            if (hw == 0) {
                j.clear();
#pragma unroll
                for (int i = 0; i < H; ++i)
                    j.add(parts[i][D], parts[i][D + 1],
                          *reinterpret_cast<const f32x4*>(&parts[i][4 * l32]));
                finish(j, row);
            }
            __syncthreads();
        }
    }
}

// Rows of a unit: 16 or 32 while they hold a sequence's rows (the bytes count), else
// 128 (the products do).  A token's heads stay together.
int unit_rows(int group, int max_new) {
    const int64_t rows = (int64_t)group * max_new;
    return rows <= 16 ? 16 : (rows <= 32 ? 32 : kWideRows);
}

// rows: what a unit is expected to hold; the joining workgroups walk all it has
template <int BM, int R, int NT>
hipError_t launch(void (*kernel)(Args), const Args& a, unsigned grid, int64_t rows,
                  hipStream_t s) {
    kernel<<<grid, NTHR, 0, s>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const unsigned per = (unsigned)((std::min<int64_t>(rows, BM) + R - 1) / R);
    join_kernel<BM, R, NT><<<dim3(grid, per), NT, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

int64_t cache_attention_ws_floats(int group, int max_new) {
    return kRecordFloats + (int64_t)kGroups * 2 * unit_rows(group, max_new) * (D + 2);
}

hipError_t launch_cache_attention(const CacheAttentionProblem& p, hipStream_t s) {
    const int bm = unit_rows(p.group, p.max_new);
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
    a.rows = bm / p.group;
    a.extra = bm == kWideRows ? plan::kWideExtra : plan::kFewExtra;
    a.cap = (int64_t)p.batch.max_pages << p.cache.page_shift;
    a.scale_log2 = 1.4426950408889634f / sqrtf((float)D);
    // no batch of these sizes has more shares than this
    const int64_t units = std::min<int64_t>(p.batch.n_seqs, p.tokens) + p.tokens / a.rows;
    const int64_t most = std::min<int64_t>(units * p.cache.kv_heads, 1 << 20) *
                         ((a.cap + p.tokens + a.rows + a.extra) / kLeast + 2);
    const unsigned grid = (unsigned)std::min<int64_t>(kGroups, most);
    const int64_t rows = (int64_t)p.group * p.max_new;
    const int shift = p.cache.page_shift;
    if (bm == 16)
        return launch<16, 1, 512>(shift < 5 ? attention_cache_kernel<1, true>
                                            : attention_cache_kernel<1, false>, a, grid, rows, s);
    if (bm == 32)
        return launch<32, 1, 512>(shift < 5 ? attention_cache_kernel<2, true>
                                            : attention_cache_kernel<2, false>, a, grid, rows, s);
    return launch<kWideRows, 8, 256>(shift < 6 ? attention_cache_wide_kernel<true>
                                                : attention_cache_wide_kernel<false>, a, grid, rows,
                                      s);
}

}  // namespace atp
