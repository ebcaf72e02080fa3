// Causal attention within documents of packed rows, for training: forward and
// backward, with key/value heads shared by `group` query heads, a prefix of each
// document that all of its rows see, scores capped by a tanh and a bias by distance.
//
//   x_ij = cap tanh(q_i . k_j / (cap sqrt(d))) - slope |i - j|,
//   o_i = sum_j softmax_j(x_ij) v_j over j in [start, max(i + 1, start + prefix))
//
// with start the first row of i's document.  Tiles of rows and keys begin at a
// document's start and end at its end, so a tile never holds two documents: what
// another document or the padding holds is not read, and inside a tile all is as in
// the causal core (attention.hip describes tiles, fragments and the running softmax).
// A row sees an interval of its document from the first key on, so the tiles that
// need a mask are those that reach past the first row's limit.
//
// Documents are found without a list of tiles, so that their lengths may change from
// replay to replay of a graph.  Up to 64 documents: a workgroup finds the tile of its
// rank in the order of falling work from the lengths alone (ranked_tile).  More:
// document d's tiles of Q rows take the slots from cu[d] / Q + d on, which do not
// overlap (floor(a + b) >= floor(a) + floor(b), and a document of n rows has at most
// floor(n / Q) + 1 tiles) and end at cu[n] / Q + n; a search over cu finds a slot's.
// Slots without a tile end at once.
//
// Backward: P from the saved log-sum-exps, delta_i = dO_i . O_i,
//   dS = P o (dO V^T - delta) o (1 - tanh^2), dQ = dS K / sqrt(d), dK = dS^T Q / sqrt(d),
//   dV = P^T dO.  A workgroup of the dK/dV kernel walks the query tiles of all query
// heads of its key head; where that leaves too few workgroups the heads are divided
// over several, which leave fp32 sums that are added in order.
//
// The weights P are rounded to bf16 for the products with V and dO, and dS for those with K
// and Q: the matrix instructions that take 32 bits have a sixteenth of the rate.  A rounding is
// off by 2^-9 of the value at most, so that outputs and gradients are off by up to 2^-9 of the
// sums of their terms' magnitudes (on unit-normal inputs 0.24% of the results' norm, of
// which the results' own rounding to bf16 is 0.17); sums, maxima, lse and delta are fp32.
//
// Kernels of 20 heads of two documents of 4096 rows, one profile: forward 194 us, 886 TFLOP/s of
// the visible pairs' products (matrix cores busy 43% of the cycles, vector units 44%: the two
// together), dQ 264 us (48% and 39%), dK and dV 478 us, where no unit is full (35%, 32%, LDS
// 39%) and the waves wait for LDS, copies and barriers 39% of their time; 579 TFLOP/s for the
// backward's five products.  Calls in a row on one document of 16384 rows and 8 heads: 503 to
// 525 us forward and 1880 to 1950 backward, 1050 to 1090 and 700 to 730 TFLOP/s.
#include <hip/hip_runtime.h>
#include <float.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "attention_tiles.h"
#include "train_kernels.h"
#include "wave_ops.h"

namespace atp {
namespace {

using namespace tiles;

constexpr float kLog2e = 1.44269504088896340736f;
// forward: a lane's sum of weights (16 keys of a row) that moves the row's reference.  Far
// below fp32's largest number, so that values up to 2^90 do not overflow; 2^20 and 2^30
// measured the same.
constexpr float kMostSum = 4096.f;

struct Common {
    const uint16_t* qkv; int64_t ldq;
    const int32_t* cu;
    const int32_t* prefix;
    const float* slopes;
    int64_t tokens;
    int n_docs, kv_heads, group, slots;
    float scale_log2;                    // log2(e) / sqrt(D)
    float cap_in, cap_log2;              // 2 log2(e) / (sqrt(D) cap), cap log2(e)
    float cap_y;                         // 1 / (sqrt(D) cap)
    float root_d;                        // sqrt(D)
};

struct Doc {
    int64_t tok0;                        // first row
    int len, tile, prefix;               // rows, this slot's tile, rows that all see
};

// A document's rows as the lists give them, kept inside the rows whatever they say.
__device__ __forceinline__ void bounds(const Common& a, int c0, int c1, int prefix, Doc& doc) {
    const int tokens = (int)a.tokens;
    const int start = min(max(c0, 0), tokens), end = min(max(c1, start), tokens);
    doc.tok0 = start;
    doc.len = end - start;               // both inside [0, tokens]: no overflow
    doc.prefix = max(0, min(prefix, doc.len));
}

// The tile at `rank` when all documents' tiles of 2^SHIFT rows are ordered by their
// index, the highest first (LAST_KEYS: by their index from the document's end):
// the longest loops lead and the last workgroups are short.  Up to 64 documents, one
// per lane: a level's first rank is the number of tiles of higher levels.  False for
// ranks behind the last tile.
template <int SHIFT, bool LAST_KEYS>
__device__ __forceinline__ bool ranked_tile(const Common& a, int rank, Doc& doc) {
    const int lane = threadIdx.x & 63;
    const bool in = lane < a.n_docs;
    const int c0 = in ? a.cu[lane] : 0, c1 = in ? a.cu[lane + 1] : 0;
    const int prefix = in && a.prefix ? a.prefix[lane] : 0;
    bounds(a, c0, c1, prefix, doc);
    const int mine = in ? (doc.len + (1 << SHIFT) - 1) >> SHIFT : 0;
    // tiles of level t and above; below 2^24, exact in fp32
    auto above = [&](int t) {
        return __builtin_amdgcn_readfirstlane((int)wave::sum64((float)max(mine - t, 0)));
    };
    if (rank >= above(0)) return false;
    // above(lo) > rank >= above(hi)
    int lo = 0, hi = (int)((a.tokens + (1 << SHIFT) - 1) >> SHIFT);
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (above(mid) > rank) lo = mid;
        else hi = mid;
    }
    const uint64_t level = __builtin_amdgcn_ballot_w64(mine > lo);
    const int place = rank - above(lo + 1);
    const bool here = mine > lo && __popcll(level & ((1ull << lane) - 1)) == place;
    const int d = __builtin_ctzll(__builtin_amdgcn_ballot_w64(here));
    doc.tok0 = __builtin_amdgcn_readlane((int)doc.tok0, d);
    doc.len = __builtin_amdgcn_readlane(doc.len, d);
    doc.prefix = __builtin_amdgcn_readlane(doc.prefix, d);
    doc.tile = LAST_KEYS ? ((doc.len + (1 << SHIFT) - 1) >> SHIFT) - 1 - lo : lo;
    return true;
}

// The document and tile of a slot of 2^SHIFT rows, for more documents; false for a slot
// without one.
template <int SHIFT>
__device__ __forceinline__ bool slot_tile(const Common& a, int slot, Doc& doc) {
    const int lane = threadIdx.x & 63;
    int lo = 0, span = a.n_docs;         // the document is in [lo, lo + span)
    for (;;) {
        const int step = (span + 63) >> 6;
        const int i = lo + lane * step;
        const bool le = lane * step < span && (a.cu[i] >> SHIFT) + i <= slot;
        const int n = __popcll(__builtin_amdgcn_ballot_w64(le));
        if (n == 0) return false;
        const int skip = (n - 1) * step;
        lo += skip;
        span = min(step, span - skip);
        if (step == 1) break;
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    const int c0 = __builtin_amdgcn_readfirstlane(a.cu[lo]);
    bounds(a, c0, __builtin_amdgcn_readfirstlane(a.cu[lo + 1]),
           a.prefix ? __builtin_amdgcn_readfirstlane(a.prefix[lo]) : 0, doc);
    doc.tile = slot - (c0 >> SHIFT) - lo;
    return doc.tile >= 0 && ((int64_t)doc.tile << SHIFT) < doc.len;
}

// Tile number i of the launch, the longest loops first where that is known.
template <int SHIFT, bool LAST_KEYS>
__device__ __forceinline__ bool find_tile(const Common& a, int i, Doc& doc) {
    const bool ok = a.n_docs <= 64
                        ? ranked_tile<SHIFT, LAST_KEYS>(a, i, doc)
                        : slot_tile<SHIFT>(a, LAST_KEYS ? i : a.slots - 1 - i, doc);
    // the same in every lane: scalars, for the copies' addresses
    doc.tok0 = __builtin_amdgcn_readfirstlane((int)doc.tok0);
    doc.len = __builtin_amdgcn_readfirstlane(doc.len);
    doc.tile = __builtin_amdgcn_readfirstlane(doc.tile);
    doc.prefix = __builtin_amdgcn_readfirstlane(doc.prefix);
    return __builtin_amdgcn_readfirstlane(ok);
}

// How scores are capped: by 1 - 2 / (1 + e^(2 y)) alone, which is off by up to 6 u of the
// cap however small the score is, or, for caps whose 6 u are no longer small beside the
// weights' rounding to bf16, by that where |y| >= 1/4 and by the series of tanh below (off by
// 2^-18 of the score).  The series takes 30% more time (20 heads of two documents of 4096
// rows forward 211 and 271 us, backward 767 and 994), so caps of up to kSmallCap do
// without: 6 u 64 = 2.3e-5 against the weights' 2^-9.
enum Cap { kNoCap, kSmall, kLarge };
constexpr float kSmallCap = 64.f;

// What is done to raw products q . k.  A bias alone is what the products are added to
// (in their units), a cap alone keeps their order (a large one but for its roundings), so
// that both keep the raw maximum; cap and bias together are formed for every score before
// it.
template <Cap CAP, bool BIAS>
struct Score {
    static constexpr bool kFormed = CAP && BIAS;
    float scale, cap_in, cap_log2, cap_y, slope, slope_raw;
    __device__ __forceinline__ Score(const Common& a, int head)
        : scale(a.scale_log2), cap_in(a.cap_in), cap_log2(a.cap_log2), cap_y(a.cap_y), slope(0.f),
          slope_raw(0.f) {
        if constexpr (BIAS) {
            slope = a.slopes[head] * kLog2e;
            slope_raw = a.slopes[head] * a.root_d;
        }
    }
    // the products' first summand
    __device__ __forceinline__ float start(float dist) const {
        if constexpr (BIAS && !CAP) return -slope_raw * __builtin_fabsf(dist);
        return 0.f;
    }
    // tanh(y) = 1 - 2 r, r = 1 / (1 + e^(2 y))
    __device__ __forceinline__ float rest_of(float raw) const {
        return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(raw * cap_in));
    }
    __device__ __forceinline__ float capped_of(float raw, float r) const {
        const float whole = __builtin_fmaf(r, -2.f * cap_log2, cap_log2);
        if constexpr (CAP != kLarge) return whole;
        // tanh(y) / y to y^8: the rest is below 2^-26 up to 1/4
        const float y = raw * cap_y, y2 = y * y;
        float t = __builtin_fmaf(y2, 62.f / 2835.f, -17.f / 315.f);
        t = __builtin_fmaf(y2, t, 2.f / 15.f);
        t = __builtin_fmaf(y2, t, -1.f / 3.f);
        t = __builtin_fmaf(y2, t, 1.f);
        return __builtin_fabsf(y) < 0.25f ? raw * scale * t : whole;
    }
    __device__ __forceinline__ float capped(float raw) const {
        return capped_of(raw, rest_of(raw));
    }
    __device__ __forceinline__ float bias(float x, float dist) const {
        if constexpr (kFormed) return __builtin_fmaf(-slope, __builtin_fabsf(dist), x);
        return x;
    }
    // Base-2 score of a row's largest raw (or formed) value.  -inf stays but under a cap alone,
    // where it may be a seen product's, with a score of -cap; of a row that sees nothing
    // (whose weights are masked one by one) -cap is a reference below all scores to come.
    __device__ __forceinline__ float top(float mx) const {
        if constexpr (kFormed) return mx;
        if constexpr (CAP) return capped(mx);
        return mx * scale;
    }
    // 2^(score - m) of a raw (or formed) value
    __device__ __forceinline__ float weight(float v, float m) const {
        if constexpr (kFormed) return __builtin_amdgcn_exp2f(v - m);
        if constexpr (CAP == kLarge) return __builtin_amdgcn_exp2f(capped(v) - m);
        if constexpr (CAP == kSmall)
            return __builtin_amdgcn_exp2f(
                __builtin_fmaf(rest_of(v), -2.f * cap_log2, cap_log2 - m));
        return __builtin_amdgcn_exp2f(__builtin_fmaf(v, scale, -m));
    }
    // The same with the product rounded as m's was: 1 at the maximum however large the
    // scores are, where the product's own last bits, kept by a fused step, pass 2^7 from
    // scores of 2^31 on.  Below m + kSlack where m is the maximum or at most so much less;
    // large caps' roundings may pass it where the series ends.
    __device__ __forceinline__ float weight_at_top(float v, float m) const {
#pragma clang fp contract(off)
        if constexpr (CAP == kLarge && !BIAS) {
            const float x = capped(v) - m;
            return __builtin_amdgcn_exp2f(x > kSlack ? kSlack : x);    // NaN stays
        }
        if constexpr (CAP) return weight(v, m);
        const float x = v * scale;
        return __builtin_amdgcn_exp2f(x - m);
    }
};

// ---------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------
struct FwdArgs : Common {
    uint16_t* out; int64_t ldo;
    float* lse;                          // [heads][tokens]
};

// bf16 pairs with an exponent of all ones have bit 15 of their half set in this.
__device__ __forceinline__ uint32_t odd_bits(uint32_t w) {
    return (w & 0x7f807f80u) + 0x00800080u;
}

__device__ __forceinline__ uint32_t without_odd(uint32_t w) {
    return w & ~(((odd_bits(w) & 0x80008000u) >> 15) * 0xffffu);
}

// Values of a masked tile may be infinite or NaN where no row of the tile, or only
// some, see them, and 0 times such a value is NaN.  These values are left out of the
// products and added to the rows that see them (as their sum with anything is what
// the weighted sum gives too).
template <int RB>
__device__ __forceinline__ void odd_values(const uint16_t* vs, int n_first,
                                           const int (&limit)[RB], int g,
                           f32x4 (&o)[RB][8]) {
#pragma unroll 1
    for (int n = 0; n < BN; ++n) {
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) {
            const int c = 16 * dt + 4 * g;
            const u32x2 w =
                *reinterpret_cast<const u32x2*>(vs + n * D + vpos(n, c >> 3) * 8 + (c & 7));
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float v = __uint_as_float(e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
                const bool odd = (__float_as_uint(v) & 0x7f800000u) == 0x7f800000u;
#pragma unroll
                for (int r = 0; r < RB; ++r)
                    if (odd && n_first + n < limit[r]) o[r][dt][e] += v;
            }
        }
    }
}

template <int RB, int KG, Cap CAP, bool BIAS>
__global__ __launch_bounds__(NTHR * KG + (KG > 1 ? NTHR : 0), KG > 1 ? 3 : 2)
void docs_fwd_kernel(FwdArgs a) {
    constexpr int QT = 64 * RB;
    constexpr bool PRODUCERS = KG > 1;
    __shared__ __attribute__((aligned(16))) uint16_t kv[KG][2][2][BN * D];   // [group][buf][K|V]
    __shared__ float mls[KG > 1 ? NWAVE * RB * 2 * 64 : 1];                // group 1's m, l
    const int lane = threadIdx.x & 63;
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool producer = PRODUCERS && wv >= KG * NWAVE;
    const int grp = producer ? 0 : wv / NWAVE, wave = wv % NWAVE;
    const int heads = a.kv_heads * a.group;
    const int head = blockIdx.x % heads, kvh = head / a.group;
    Doc doc = {};
    if (!find_tile<RB == 2 ? 7 : 6, false>(a, (int)(blockIdx.x / heads), doc)) return;
    const int qt = doc.tile;
    const int64_t tok0 = doc.tok0;
    const int64_t hc = (int64_t)kvh * (a.group + 2) * D;
    const int64_t qc = hc + (int64_t)(head - kvh * a.group) * D;

    const int last = min(qt * QT + QT, doc.len) - 1;
    const int nkt = (max(last + 1, doc.prefix) + BN - 1) / BN;
    const int half = KG > 1 ? (nkt + 1) / 2 : nkt;
    const int kt0 = grp == 0 ? 0 : half;
    const int mine = grp == 0 ? half : nkt - half;   // <= half
    // With a bias the last tile, with the diagonal, comes first, so that near keys, which it
    // favours, do not move the weights' reference at every tile (20 heads of two documents
    // of 4096 rows: 270 us in ascending order, 226 so; of nine documents of up to 1500 rows,
    // half of each a prefix, 55 and 60).
    constexpr bool BACK = KG == 1 && BIAS;
    auto tile_of = [&](int i) { return BACK ? nkt - 1 - i : kt0 + i; };
    uint16_t(*buf)[2][BN * D] = kv[grp];
    TileDma2<true> cp;
    cp.init(a.ldq, a.ldq, wave, lane);
    const uint16_t* kbase = a.qkv + hc + (int64_t)a.group * D;
    const uint16_t* vbase = kbase + D;
    if constexpr (PRODUCERS) {
        if (producer) {
            produce<KG>(cp, kbase, vbase, a.ldq, tok0, nkt, doc.len, kv, wave);
            return;
        }
    } else {
        if (mine > 0)
            cp.issue(kbase, a.ldq, vbase, a.ldq, tok0, tile_of(0) * BN, doc.len, buf[0][0],
                     buf[0][1], wave);
        dma::wait_vmcnt<0>();
    }
    int mrow[RB], limit[RB];             // rows in the document, keys that they see
    bf16x8 qf[RB][4];
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        mrow[r] = qt * QT + 64 * r + wave * 16 + (lane & 15);
        limit[r] = max(mrow[r] + 1, doc.prefix);
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            if (mrow[r] < doc.len)
                qf[r][ks] = *reinterpret_cast<const bf16x8*>(
                    a.qkv + (tok0 + mrow[r]) * a.ldq + qc + 32 * ks + 8 * (lane >> 4));
            else
                qf[r][ks] = __builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0});
        }
    }
    const Score<CAP, BIAS> score(a, head);

    f32x4 o[RB][8];
    float mrun[RB], lrun[RB];
#pragma unroll
    for (int r = 0; r < RB; ++r) {
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) o[r][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
        mrun[r] = -INFINITY;
        lrun[r] = 0.f;
    }

    __syncthreads();
    const int g = lane >> 4, l16 = lane & 15;
    int koff[4], voff[8];
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) koff[ks] = l16 * D + kpos(l16, 4 * ks + g) * 8;
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) voff[dt] = tr_offset(lane, dt);
    // keys that all rows of the tile see; keys that any row of a block sees
    const int clear = max(qt * QT + 1, doc.prefix);
    int reach[RB];
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        const int top = qt * QT + 64 * r;
        reach[r] = top < doc.len ? max(min(top + 64, doc.len), doc.prefix) : 0;
    }
    // One key tile for the row blocks [R0, R1), those that see some of it.
    const std::integral_constant<int, 0> b0;
    const std::integral_constant<int, 1> b1;
    // Without masks there is a next tile, whose copies then stand between the products without
    // a branch, so that a slice's fragments are read while the slice before is multiplied.
    auto step = [&](int i, auto r0, auto r1, auto mask) {
        constexpr int R0 = decltype(r0)::value, R1 = decltype(r1)::value;
        constexpr bool MASKED = decltype(mask)::value;
        const int kt = tile_of(i);
        const uint16_t* ks_ = buf[i & 1][0];
        const uint16_t* vs_ = buf[i & 1][1];
        const bool more = !PRODUCERS && (!MASKED || i + 1 < mine);
        const auto next = cp.rounds(kbase, a.ldq, vbase, a.ldq, tok0,
                                    tile_of(i + 1) * BN, doc.len,
                                    buf[(i + 1) & 1][0], buf[(i + 1) & 1][1]);
        f32x4 s[RB][4];
#pragma unroll
        for (int r = R0; r < R1; ++r) {
            const float ahead = (float)(mrow[r] - kt * BN - 4 * g);
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    s[r][j][e] = score.start(ahead - (float)(16 * j + e));
        }
        bf16x8 kf[4], kn[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            kf[j] = *reinterpret_cast<const bf16x8*>(ks_ + 16 * j * D + koff[0]);
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            if (ks < 3) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    kn[j] = *reinterpret_cast<const bf16x8*>(ks_ + 16 * j * D + koff[ks + 1]);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int r = R0; r < R1; ++r)
                    s[r][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[j], qf[r][ks], s[r][j], 0,
                                                                      0, 0);
            if (more) cp.round(next, ks, wave);
#pragma unroll
            for (int j = 0; j < 4; ++j) kf[j] = kn[j];
        }
        if constexpr (Score<CAP, BIAS>::kFormed) {
#pragma unroll
            for (int r = R0; r < R1; ++r) {
                const float ahead = (float)(mrow[r] - kt * BN - 4 * g);
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        s[r][j][e] =
                            score.bias(score.capped(s[r][j][e]), ahead - (float)(16 * j + e));
            }
        }
        // keys past the document are past every limit of its rows
        bool odd = false;
        if constexpr (MASKED) {
#pragma unroll
            for (int r = R0; r < R1; ++r)
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (kt * BN + 16 * j + 4 * g + e >= limit[r]) s[r][j][e] = -INFINITY;
            uint32_t seen = 0;
#pragma unroll 2
            for (int c = 0; c < BN * D / 512; ++c) {
                const u32x4 w = *reinterpret_cast<const u32x4*>(vs_ + (c * 64 + lane) * 8);
                seen |= odd_bits(w[0]) | odd_bits(w[1]) | odd_bits(w[2]) | odd_bits(w[3]);
            }
            odd = __builtin_amdgcn_ballot_w64((seen & 0x80008000u) != 0) != 0;
        }
        // The weights 2^(x - m) take the reference m of earlier tiles; it moves, to the row's
        // maximum, when a lane's sum of weights passes kMostSum.  O / l and m + log2 l do not
        // depend on m, so the results differ from a maximum at every step by rounding only,
        // and the maxima, a third of the vector instructions, are spared.
        bf16x8 pf[RB][2];
#pragma unroll
        for (int r = R0; r < R1; ++r) {
            auto weights = [&](auto form, float m, bool moved) {
                float sum = 0.f;
#pragma unroll
                for (int j = 0; j < 4; j += 2) {
                    f32x4 p[2];
#pragma unroll
                    for (int k = 0; k < 2; ++k)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float x = s[r][j + k][e];
                            if constexpr (decltype(form)::value == 0)
                                p[k][e] = score.weight(x, m);
                            else if constexpr (KG > 1)
                                p[k][e] = score.weight_at_top(x, m);
                            else
                                p[k][e] = moved ? score.weight_at_top(x, m) : score.weight(x, m);
                            // a cap makes a finite score of a masked one's -inf
                            if constexpr (MASKED && CAP && !BIAS)
                                if (kt * BN + 16 * (j + k) + 4 * g + e >= limit[r]) p[k][e] = 0.f;
                            sum += p[k][e];
                        }
                    pf[r][j / 2] = pack_pair(p[0], p[1]);
                }
                return sum;
            };
            // Where the reference moves it does so row by row, so that no row's bits depend on
            // its neighbours.
            auto move_to_top = [&](bool move) {
                const float mnew =
                    move ? fmaxf(mrun[r], score.top(row_max4(max16(s[r])))) : mrun[r];
                // a row that has seen no key keeps -inf: subtract 0
                const float alpha =
                    __builtin_amdgcn_exp2f(mrun[r] - (mnew == -INFINITY ? 0.f : mnew));
                lrun[r] *= alpha;
#pragma unroll
                for (int dt = 0; dt < 8; ++dt) o[r][dt] *= alpha;
                mrun[r] = mnew;
            };
            float rs = 0.f;
            if constexpr (KG > 1) {
                // a group's few tiles: by the maximum of each, when it is 2^8 above
                const float top = score.top(row_max4(max16(s[r])));
                const bool move = top > mrun[r] + kSlack;
                if (__builtin_amdgcn_ballot_w64(move) != 0) move_to_top(move);
                rs = weights(b1, mrun[r] == -INFINITY ? 0.f : mrun[r], true);
            } else {
                // The first tile sets the reference.  Where a row sees nothing in it (from the
                // back) or, without a cap, scores of -inf alone, m stays -inf, and the next
                // sums are infinite or NaN.
                const bool first = !BACK && i == 0;
                if (!first) rs = weights(b0, mrun[r], false);
                const bool over = !(rs <= kMostSum);
                if (first || __builtin_amdgcn_ballot_w64(over) != 0) {
                    const bool move = first || row_max4(over ? 1.f : 0.f) > 0.f;
                    move_to_top(move);
                    rs = weights(b1, mrun[r] == -INFINITY ? 0.f : mrun[r], move);
                }
            }
            lrun[r] += rs;               // the lane's share: a row's four lanes join at the end
        }

        // O += P V over two 32-key slices
        auto add_values = [&](auto clean) {
#pragma unroll
            for (int sl = 0; sl < 2; ++sl) {
#pragma unroll
                for (int dt = 0; dt < 8; ++dt) {
                    bf16x8 vf = frag_tr_at(vs_ + 32 * sl * D + voff[dt]);
                    if constexpr (decltype(clean)::value) {
                        u32x4 w = __builtin_bit_cast(u32x4, vf);
#pragma unroll
                        for (int k = 0; k < 4; ++k) w[k] = without_odd(w[k]);
                        vf = __builtin_bit_cast(bf16x8, w);
                    }
#pragma unroll
                    for (int r = R0; r < R1; ++r)
                        o[r][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[r][sl], o[r][dt],
                                                                           0, 0, 0);
                }
            }
        };
        if constexpr (KG > 1) {          // the groups' tiles differ: fragments are cleaned
            if (odd) {
                odd_values<RB>(vs_, kt * BN, limit, g, o);
                add_values(std::true_type{});
                return;
            }
        } else if (odd) {                // by all waves: the tile is cleaned
            odd_values<RB>(vs_, kt * BN, limit, g, o);
            __syncthreads();
            u32x4* own = reinterpret_cast<u32x4*>(buf[i & 1][1]) + wave * 64 + lane;
#pragma unroll 1
            for (int c = 0; c < BN * D / 8; c += NTHR) {
                u32x4 w = own[c];
                for (int k = 0; k < 4; ++k) w[k] = without_odd(w[k]);
                own[c] = w;
            }
            __syncthreads();
        }
        add_values(std::false_type{});
    };
    const std::integral_constant<int, RB> bn;
    const std::true_type yes;
    const std::false_type no;
    auto end_step = [&] {
        // this wave's copies of its next step have landed; after the barrier
        // every wave's have, and no wave reads the buffers of this step
        dma::wait_vmcnt<0>();
        __syncthreads();
    };
    // tiles that every row sees whole
    const int whole = max(0, min(clear / BN - kt0, mine));
    int i = 0;
    if constexpr (BACK) {
        if (reach[RB - 1] > 0) {
            if constexpr (RB > 1)        // behind all keys of the first block
                for (; tile_of(i) * BN >= reach[0]; ++i) {
                    step(i, b1, bn, yes);
                    end_step();
                }
            for (; i < nkt - whole; ++i) {
                step(i, b0, bn, yes);
                end_step();
            }
            for (; i < nkt - 1; ++i) {
                step(i, b0, bn, no);
                end_step();
            }
            if (i < nkt) {
                step(i, b0, bn, yes);
                end_step();
            }
        } else {                         // the second block lies past the document
            for (; i < nkt; ++i) {
                step(i, b0, b1, yes);
                end_step();
            }
        }
    } else if (RB == 1 || reach[RB - 1] > 0) {
        for (; i < (PRODUCERS ? whole : min(whole, mine - 1)); ++i) {
            step(i, b0, bn, no);
            end_step();
        }
        for (; i < mine && (RB == 1 || (kt0 + i) * BN < reach[0]); ++i) {
            step(i, b0, bn, yes);
            end_step();
        }
        if constexpr (RB > 1)
            for (; i < mine; ++i) {
                step(i, b1, bn, yes);
                end_step();
            }
    } else {
        for (; i < mine; ++i) {
            step(i, b0, b1, yes);
            end_step();
        }
    }
    for (; i < half; ++i) end_step();    // a group with fewer tiles idles
#pragma unroll
    for (int r = 0; r < RB; ++r) lrun[r] = row_sum4(lrun[r]);

    if constexpr (KG > 1) {
        f32x4* ox = reinterpret_cast<f32x4*>(&kv[1][0][0][0]);
        if (grp == 1) {
#pragma unroll
            for (int r = 0; r < RB; ++r) {
#pragma unroll
                for (int dt = 0; dt < 8; ++dt)
                    ox[((wave * RB + r) * 8 + dt) * 64 + lane] = o[r][dt];
                mls[((wave * RB + r) * 2 + 0) * 64 + lane] = mrun[r];
                mls[((wave * RB + r) * 2 + 1) * 64 + lane] = lrun[r];
            }
        }
        __syncthreads();
        if (grp == 1) return;
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            const float m1 = mls[((wave * RB + r) * 2 + 0) * 64 + lane];
            const float l1 = mls[((wave * RB + r) * 2 + 1) * 64 + lane];
            const float mn = fmaxf(mrun[r], m1);          // key 0 is group 0's
            const float a0 = __builtin_amdgcn_exp2f(mrun[r] - mn);
            const float a1 = __builtin_amdgcn_exp2f(m1 - mn);   // 0 when m1 = -inf
#pragma unroll
            for (int dt = 0; dt < 8; ++dt)
                o[r][dt] = o[r][dt] * a0 + ox[((wave * RB + r) * 8 + dt) * 64 + lane] * a1;
            lrun[r] = lrun[r] * a0 + l1 * a1;
            mrun[r] = mn;
        }
    }

#pragma unroll
    for (int r = 0; r < RB; ++r) {
        if (mrow[r] >= doc.len) continue;
        const float inv = 1.0f / lrun[r];
        uint16_t* orow = a.out + (tok0 + mrow[r]) * a.ldo + (int64_t)head * D;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) {
            const u32x2 w = {pack_bf16x2(o[r][dt][0] * inv, o[r][dt][1] * inv),
                             pack_bf16x2(o[r][dt][2] * inv, o[r][dt][3] * inv)};
            *reinterpret_cast<u32x2*>(orow + 16 * dt + 4 * g) = w;
        }
        if (g == 0)
            a.lse[(int64_t)head * a.tokens + tok0 + mrow[r]] =
                (mrun[r] + __log2f(lrun[r])) * 0.69314718055994530942f;
    }
}

// ---------------------------------------------------------------------------
// backward
// ---------------------------------------------------------------------------
struct BwdArgs : Common {
    const uint16_t* out; int64_t ldo;
    const uint16_t* dout; int64_t lddo;
    const float* lse;                    // [heads][tokens]
    float* delta;                        // [heads][tokens]
    uint16_t* dqkv; int64_t lddq;
    float* sums;                         // parts > 1: [parts][tokens][kv_heads][2][D]
    int parts, part_heads;               // divisions of a group's query heads, heads in one
    float inv_sqrt_d;
};

// P and dS of one element from the raw score, dO . v, and the row's lse and delta.
template <Cap CAP, bool BIAS>
__device__ __forceinline__ void grad_of(const Score<CAP, BIAS>& f, float raw, float dist, float l2,
                                        float dl, bool hidden, float& p, float& ds) {
    float pv, d;
    if constexpr (CAP) {
        const float r = f.rest_of(raw), r4 = 4.f * r;
        if constexpr (CAP == kLarge)
            pv = __builtin_amdgcn_exp2f(f.bias(f.capped_of(raw, r) - l2, dist));
        else
            pv = __builtin_amdgcn_exp2f(
                f.bias(__builtin_fmaf(r, -2.f * f.cap_log2, f.cap_log2 - l2), dist));
        d = pv * (ds - dl) * __builtin_fmaf(-r4, r, r4);     // 1 - tanh^2 = 4 r (1 - r)
    } else {
        pv = __builtin_amdgcn_exp2f(__builtin_fmaf(raw, f.scale, -l2));
        d = pv * (ds - dl);
    }
    p = hidden ? 0.f : pv;
    ds = hidden ? 0.f : d;
}

// dK and dV of a 64-key tile, 16 keys per wave, 32 queries at a time (so that scores and
// dP take 16 registers each).  KG groups of four waves split the steps (group 0 the
// first half, group 1 the rest, added through LDS at the end).  20 heads of two documents
// of 4096 rows took 100 us more with 32 keys per wave, which halve the fragments' reads
// but leave one wave per SIMD; 25 us more with the products at a raised wave priority; and
// 230 us more with the first transposed fragments read ahead of the weights (spills).
template <int KG, Cap CAP, bool BIAS>
__global__ __launch_bounds__(NTHR * KG, 2 / KG) void docs_dkv_kernel(BwdArgs a) {
    __shared__ __attribute__((aligned(16))) uint16_t qd[KG][2][2][BM * D];   // [grp][buf][Q|dO]
    __shared__ __attribute__((aligned(16))) float rowv[KG][2][2][BM];   // [grp][buf][lse2|delta]
    const int lane = threadIdx.x & 63, g = lane >> 4;
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int grp = wv / NWAVE, wave = wv % NWAVE;
    const int tid = (int)threadIdx.x % NTHR;   // thread index within the group
    const int per_slot = a.kv_heads * a.parts;
    const int which = blockIdx.x % per_slot;
    const int kvh = which % a.kv_heads, part = which / a.kv_heads;
    Doc doc = {};
    if (!find_tile<6, true>(a, (int)(blockIdx.x / per_slot), doc)) return;
    const int kt = doc.tile;
    const int64_t tok0 = doc.tok0, T = a.tokens;
    const int64_t hc = (int64_t)kvh * (a.group + 2) * D;
    const int h0 = kvh * a.group + part * a.part_heads;          // first query head
    const int nh = min(a.part_heads, a.group - part * a.part_heads);

    const int kabs = kt * BN + wave * 16 + (lane & 15);
    bf16x8 kf[4], vf[4];
    f32x4 dk[8], dv[8];
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
        if (kabs < doc.len) {
            const uint16_t* row = a.qkv + (tok0 + kabs) * a.ldq + hc + (int64_t)a.group * D;
            kf[ks] = *reinterpret_cast<const bf16x8*>(row + 32 * ks + 8 * g);
            vf[ks] = *reinterpret_cast<const bf16x8*>(row + D + 32 * ks + 8 * g);
        } else {
            kf[ks] = __builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0});
            vf[ks] = kf[ks];
        }
    }
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) {
        dk[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
        dv[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    auto load_rows = [&](int head, int qt, float& l2, float& dl) {
        const int t = qt * BM + tid;
        if (tid < BM && t < doc.len) {
            l2 = a.lse[(int64_t)head * T + tok0 + t] * kLog2e;
            dl = a.delta[(int64_t)head * T + tok0 + t];
        } else {
            l2 = 0.f;
            dl = 0.f;
        }
    };
    // the device's first query head is at column hc of a row, head h at hc + (h - kvh group) D
    const int64_t qshift = hc - (int64_t)kvh * a.group * D;
    int boff[4], toff[8];
    offsets(lane, boff, toff);
    TileDma2<false> cp;
    cp.init(a.ldq, a.lddo, wave, lane);
    // every head's query tiles from the first that sees the key tile to the document's
    // last; the steps of all heads in turn, group 0 the first half, group 1 the rest
    const int tiles_ = (doc.len + BM - 1) / BM;
    const int first = kt * BN < doc.prefix ? 0 : kt;
    const int per = tiles_ - first;
    const int nsteps = nh * per;
    const int half = KG > 1 ? (nsteps + 1) / 2 : nsteps;
    const int begin = grp == 0 ? 0 : half;
    const int mine = grp == 0 ? half : nsteps - half;   // <= half
    int head = h0 + begin / per, qt = first + begin % per;
    uint16_t(*qb)[2][BM * D] = qd[grp];
    float(*rv)[2][BM] = rowv[grp];
    float l2r = 0.f, dlr = 0.f;
    if (mine > 0) {
        cp.issue(a.qkv + qshift + (int64_t)head * D, a.ldq, a.dout + (int64_t)head * D, a.lddo,
                 tok0, qt * BM, doc.len, qb[0][0], qb[0][1], wave);
        load_rows(head, qt, l2r, dlr);
        if (tid < BM) { rv[0][0][tid] = l2r; rv[0][1][tid] = dlr; }
    }
    dma::wait_vmcnt<0>();
    __syncthreads();
    for (int i = 0; i < half; ++i) {
        if (i < mine) {
            const int buf = i & 1;
            const uint16_t* qs = qb[buf][0];
            const uint16_t* ds_ = qb[buf][1];
            const bool more = i + 1 < mine;
            const bool wrap = qt + 1 == tiles_;
            const int head2 = head + (wrap ? 1 : 0), qt2 = wrap ? first : qt + 1;
            const auto next = cp.rounds(a.qkv + qshift + (int64_t)head2 * D, a.ldq,
                                        a.dout + (int64_t)head2 * D, a.lddo, tok0, qt2 * BM,
                                        doc.len, qb[buf ^ 1][0], qb[buf ^ 1][1]);
            if (more) load_rows(head2, qt2, l2r, dlr);
            const Score<CAP, BIAS> score(a, head);
            // 32 queries: their scores and dP (lane: key kabs, query 16 j + 4 g + e), then
            // their share of dV and dK
            auto slice = [&](auto sl_, auto mask) {
                constexpr int sl = decltype(sl_)::value;
                constexpr bool MASKED = decltype(mask)::value;
                const float ahead = (float)(qt * BM + 32 * sl + 4 * g - kabs);
                f32x4 p[2], d[2];
#pragma unroll
                for (int jj = 0; jj < 2; ++jj)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        p[jj][e] = score.start(ahead + (float)(16 * jj + e));
                        d[jj][e] = 0.f;
                    }
#pragma unroll
                for (int ks = 0; ks < 4; ++ks) {
#pragma unroll
                    for (int jj = 0; jj < 2; ++jj) {
                        const int j = 2 * sl + jj;
                        const bf16x8 qf =
                            *reinterpret_cast<const bf16x8*>(qs + 16 * j * D + boff[ks]);
                        const bf16x8 of =
                            *reinterpret_cast<const bf16x8*>(ds_ + 16 * j * D + boff[ks]);
                        p[jj] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qf, kf[ks], p[jj], 0, 0, 0);
                        d[jj] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(of, vf[ks], d[jj], 0, 0, 0);
                    }
                    if (sl == 0 && more) cp.round(next, ks, wave);
                }
#pragma unroll
                for (int jj = 0; jj < 2; ++jj)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int ql = 16 * (2 * sl + jj) + 4 * g + e;
                        const int qabs = qt * BM + ql;
                        const bool hidden =
                            MASKED && (kabs >= max(qabs + 1, doc.prefix) || qabs >= doc.len);
                        float pv, dsv = d[jj][e];
                        grad_of(score, p[jj][e], ahead + (float)(16 * jj + e), rv[buf][0][ql],
                                rv[buf][1][ql], hidden, pv, dsv);
                        p[jj][e] = pv;
                        d[jj][e] = dsv;
                        // two at a time: with the series of all eight more spills (1024 us)
                        if constexpr (CAP == kLarge)
                            if (e & 1) __builtin_amdgcn_sched_barrier(0);
                    }
                const bf16x8 pf = pack_pair(p[0], p[1]), sf = pack_pair(d[0], d[1]);
#pragma unroll
                for (int dt = 0; dt < 8; ++dt) {
                    const bf16x8 of = frag_tr_at(ds_ + 32 * sl * D + toff[dt]);
                    const bf16x8 qf = frag_tr_at(qs + 32 * sl * D + toff[dt]);
                    dv[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(of, pf, dv[dt], 0, 0, 0);
                    dk[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qf, sf, dk[dt], 0, 0, 0);
                }
            };
            const std::integral_constant<int, 0> s0;
            const std::integral_constant<int, 1> s1;
            // a tile whose first row sees the whole key tile, and that ends inside the
            // document, needs no mask
            if ((kt + 1) * BN <= max(qt * BM + 1, doc.prefix) && (qt + 1) * BM <= doc.len) {
                slice(s0, std::false_type{});
                slice(s1, std::false_type{});
            } else {
                slice(s0, std::true_type{});
                if (qt * BM + 32 < doc.len) slice(s1, std::true_type{});
            }
            if (more && tid < BM) {
                rv[buf ^ 1][0][tid] = l2r;
                rv[buf ^ 1][1][tid] = dlr;
            }
            head = head2;
            qt = qt2;
        }
        dma::wait_vmcnt<0>();
        __syncthreads();
    }
    if constexpr (KG > 1) {
        f32x4* x = reinterpret_cast<f32x4*>(&qd[1][0][0][0]);
        if (grp == 1) {
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) {
                x[((wave * 2 + 0) * 8 + dt) * 64 + lane] = dk[dt];
                x[((wave * 2 + 1) * 8 + dt) * 64 + lane] = dv[dt];
            }
        }
        __syncthreads();
        if (grp == 1) return;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) {
            dk[dt] += x[((wave * 2 + 0) * 8 + dt) * 64 + lane];
            dv[dt] += x[((wave * 2 + 1) * 8 + dt) * 64 + lane];
        }
    }
    if (kabs >= doc.len) return;
    if (a.parts > 1) {
        float* to = a.sums + (((int64_t)part * T + tok0 + kabs) * a.kv_heads + kvh) * 2 * D;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) {
            *reinterpret_cast<f32x4*>(to + 16 * dt + 4 * g) = dk[dt];
            *reinterpret_cast<f32x4*>(to + D + 16 * dt + 4 * g) = dv[dt];
        }
        return;
    }
    uint16_t* row = a.dqkv + (tok0 + kabs) * a.lddq + hc + (int64_t)a.group * D;
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) {
        const f32x4 k = dk[dt] * a.inv_sqrt_d, v = dv[dt];
        *reinterpret_cast<u32x2*>(row + 16 * dt + 4 * g) =
            u32x2{pack_bf16x2(k[0], k[1]), pack_bf16x2(k[2], k[3])};
        *reinterpret_cast<u32x2*>(row + D + 16 * dt + 4 * g) =
            u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
    }
}

// dK, dV of a row and key head from the parts' sums, in order; 32 lanes each.
__global__ __launch_bounds__(256) void docs_join_kernel(BwdArgs a) {
    const int64_t i = (int64_t)blockIdx.x * 8 + threadIdx.x / 32;
    const int64_t t = i / a.kv_heads;
    const int kvh = (int)(i - t * a.kv_heads), c = (threadIdx.x & 31) * 8;
    if (t >= a.tokens || t < a.cu[0] || t >= a.cu[a.n_docs]) return;
    float s[8] = {};
    for (int p = 0; p < a.parts; ++p) {
        wave::Eight<float> v;
        v.load(a.sums + (((int64_t)p * a.tokens + t) * a.kv_heads + kvh) * 2 * D + c);
        float f[8];
        v.get(f);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] += f[e];
    }
    if (c < D) {
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] *= a.inv_sqrt_d;
    }
    wave::Eight<uint16_t> o;
    o.set(s);
    o.store(a.dqkv + t * a.lddq + ((int64_t)kvh * (a.group + 2) + a.group) * D + c);
}

template <int RB, int KG, Cap CAP, bool BIAS>
__global__ __launch_bounds__(NTHR * KG + (KG > 1 ? NTHR : 0), KG > 1 ? 3 : 2)
void docs_dq_kernel(BwdArgs a) {
    constexpr int QT = 64 * RB;
    constexpr bool PRODUCERS = KG > 1;
    __shared__ __attribute__((aligned(16))) uint16_t kv[KG][2][2][BN * D];   // [grp][buf][K|V]
    const int lane = threadIdx.x & 63, g = lane >> 4;
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool producer = PRODUCERS && wv >= KG * NWAVE;
    const int grp = producer ? 0 : wv / NWAVE, wave = wv % NWAVE;
    const int heads = a.kv_heads * a.group;
    const int head = blockIdx.x % heads, kvh = head / a.group;
    Doc doc = {};
    if (!find_tile<RB == 2 ? 7 : 6, false>(a, (int)(blockIdx.x / heads), doc)) return;
    const int qt = doc.tile;
    const int64_t tok0 = doc.tok0, T = a.tokens;
    const int64_t hc = (int64_t)kvh * (a.group + 2) * D;
    const int64_t qc = hc + (int64_t)(head - kvh * a.group) * D;

    const uint16_t* kbase = a.qkv + hc + (int64_t)a.group * D;
    const uint16_t* vbase = kbase + D;
    const int last = min(qt * QT + QT, doc.len) - 1;
    const int nk = (max(last + 1, doc.prefix) + BN - 1) / BN;
    const int half = KG > 1 ? (nk + 1) / 2 : nk;
    const int k0 = grp == 0 ? 0 : half;
    const int mine = grp == 0 ? half : nk - half;   // <= half
    uint16_t(*kb)[2][BN * D] = kv[grp];
    TileDma2<false> cp;
    cp.init(a.ldq, a.ldq, wave, lane);
    if constexpr (PRODUCERS) {
        if (producer) {
            produce<KG>(cp, kbase, vbase, a.ldq, tok0, nk, doc.len, kv, wave);
            return;
        }
    } else {
        if (mine > 0)
            cp.issue(kbase, a.ldq, vbase, a.ldq, tok0, k0 * BN, doc.len, kb[0][0], kb[0][1], wave);
        dma::wait_vmcnt<0>();
    }
    int qabs[RB], limit[RB];
    bf16x8 qf[RB][4], of[RB][4];
    float l2[RB], dl[RB];
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        qabs[r] = qt * QT + 64 * r + wave * 16 + (lane & 15);
        limit[r] = max(qabs[r] + 1, doc.prefix);
        l2[r] = 0.f;
        dl[r] = 0.f;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            if (qabs[r] < doc.len) {
                qf[r][ks] = *reinterpret_cast<const bf16x8*>(
                    a.qkv + (tok0 + qabs[r]) * a.ldq + qc + 32 * ks + 8 * g);
                of[r][ks] = *reinterpret_cast<const bf16x8*>(
                    a.dout + (tok0 + qabs[r]) * a.lddo + (int64_t)head * D + 32 * ks + 8 * g);
            } else {
                qf[r][ks] = __builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0});
                of[r][ks] = qf[r][ks];
            }
        }
        // delta of the row: each of its four lanes sums 32 columns
        float acc = 0.f;
        if (qabs[r] < doc.len) {
            l2[r] = a.lse[(int64_t)head * T + tok0 + qabs[r]] * kLog2e;
            const uint16_t* orow = a.out + (tok0 + qabs[r]) * a.ldo + (int64_t)head * D;
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) {
                const u32x4 o = *reinterpret_cast<const u32x4*>(orow + 32 * ks + 8 * g);
                const u32x4 d = __builtin_bit_cast(u32x4, of[r][ks]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    acc += __uint_as_float(o[e] << 16) * __uint_as_float(d[e] << 16);
                    acc +=
                        __uint_as_float(o[e] & 0xffff0000u) * __uint_as_float(d[e] & 0xffff0000u);
                }
            }
        }
        dl[r] = row_sum4(acc);   // every lane of the wave takes part
        // the dK/dV kernel, launched after this one, reads it
        if (grp == 0 && g == 0 && qabs[r] < doc.len)
            a.delta[(int64_t)head * T + tok0 + qabs[r]] = dl[r];
    }
    const Score<CAP, BIAS> score(a, head);
    f32x4 dq[RB][8];
#pragma unroll
    for (int r = 0; r < RB; ++r)
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) dq[r][dt] = f32x4{0.f, 0.f, 0.f, 0.f};

    int boff[4], toff[8];
    offsets(lane, boff, toff);
    __syncthreads();
    const int clear = max(qt * QT + 1, doc.prefix);
    int reach[RB];                       // keys that any row of a block sees
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        const int top = qt * QT + 64 * r;
        reach[r] = top < doc.len ? max(min(top + 64, doc.len), doc.prefix) : 0;
    }
    auto step = [&](int i, auto r0, auto r1, auto mask) {
        constexpr int R0 = decltype(r0)::value, R1 = decltype(r1)::value;
        constexpr bool MASKED = decltype(mask)::value;
        const int kt = k0 + i;
        const uint16_t* ks_ = kb[i & 1][0];
        const uint16_t* vs_ = kb[i & 1][1];
        const bool more = !PRODUCERS && i + 1 < mine;
        const auto next = cp.rounds(kbase, a.ldq, vbase, a.ldq, tok0, (kt + 1) * BN, doc.len,
                                    kb[(i + 1) & 1][0], kb[(i + 1) & 1][1]);
        constexpr int JG = RB == 1 ? 4 : 2;
        f32x4 dsv[RB][4];
#pragma unroll
        for (int j0 = 0; j0 < 4; j0 += JG) {
            f32x4 sacc[RB][JG], dacc[RB][JG];
#pragma unroll
            for (int r = R0; r < R1; ++r)
#pragma unroll
                for (int jj = 0; jj < JG; ++jj)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int n = kt * BN + 16 * (j0 + jj) + 4 * g + e;
                        sacc[r][jj][e] = score.start((float)(qabs[r] - n));
                        dacc[r][jj][e] = 0.f;
                    }
#pragma unroll
            for (int ks = 0; ks < 4; ++ks)
#pragma unroll
                for (int jj = 0; jj < JG; ++jj) {
                    const int j = j0 + jj;
                    const bf16x8 kf = *reinterpret_cast<const bf16x8*>(ks_ + 16 * j * D + boff[ks]);
                    const bf16x8 vf = *reinterpret_cast<const bf16x8*>(vs_ + 16 * j * D + boff[ks]);
#pragma unroll
                    for (int r = R0; r < R1; ++r) {
                        sacc[r][jj] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[r][ks],
                                                                              sacc[r][jj], 0, 0, 0);
                        dacc[r][jj] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, of[r][ks],
                                                                              dacc[r][jj], 0, 0, 0);
                    }
                    if (j0 == 0 && jj == JG - 1 && more) cp.round(next, ks, wave);
                }
#pragma unroll
            for (int jj = 0; jj < JG; ++jj)
#pragma unroll
                for (int r = R0; r < R1; ++r)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int n = kt * BN + 16 * (j0 + jj) + 4 * g + e;
                        float p, d = dacc[r][jj][e];
                        grad_of(score, sacc[r][jj][e], (float)(qabs[r] - n), l2[r], dl[r],
                                MASKED && n >= limit[r], p, d);
                        dsv[r][j0 + jj][e] = d;
                    }
        }
#pragma unroll
        for (int sl = 0; sl < 2; ++sl) {
            bf16x8 sf[RB];
#pragma unroll
            for (int r = R0; r < R1; ++r) sf[r] = pack_pair(dsv[r][2 * sl], dsv[r][2 * sl + 1]);
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) {
                const bf16x8 kt_ = frag_tr_at(ks_ + 32 * sl * D + toff[dt]);
#pragma unroll
                for (int r = R0; r < R1; ++r)
                    dq[r][dt] =
                        __builtin_amdgcn_mfma_f32_16x16x32_bf16(kt_, sf[r], dq[r][dt], 0, 0, 0);
            }
        }
    };
    const std::integral_constant<int, 0> b0;
    const std::integral_constant<int, 1> b1;
    const std::integral_constant<int, RB> bn;
    auto end_step = [&] {
        dma::wait_vmcnt<0>();
        __syncthreads();
    };
    // as in the forward
    const int whole = max(0, min(clear / BN - k0, mine));
    int i = 0;
    if (RB == 1 || reach[RB - 1] > 0) {
        for (; i < whole; ++i) {
            step(i, b0, bn, std::false_type{});
            end_step();
        }
        for (; i < mine && (RB == 1 || (k0 + i) * BN < reach[0]); ++i) {
            step(i, b0, bn, std::true_type{});
            end_step();
        }
        if constexpr (RB > 1)
            for (; i < mine; ++i) {
                step(i, b1, bn, std::true_type{});
                end_step();
            }
    } else {
        for (; i < mine; ++i) {
            step(i, b0, b1, std::true_type{});
            end_step();
        }
    }
    for (; i < half; ++i) end_step();
    if constexpr (KG > 1) {
        f32x4* x = reinterpret_cast<f32x4*>(&kv[1][0][0][0]);
        if (grp == 1) {
#pragma unroll
            for (int r = 0; r < RB; ++r)
#pragma unroll
                for (int dt = 0; dt < 8; ++dt)
                    x[((wave * RB + r) * 8 + dt) * 64 + lane] = dq[r][dt];
        }
        __syncthreads();
        if (grp == 1) return;
#pragma unroll
        for (int r = 0; r < RB; ++r)
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) dq[r][dt] += x[((wave * RB + r) * 8 + dt) * 64 + lane];
    }
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        if (qabs[r] >= doc.len) continue;
        uint16_t* row = a.dqkv + (tok0 + qabs[r]) * a.lddq + qc;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) {
            const u32x2 w = {pack_bf16x2(dq[r][dt][0] * a.inv_sqrt_d, dq[r][dt][1] * a.inv_sqrt_d),
                             pack_bf16x2(dq[r][dt][2] * a.inv_sqrt_d, dq[r][dt][3] * a.inv_sqrt_d)};
            *reinterpret_cast<u32x2*>(row + 16 * dt + 4 * g) = w;
        }
    }
}

// ---------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------
// The kernels of 128 rows (64 keys for dK and dV) are taken where they leave `full_tiles`
// 64-row tiles of all heads; below that those of 64 rows whose loops are split over two
// groups of waves.  These halve the long loops of an emptier chip, but take twice the
// starts, which is most of a short document's time: four tiles per CU for documents of more
// than 2048 rows on the average, fewer for shorter ones (empty documents count).  Whole and
// split, forward + backward, us:
//   rows of 128: 288 tiles 11 + 25 and 14 + 36;
//   of 520: 292 tiles 20 + 47 and 17 + 42, 584 tiles 22 + 54 and 26 + 71;
//   of 1024: 512 tiles 27 + 75 and 24 + 68, 768 tiles 30 + 84 and 35 + 100;
//   of 2048: 512 tiles 44 + 131 and 33 + 102, 768 tiles 48 + 140 and 49 + 154;
//   of 4096 and 2048: 768 tiles 85 + 253 and 69 + 211; of 4096: 1024 tiles 96 + 310 and
//   103 + 350.
int64_t full_tiles(int64_t tokens, int n_docs) {
    const int64_t rows = tokens / n_docs;
    return 256 * (rows < 256 ? 1 : rows < 1024 ? 2 : rows <= 2048 ? 3 : 4);
}

void fill(Common& c, const DocsView& d, const uint16_t* qkv, int64_t ldq, int64_t tokens,
          int kv_heads, int group) {
    c.qkv = qkv;
    c.ldq = ldq;
    c.cu = d.cu;
    c.prefix = d.prefix;
    c.slopes = d.slopes;
    c.tokens = tokens;
    c.n_docs = d.n_docs;
    c.kv_heads = kv_heads;
    c.group = group;
    c.slots = 0;
    const float root = sqrtf((float)D);
    c.scale_log2 = kLog2e / root;
    c.root_d = root;
    // finite for the smallest caps too: products of 0 score 0
    c.cap_in = d.cap > 0.f ? std::min(2.f * kLog2e / (root * d.cap), FLT_MAX) : 0.f;
    c.cap_y = d.cap > 0.f ? std::min(1.f / (root * d.cap), FLT_MAX) : 0.f;
    c.cap_log2 = d.cap * kLog2e;
}
// Slots of tiles of `rows` rows: up to cu[n] / rows + n.
int64_t slots_of(int64_t tokens, int rows, int n_docs) { return tokens / rows + n_docs; }

// Divisions of a group's heads for the dK/dV kernel: as many as it takes for `tiles` of 64
// keys.  Four per CU (16 heads of two key heads, one document of 4096 rows: 317 us; for two
// per CU 391, for eight 349); where documents have fewer than 512 rows, what fills the chip,
// since each division starts anew and leaves sums to be joined.  Backward by both rules, what
// fills the chip and four per CU, us, ragged documents of an average of
//   128 rows, heads of 4 x 3: 62 and 75; 1 x 12: 79 and 68; 4 x 5: 108 and 132;
//   256: 80 and 74; 84 and 88; 151 and 156;      350: 85 and 79; 90 and 95; 163 and 171;
//   450: 98 and 86; 101 and 102; 193 and 198;    512: 125 and 101; 118 and 119; 231 and 202;
//   650: 126 and 100; 122 and 111; 253 and 238;  1024: 158 and 128; 168 and 168; 297 and 296.
// Between 200 and 500 the layouts differ in which is faster, by up to 13%.
constexpr int64_t kPartTiles = 1024;
int64_t part_tiles(int64_t tokens, int n_docs) {
    return tokens / n_docs < 512 ? full_tiles(tokens, n_docs) : kPartTiles;
}
int dkv_parts(int64_t tokens, int kv_heads, int group, int64_t most, int* heads) {
    const int64_t tiles = std::max<int64_t>(1, tokens / BM) * kv_heads;
    const int64_t want = std::min<int64_t>(group, (most + tiles - 1) / tiles);
    *heads = (int)((group + want - 1) / want);
    return (group + *heads - 1) / *heads;
}
int64_t delta_floats(int64_t tokens, int heads) { return (tokens * heads + 63) / 64 * 64; }

template <int RB, int KG, Cap CAP, bool BIAS>
void fwd(FwdArgs& a, hipStream_t s) {
    a.slots = (int)slots_of(a.tokens, 64 * RB, a.n_docs);
    docs_fwd_kernel<RB, KG, CAP, BIAS>
        <<<dim3((unsigned)((int64_t)a.slots * a.kv_heads * a.group)), KG > 1 ? 3 * NTHR : NTHR, 0,
           s>>>(a);
}
// Whether the kernels that split their loops, of `threads` threads, can be launched: empty
// documents have slots too.
bool split_fits(const Common& a, int64_t heads, int threads) {
    return fits_launch(slots_of(a.tokens, 64, a.n_docs) * heads, threads);
}
template <Cap CAP, bool BIAS>
void fwd_of(FwdArgs& a, hipStream_t s) {
    const int64_t tiles = (a.tokens + 127) / 128 * a.kv_heads * a.group;
    if (2 * tiles >= full_tiles(a.tokens, a.n_docs) ||
        !split_fits(a, a.kv_heads * a.group, 3 * NTHR))
        fwd<2, 1, CAP, BIAS>(a, s);
    else fwd<1, 2, CAP, BIAS>(a, s);
}

template <Cap CAP, bool BIAS>
hipError_t bwd_of(BwdArgs& a, hipStream_t s) {
    const int heads = a.kv_heads * a.group;
    const int64_t s64 = slots_of(a.tokens, 64, a.n_docs);
    const int64_t full = full_tiles(a.tokens, a.n_docs);
    const bool split = (a.tokens + 63) / 64 * heads < full && split_fits(a, heads, 3 * NTHR);
    if (split) {
        a.slots = (int)s64;
        docs_dq_kernel<1, 2, CAP, BIAS>
            <<<dim3((unsigned)(s64 * heads)), 3 * NTHR, 0, s>>>(a);
    } else {
        a.slots = (int)slots_of(a.tokens, 128, a.n_docs);
        docs_dq_kernel<2, 1, CAP, BIAS>
            <<<dim3((unsigned)((int64_t)a.slots * heads)), NTHR, 0, s>>>(a);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int per_slot = a.kv_heads * a.parts;
    a.slots = (int)s64;
    if ((a.tokens + 63) / 64 * per_slot < full && split_fits(a, per_slot, 2 * NTHR)) {
        docs_dkv_kernel<2, CAP, BIAS><<<dim3((unsigned)(s64 * per_slot)), 2 * NTHR, 0, s>>>(a);
    } else {
        docs_dkv_kernel<1, CAP, BIAS><<<dim3((unsigned)(s64 * per_slot)), NTHR, 0, s>>>(a);
    }
    return hipGetLastError();
}

}  // namespace

// Enough for any number of documents (fewer tiles never give more parts) and for every
// smaller number of rows: the sums of more divisions of fewer rows may be the larger ones, so
// each number of divisions counts with the most rows that take it.
int64_t docs_attention_ws_floats(int64_t tokens, int kv_heads, int group) {
    int64_t sums = 0;
    for (int want = 2; want <= group; ++want) {
        const int most = (int)(kPartTiles - 1) / (want - 1) / kv_heads;   // tiles of 64 rows
        if (most < 1) break;
        const int heads = (group + want - 1) / want, parts = (group + heads - 1) / heads;
        sums = std::max(sums, parts * std::min<int64_t>(tokens, (int64_t)BM * most + BM - 1));
    }
    return delta_floats(tokens, kv_heads * group) + sums * kv_heads * 2 * D;
}

hipError_t launch_docs_attention(const DocsAttentionProblem& p, hipStream_t s) {
    if (p.tokens == 0 || p.docs.n_docs == 0) return hipSuccess;
    FwdArgs a;
    fill(a, p.docs, p.qkv, p.ldq, p.tokens, p.kv_heads, p.group);
    a.out = p.out;
    a.ldo = p.ldo;
    a.lse = p.lse;
    if (p.docs.cap > kSmallCap) {
        if (p.docs.slopes) fwd_of<kLarge, true>(a, s);
        else fwd_of<kLarge, false>(a, s);
    } else if (p.docs.cap > 0.f) {
        if (p.docs.slopes) fwd_of<kSmall, true>(a, s);
        else fwd_of<kSmall, false>(a, s);
    } else {
        if (p.docs.slopes) fwd_of<kNoCap, true>(a, s);
        else fwd_of<kNoCap, false>(a, s);
    }
    return hipGetLastError();
}

hipError_t launch_docs_attention_bwd(const DocsAttentionBwdProblem& p, hipStream_t s) {
    if (p.tokens == 0 || p.docs.n_docs == 0) return hipSuccess;
    BwdArgs a;
    fill(a, p.docs, p.qkv, p.ldq, p.tokens, p.kv_heads, p.group);
    a.out = p.out; a.ldo = p.ldo;
    a.dout = p.dout; a.lddo = p.lddo;
    a.lse = p.lse;
    a.delta = p.ws;
    a.sums = p.ws + delta_floats(p.tokens, p.kv_heads * p.group);
    a.dqkv = p.dqkv; a.lddq = p.lddq;
    a.parts = dkv_parts(p.tokens, p.kv_heads, p.group, part_tiles(p.tokens, p.docs.n_docs),
                        &a.part_heads);
    a.inv_sqrt_d = 1.0f / sqrtf((float)D);
    hipError_t e;
    if (p.docs.cap > kSmallCap) {
        if (p.docs.slopes) e = bwd_of<kLarge, true>(a, s);
        else e = bwd_of<kLarge, false>(a, s);
    } else if (p.docs.cap > 0.f) {
        if (p.docs.slopes) e = bwd_of<kSmall, true>(a, s);
        else e = bwd_of<kSmall, false>(a, s);
    } else {
        if (p.docs.slopes) e = bwd_of<kNoCap, true>(a, s);
        else e = bwd_of<kNoCap, false>(a, s);
    }
    if (e != hipSuccess || a.parts < 2) return e;
    docs_join_kernel<<<dim3((unsigned)((p.tokens * p.kv_heads + 7) / 8)), 256, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace atp
