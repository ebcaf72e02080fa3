// Tiles of the attention kernels: LDS layouts of 64-row tiles of 128 columns,
// fragments read from them, the copies that fill them, and the exchanges of the
// four lanes that hold a score row.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "lds_dma.h"

namespace atp {
namespace tiles {

constexpr int D = 128;          // head dimension
constexpr int BM = 64;          // query rows per workgroup
constexpr int BN = 64;          // keys per step
constexpr int NWAVE = 4;
constexpr int NTHR = NWAVE * 64;
// forward softmax: largest base-2 gain of a row maximum absorbed without
// rescaling the running output (weights stay below 2^8, exact in bf16's range)
constexpr float kSlack = 8.f;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef short i16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) i16x4 lds_i16x4;

// 16-byte chunk c of tile row n is kept at these places: distinct banks for the fragment
// reads (both) and for the transposing reads (vpos).
__device__ __forceinline__ int kpos(int n, int c) { return c ^ (n & 15); }
__device__ __forceinline__ int vpos(int n, int c) { return c ^ (2 * (n & 3) + 8 * ((n >> 2) & 1)); }

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// The four lanes l, l ^ 16, l ^ 32, l ^ 48 hold one score row's columns.
// Their maximum and sum come from gfx950's lane swaps (v_permlane16_swap
// pairs the 16-lane rows 0-1 and 2-3, v_permlane32_swap the two halves),
// which stay in the VALU instead of a round trip through LDS.  With both
// operands x, the first result is the lower member of each pair and the
// second the upper, so every lane of the four combines the same values in
// the same order: (r0 op r1) op (r2 op r3), bit-identical in all four.
__device__ __forceinline__ float row_max4(float x) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x),
                                                    false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x),
                                                    false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// Maximum of a lane's 16 scores of one row block as a shallow tree: five
// independent three-input maxima over 15 scores, two more over those and
// the last score, and one two-input maximum (three dependent steps instead
// of a chain through all sixteen).
__device__ __forceinline__ float max16(const f32x4 (&v)[4]) {
    const float a = fmaxf(fmaxf(v[0][0], v[0][1]), v[0][2]);
    const float b = fmaxf(fmaxf(v[0][3], v[1][0]), v[1][1]);
    const float c = fmaxf(fmaxf(v[1][2], v[1][3]), v[2][0]);
    const float d = fmaxf(fmaxf(v[2][1], v[2][2]), v[2][3]);
    const float e = fmaxf(fmaxf(v[3][0], v[3][1]), v[3][2]);
    return fmaxf(fmaxf(fmaxf(a, b), c), fmaxf(fmaxf(d, e), v[3][3]));
}

__device__ __forceinline__ float row_sum4(float x) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x),
                                                    false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x),
                                                    false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// Two floats to bf16 (round to nearest even: one v_cvt_pk_bf16_f32).
__device__ __forceinline__ uint32_t pack_bf16x2(float a, float b) {
    const f32x2 v = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}

// Element offsets of a lane's transposing reads of a [key][d] tile in the
// vpos layout, rows 4 g + lane%16 / 4 (+ 32 sl, + 16 for the second read:
// same swizzle), columns 16 dt + 4 (lane % 4): one per dt.
__device__ __forceinline__ int tr_offset(int lane, int dt) {
    const int g = lane >> 4, j16 = lane & 15;
    const int r = 4 * g + (j16 >> 2);
    const int col = 16 * dt + 4 * (j16 & 3);
    return r * D + vpos(r, col >> 3) * 8 + (col & 7);
}

// Rows [n0, n0 + 64) of two 128-column runs of one sequence's token rows
// straight into two LDS tiles (the first in the kpos layout when KPOS0,
// else vpos; the second in vpos): copy instruction i (wave w issues
// i = w + 4 r) fills slots 64 i .. 64 i + 63, i.e. row 4 w + 16 r + lane/16,
// position lane % 16, so the lane fetches the chunk its slot holds (kpos and
// vpos are XORs, their own inverses, and depend only on the row's low four
// bits).  Rows past the sequence are past the range and read zeros.
template <bool KPOS0>
struct TileDma2 {
    uint32_t off0, off1, st0, st1;   // lane offsets of r = 0, bytes per 16 rows
    __device__ __forceinline__ void init(int64_t ld0, int64_t ld1, int wave, int lane) {
        const int n = 4 * wave + lane / 16, pos = lane % 16;
        const int c0 = KPOS0 ? kpos(n, pos) : vpos(n, pos);
        off0 = (uint32_t)((n * ld0 + 8 * c0) * 2);
        off1 = (uint32_t)((n * ld1 + 8 * vpos(n, pos)) * 2);
        st0 = (uint32_t)(16 * ld0 * 2);
        st1 = (uint32_t)(16 * ld1 * 2);
    }
    __device__ __forceinline__ void issue(const uint16_t* b0, int64_t ld0, const uint16_t* b1,
                                          int64_t ld1, int64_t tok0, int n0, int seq, uint16_t* t0,
                                          uint16_t* t1, int wave) const {
        const int64_t left = seq - n0;
        const int64_t vr = left < 0 ? 0 : (left < 64 ? left : 64);
        const dma::u32x4 r0 = dma::rsrc_words(b0 + (tok0 + n0) * ld0, vr * ld0 * 2);
        const dma::u32x4 r1 = dma::rsrc_words(b1 + (tok0 + n0) * ld1, vr * ld1 * 2);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int ins = wave + NWAVE * r;
            dma::lds_dma16(r0, t0 + ins * 64 * 8, off0 + r * st0, 0u);
            dma::lds_dma16(r1, t1 + ins * 64 * 8, off1 + r * st1, 0u);
        }
    }
    // The same tile in four rounds (r = 0..3) that the main loops spread over
    // their score products, one per head-dimension slice: a wave stands at a
    // copy instruction while the CU's memory path is busy, so a burst of all
    // eight copies of every wave at the start of a step held the first
    // products up for as long as the path needs for the tile (wide share
    // forward 67 -> 60 us and backward 224 -> 206, GPT-3 share 33 -> 27.5 and 86 ->
    // 78; the second operand's copies during the second products: 63 and 219).
    struct Rounds {
        dma::u32x4 r0, r1;
        uint16_t *t0, *t1;
    };
    __device__ __forceinline__ Rounds rounds(const uint16_t* b0, int64_t ld0, const uint16_t* b1,
                                             int64_t ld1, int64_t tok0, int n0, int seq,
                                             uint16_t* t0, uint16_t* t1) const {
        const int64_t left = seq - n0;
        const int64_t vr = left < 0 ? 0 : (left < 64 ? left : 64);
        return Rounds{dma::rsrc_words(b0 + (tok0 + n0) * ld0, vr * ld0 * 2),
                      dma::rsrc_words(b1 + (tok0 + n0) * ld1, vr * ld1 * 2), t0, t1};
    }
    __device__ __forceinline__ void round(const Rounds& q, int r, int wave) const {
        const int ins = wave + NWAVE * r;
        dma::lds_dma16(q.r0, q.t0 + ins * 64 * 8, off0 + r * st0, 0u);
        dma::lds_dma16(q.r1, q.t1 + ins * 64 * 8, off1 + r * st1, 0u);
    }
};

// The four producer waves of a kernel whose KG groups of consumer waves split
// nkt key tiles (group 0 the first half, group 1 the rest): they copy every
// group's K and V tile of step i into its buffer i & 1 before barrier i, at
// which all consumers have finished step i - 1 (so step i - 2, the buffer's last
// reader, since barrier i - 1).  Consumer waves then never stand at a copy
// instruction (GPT-3 share forward 28 -> 25.4 us, one head of 4096 tokens 46.5 ->
// 39.5).  Their barriers: one before the loop, one per step, one in the merge.
template <int KG, class Cp>
__device__ __forceinline__ void produce(const Cp& cp, const uint16_t* kbase,
                                        const uint16_t* vbase, int64_t ld, int64_t tok0, int nkt,
                                        int seq, uint16_t (&kv)[KG][2][2][BN * D], int wave) {
    const int half = (nkt + 1) / 2;
    for (int i = 0; i <= half; ++i) {
        if (i < half) {
#pragma unroll
            for (int gr = 0; gr < KG; ++gr)
                if (i < (gr == 0 ? half : nkt - half))
                    cp.issue(kbase, ld, vbase, ld, tok0, (gr * half + i) * BN, seq,
                             kv[gr][i & 1][0], kv[gr][i & 1][1], wave);
            dma::wait_vmcnt<0>();
        }
        __syncthreads();
    }
    __syncthreads();
}

// Lane offsets into a [row][d] tile in the vpos layout: ds_read_b128
// fragments of row 16 j + lane%16, chunk 4 ks + lane/16 (boff[ks]; j adds
// 16 rows, same swizzle), and transposing reads (toff[dt], see tr_offset).
__device__ __forceinline__ void offsets(int lane, int (&boff)[4], int (&toff)[8]) {
    const int g = lane >> 4, l16 = lane & 15;
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) boff[ks] = l16 * D + vpos(l16, 4 * ks + g) * 8;
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) toff[dt] = tr_offset(lane, dt);
}
// Transposing fragment at p (rows p, p + 16 D): lane (group g, j) gets
// column 16 dt + j, keys or queries rb + 4 g + 0..3 and rb + 16 + 4 g + 0..3.
__device__ __forceinline__ bf16x8 frag_tr_at(const uint16_t* p) {
    const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)p);
    const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(p + 16 * D));
    const i16x8 v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    return __builtin_bit_cast(bf16x8, v);
}
__device__ __forceinline__ bf16x8 pack_pair(const f32x4& a, const f32x4& b) {
    const u32x4 w = {pack_bf16x2(a[0], a[1]), pack_bf16x2(a[2], a[3]), pack_bf16x2(b[0], b[1]),
                     pack_bf16x2(b[2], b[3])};
    return __builtin_bit_cast(bf16x8, w);
}

}  // namespace tiles
}  // namespace atp
