// Sums over the lanes of a wave and conversions of eight values, shared by the
// kernels that keep rows in registers.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace atp {
namespace wave {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

template <int CTRL>
__device__ __forceinline__ float dpp_add(float x) {
    const int y = __builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true);
    return x + __int_as_float(y);
}

// Sum over the 64 lanes, the same bits in every lane: within rows of 16 by
// exchanges of neighbours, pairs, quads (mirror) and halves, then the rows by
// gfx950's lane swaps.
__device__ __forceinline__ float sum64(float x) {
    x = dpp_add<0xb1>(x);     // quad_perm [1, 0, 3, 2]
    x = dpp_add<0x4e>(x);     // quad_perm [2, 3, 0, 1]
    x = dpp_add<0x141>(x);    // row_half_mirror
    x = dpp_add<0x140>(x);    // row_mirror
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                    false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                    false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// Two floats to bf16, nearest even (one v_cvt_pk_bf16_f32).
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    const f32x2 v = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}
__device__ __forceinline__ u32x4 pack8(const float* v) {
    return u32x4{pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7])};
}
__device__ __forceinline__ void unpack8(const u32x4& w, float* v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}

// Eight consecutive values as they are stored: 16 bytes of bf16 or 32 of fp32.
template <class T>
struct Eight;
template <>
struct Eight<uint16_t> {
    u32x4 w;
    __device__ __forceinline__ void load(const uint16_t* p) {
        w = *reinterpret_cast<const u32x4*>(p);
    }
    __device__ __forceinline__ void store(uint16_t* p) const { *reinterpret_cast<u32x4*>(p) = w; }
    __device__ __forceinline__ void get(float* v) const { unpack8(w, v); }
    __device__ __forceinline__ void set(const float* v) { w = pack8(v); }
};
template <>
struct Eight<float> {
    f32x4 a, b;
    __device__ __forceinline__ void load(const float* p) {
        a = *reinterpret_cast<const f32x4*>(p);
        b = *reinterpret_cast<const f32x4*>(p + 4);
    }
    __device__ __forceinline__ void store(float* p) const {
        *reinterpret_cast<f32x4*>(p) = a;
        *reinterpret_cast<f32x4*>(p + 4) = b;
    }
    __device__ __forceinline__ void get(float* v) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[i] = a[i];
            v[4 + i] = b[i];
        }
    }
    __device__ __forceinline__ void set(const float* v) {
        a = f32x4{v[0], v[1], v[2], v[3]};
        b = f32x4{v[4], v[5], v[6], v[7]};
    }
};

}  // namespace wave
}  // namespace atp
