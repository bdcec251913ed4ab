// Values in memory and operands of the matrix instructions, as several kernels take them.
#pragma once
#include "beam_select.h"

namespace lshbeam {

struct RowsPitch { int64_t row, token, head; };   // elements; the values of a head lie side by side

template <int TYPE> __device__ __forceinline__ float value_at(const void* p, int64_t i) {
    return word_f32<TYPE>(static_cast<const typename WordOf<TYPE>::type*>(p)[i]);
}

// Eight values from any element on.
template <int TYPE> __device__ __forceinline__ void load_values(const void* p, int64_t i, float (&x)[8]) {
    using T = typename WordOf<TYPE>::type;
    const T* from = static_cast<const T*>(p) + i;
#pragma unroll
    for (int h = 0; h < (TYPE == kTypeF32 ? 2 : 1); ++h) {
        const Chunk16U<T> v = *reinterpret_cast<const Chunk16U<T>*>(from + 4 * h);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if constexpr (TYPE == kTypeF32) x[4 * h + q] = __uint_as_float(v.w[q]);
            else { x[2 * q] = word_f32<TYPE>((T)(v.w[q] & 0xffffu)); x[2 * q + 1] = word_f32<TYPE>((T)(v.w[q] >> 16)); }
        }
    }
}

template <int TYPE> __device__ __forceinline__ void put_value(void* p, int64_t i, float v) {
    if constexpr (TYPE == kTypeF32) static_cast<float*>(p)[i] = v;
    else if constexpr (TYPE == kTypeF16) static_cast<uint16_t*>(p)[i] = __half_as_ushort(__float2half_rn(v));
    else {
        const uint32_t u = __float_as_uint(v);   // nearest even; a NaN stays one
        static_cast<uint16_t*>(p)[i] = v != v ? (uint16_t)0x7fc0 : (uint16_t)((u + 0x7fffu + (u >> 16 & 1u)) >> 16);
    }
}

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

template <int TYPE> constexpr int kPlanes = TYPE == kTypeBf16 ? 1 : TYPE == kTypeF16 ? 2 : 3;
// Eight values as NP operands that add up to them: each but a rounded single one holds the upper 16 bits of what is left.
template <int NP> __device__ __forceinline__ void planes_of(const float (&x)[8], uint4 (&out)[NP]) {
    if constexpr (NP == 1) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f32x2 v = {x[2 * i], x[2 * i + 1]};
            w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
        }
        out[0] = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
        float rest[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) rest[i] = x[i];
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                w[i] = __builtin_amdgcn_perm(__float_as_uint(rest[2 * i + 1]), __float_as_uint(rest[2 * i]), 0x07060302u);
            out[p] = make_uint4(w[0], w[1], w[2], w[3]);
#pragma unroll
            for (int i = 0; i < 8; ++i) rest[i] -= __uint_as_float(__float_as_uint(rest[i]) & 0xffff0000u);
        }
    }
}

}  // namespace lshbeam
