// Keys and values of new tokens into a paged cache of 8-bit codes (lsh_cache_write).
//
// Code: OCP e4m3 (largest value 448), value = code * scale, one fp32 scale for each block and head, of k and of v.  The scale is
// the smallest power of two with amax <= 448 * scale, so a division by it is exact and a value errs by its rounding to e4m3 alone
// (half a step: 2^-4 of it, 2^-10 * scale near zero).  A block that gets a larger value gets a larger scale, and its earlier
// codes are divided by the ratio: exact for a power of two, except where a code becomes subnormal.
//
// Layout (chosen for the matrix operands of the attention, so that a wave's loads of 16 bytes per lane are contiguous):
//   k [n_blocks, heads, D / 16, block, 16]   16 of a token's values together, then the next token's
//   v [n_blocks, heads, block / 16, D, 16]   a value of 16 tokens together, then the next value
//
// A workgroup per row, head and block of tokens: it alone writes that head of that block.
#pragma once
#include "beam_select.h"

namespace lshbeam {

struct RowsPitch { int64_t row, token, head; };   // elements; the values of a head lie side by side

struct WriteArgs {
    int T, n_blocks, block, heads, D;
    int per_row;               // blocks that a row's tokens can touch
    const void* k;
    const void* v;
    RowsPitch kp, vp;
    const int32_t* slots;      // [R, T]
    const int32_t* copy_from;  // [R] or null
    uint8_t* codes_k;
    uint8_t* codes_v;
    float* scale_k;            // [n_blocks, heads]
    float* scale_v;
};

// The smallest power of two s (from 2^-126 on) with amax <= 448 s; 0 for amax = 0.
__device__ __forceinline__ float scale_for(float amax) {
    if (!(amax > 0.f)) return 0.f;
    const uint32_t u = __float_as_uint(amax);
    // amax = f 2^e, 1 <= f < 2 (a subnormal amax: e below -126); 448 = 1.75 * 2^8
    const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u);
    return __uint_as_float((uint32_t)(max(e, -126) + 127) << 23);
}

// Four values to four codes, nearest even; NaN and infinities to NaN.
__device__ __forceinline__ uint32_t to_codes(float a, float b, float c, float d) {
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
}
typedef float f32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t scaled_codes(uint32_t w, float ratio) {
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    return to_codes(lo.x * ratio, lo.y * ratio, hi.x * ratio, hi.y * ratio);
}

template <int TYPE> __device__ __forceinline__ float value_at(const void* p, int64_t i) {
    return word_f32<TYPE>(static_cast<const typename WordOf<TYPE>::type*>(p)[i]);
}

// grid = (R * per_row, heads), 256 threads.
template <int TYPE>
__global__ void __launch_bounds__(256) k_cache_write(WriteArgs a) {
    __shared__ float amax[2][4];
    __shared__ int run;
    const int64_t r = blockIdx.x / a.per_row;
    const int piece = blockIdx.x - (int)r * a.per_row, h = blockIdx.y;
    const int32_t* slots = a.slots + r * a.T;
    // the tokens of this block: those whose slots follow the first one's to the block's end
    const int32_t slot0 = slots[0];
    if (slot0 < 0) return;
    const int t0 = max(0, piece * a.block - slot0 % a.block);
    if (t0 >= a.T) return;
    const int32_t slot = slots[t0];
    if (slot < 0 || slot / a.block >= a.n_blocks || (piece > 0 && slot % a.block != 0)) return;
    const int block = slot / a.block, at = slot % a.block;
    if (threadIdx.x == 0) run = min(a.T - t0, a.block - at);
    __syncthreads();
    const int most = min(a.T - t0, a.block - at);
    for (int i = threadIdx.x; i < most; i += 256)
        if (slots[t0 + i] != slot + i) atomicMin(&run, i);
    __syncthreads();
    const int n = run;
    int src = block;
    if (piece == 0 && at > 0 && a.copy_from) {
        const int c = a.copy_from[r];
        if (c >= 0 && c < a.n_blocks) src = c;
    }
    const int64_t k0 = r * a.kp.row + t0 * a.kp.token + h * a.kp.head, v0 = r * a.vp.row + t0 * a.vp.token + h * a.vp.head;
    float mk = 0.f, mv = 0.f;
    for (int i = threadIdx.x; i < n * a.D; i += 256) {
        const int t = i / a.D, d = i - t * a.D;
        const float x = fabsf(value_at<TYPE>(a.k, k0 + t * a.kp.token + d)), y = fabsf(value_at<TYPE>(a.v, v0 + t * a.vp.token + d));
        mk = x < INFINITY ? fmaxf(mk, x) : mk;
        mv = y < INFINITY ? fmaxf(mv, y) : mv;
    }
    mk = wave_max_f32(mk);
    mv = wave_max_f32(mv);
    if (lane_id() == 0) { amax[0][wave_id()] = mk; amax[1][wave_id()] = mv; }
    const int64_t from = (int64_t)src * a.heads + h, to = (int64_t)block * a.heads + h;
    float before[2] = {0.f, 0.f}, scale[2], inverse[2];
    if (at > 0) { before[0] = a.scale_k[from]; before[1] = a.scale_v[from]; }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (!(before[i] > 0.f && before[i] < INFINITY)) before[i] = 0.f;
        scale[i] = fmaxf(before[i], scale_for(fmaxf(fmaxf(amax[i][0], amax[i][1]), fmaxf(amax[i][2], amax[i][3]))));
        inverse[i] = scale[i] > 0.f ? 1.f / scale[i] : 0.f;
    }
    if (threadIdx.x == 0) { a.scale_k[to] = scale[0]; a.scale_v[to] = scale[1]; }
    const int64_t bytes = (int64_t)a.block * a.D;
    // keys: a line of 16 bytes is 16 values of a token
    for (int i = threadIdx.x; i < (at + n) * (a.D >> 4); i += 256) {
        const int c = i / (at + n), t = i - c * (at + n);
        const int64_t line = ((int64_t)c * a.block + t) * 16;
        uint4 w;
        if (t < at) {
            if (src == block && before[0] == scale[0]) continue;
            w = *reinterpret_cast<const uint4*>(a.codes_k + from * bytes + line);
            const float ratio = before[0] * inverse[0];
            w = make_uint4(scaled_codes(w.x, ratio), scaled_codes(w.y, ratio), scaled_codes(w.z, ratio), scaled_codes(w.w, ratio));
        } else {
            const int64_t x = k0 + (t - at) * a.kp.token + c * 16;
            uint32_t u[4];
#pragma unroll
            for (int q = 0; q < 4; ++q)
                u[q] = to_codes(value_at<TYPE>(a.k, x + 4 * q) * inverse[0], value_at<TYPE>(a.k, x + 4 * q + 1) * inverse[0],
                                value_at<TYPE>(a.k, x + 4 * q + 2) * inverse[0], value_at<TYPE>(a.k, x + 4 * q + 3) * inverse[0]);
            w = make_uint4(u[0], u[1], u[2], u[3]);
        }
        *reinterpret_cast<uint4*>(a.codes_k + to * bytes + line) = w;
    }
    // values: a line of 16 bytes is a value of 16 tokens, some of them earlier ones, some new, some that stay
    for (int i = threadIdx.x; i < ((at + n + 15) >> 4) * a.D; i += 256) {
        const int g = i / a.D, d = i - g * a.D;
        const int64_t line = (int64_t)i * 16;
        const bool same = src == block && before[1] == scale[1];
        if (same && 16 * g + 16 <= at) continue;
        const float ratio = before[1] * inverse[1];
        const uint4 stay = *reinterpret_cast<const uint4*>(a.codes_v + to * bytes + line);
        const uint4 old = at > 16 * g ? *reinterpret_cast<const uint4*>(a.codes_v + from * bytes + line) : stay;
        const uint32_t s[4] = {stay.x, stay.y, stay.z, stay.w}, o[4] = {old.x, old.y, old.z, old.w};
        uint32_t u[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint32_t kept = same ? o[q] : scaled_codes(o[q], ratio);
            float x[4];
            uint32_t is_old = 0, is_new = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int t = 16 * g + 4 * q + j;
                x[j] = 0.f;
                if (t < at) is_old |= 0xffu << (8 * j);
                else if (t < at + n) {
                    is_new |= 0xffu << (8 * j);
                    x[j] = value_at<TYPE>(a.v, v0 + (t - at) * a.vp.token + d) * inverse[1];
                }
            }
            u[q] = (kept & is_old) | (to_codes(x[0], x[1], x[2], x[3]) & is_new) | (s[q] & ~(is_old | is_new));
        }
        *reinterpret_cast<uint4*>(a.codes_v + to * bytes + line) = make_uint4(u[0], u[1], u[2], u[3]);
    }
}

}  // namespace lshbeam
