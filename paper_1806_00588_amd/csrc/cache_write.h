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
__device__ __forceinline__ float finite_size(float m, float x) {   // the larger of m and |x|, if x is finite
    x = fabsf(x);
    return x < INFINITY ? fmaxf(m, x) : m;
}

// A block's earlier tokens, for one head of keys or values: scales, and what becomes of the codes.
struct Earlier { float before, scale, inverse; bool same; };   // same: codes stay as they are, where they are
__device__ __forceinline__ Earlier new_scale(float before, float amax, bool in_place) {
    Earlier e;
    e.before = before > 0.f && before < INFINITY ? before : 0.f;
    e.scale = fmaxf(e.before, scale_for(amax));
    e.inverse = e.scale > 0.f ? 1.f / e.scale : 0.f;
    e.same = in_place && e.before == e.scale;
    return e;
}
// The first `at` tokens' codes with another scale, or in another block.
__device__ __forceinline__ void move_keys(const uint8_t* from, uint8_t* to, int at, int block, int D, const Earlier& e, int thread, int threads) {
    const float ratio = e.before * e.inverse;
    for (int i = thread; i < at * (D >> 4); i += threads) {
        const int c = (int)((unsigned)i / (unsigned)at), t = i - c * at;
        const int64_t line = ((int64_t)c * block + t) * 16;
        uint4 w = *reinterpret_cast<const uint4*>(from + line);
        if (e.before != e.scale) w = make_uint4(scaled_codes(w.x, ratio), scaled_codes(w.y, ratio), scaled_codes(w.z, ratio), scaled_codes(w.w, ratio));
        *reinterpret_cast<uint4*>(to + line) = w;
    }
}

// One token for each row (T = 1), grid = (R, heads), 256 threads: the first half has the keys, the other the values, two of a head
// each.  Bound by latency: slot and values are asked for at once, then the block's scales; its codes only if they change.
// 160 rows of 8 heads of 128, bf16: 5.0 us; the general kernel 8.2.
template <int TYPE>
__global__ void __launch_bounds__(256) k_cache_write_one(WriteArgs a) {
    __shared__ float amax[4];
    const int64_t r = blockIdx.x;
    const int h = blockIdx.y, half = threadIdx.x >> 7, d = 2 * (threadIdx.x & 127);
    const int32_t slot = a.slots[r];
    const int32_t copy = a.copy_from ? a.copy_from[r] : -1;
    const void* x = half ? a.v : a.k;
    const RowsPitch& pitch = half ? a.vp : a.kp;
    const int64_t from_x = r * pitch.row + h * pitch.head + d;
    float x0 = 0.f, x1 = 0.f;
    if (d < a.D) { x0 = value_at<TYPE>(x, from_x); x1 = value_at<TYPE>(x, from_x + 1); }
    if (slot < 0 || slot / a.block >= a.n_blocks) return;
    const int block = slot / a.block, at = slot & (a.block - 1), src = at > 0 && copy >= 0 && copy < a.n_blocks ? copy : block;
    const int64_t from = (int64_t)src * a.heads + h, to = (int64_t)block * a.heads + h, bytes = (int64_t)a.block * a.D;
    float* scales = half ? a.scale_v : a.scale_k;
    const float before = at > 0 ? scales[from] : 0.f;
    const float m = wave_max_f32(finite_size(finite_size(0.f, x0), x1));
    if (lane_id() == 0) amax[wave_id()] = m;
    __syncthreads();                                     // (and all have read the scales)
    const Earlier e = new_scale(before, fmaxf(amax[2 * half], amax[2 * half + 1]), src == block);
    if ((threadIdx.x & 127) == 0) scales[to] = e.scale;
    const uint32_t code = to_codes(x0 * e.inverse, x1 * e.inverse, 0.f, 0.f);
    if (half == 0) {
        uint8_t* codes = a.codes_k + to * bytes;
        if (at > 0 && !e.same) move_keys(a.codes_k + from * bytes, codes, at, a.block, a.D, e, threadIdx.x, 128);
        if (d < a.D) *reinterpret_cast<uint16_t*>(codes + ((int64_t)(d >> 4) * a.block + at) * 16 + (d & 15)) = (uint16_t)code;
    } else {
        uint8_t* codes = a.codes_v + to * bytes;
        const uint8_t* old = a.codes_v + from * bytes;
        // whole groups of 16 earlier tokens, then the group that the token belongs to (whose thread for value d it is)
        const float ratio = e.before * e.inverse;
        const int g = at >> 4;
        if (at > 0 && !e.same) {
            for (int i = threadIdx.x & 127; i < g * a.D; i += 128) {
                uint4 w = *reinterpret_cast<const uint4*>(old + (int64_t)i * 16);
                if (e.before != e.scale) w = make_uint4(scaled_codes(w.x, ratio), scaled_codes(w.y, ratio), scaled_codes(w.z, ratio), scaled_codes(w.w, ratio));
                *reinterpret_cast<uint4*>(codes + (int64_t)i * 16) = w;
            }
        }
        if (d < a.D) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int64_t line = ((int64_t)g * a.D + d + k) * 16;
                if ((at & 15) > 0 && !e.same) {
                    const uint4 o = *reinterpret_cast<const uint4*>(old + line), s = *reinterpret_cast<const uint4*>(codes + line);
                    const uint32_t ow[4] = {o.x, o.y, o.z, o.w}, sw[4] = {s.x, s.y, s.z, s.w};
                    uint32_t u[4];
#pragma unroll
                    for (int q = 0; q < 4; ++q) {        // bytes of earlier tokens
                        const int n = min(max((at & 15) - 4 * q, 0), 4);
                        const uint32_t is_old = n == 4 ? 0xffffffffu : (1u << (8 * n)) - 1u;
                        u[q] = ((e.before != e.scale ? scaled_codes(ow[q], ratio) : ow[q]) & is_old) | (sw[q] & ~is_old);
                    }
                    *reinterpret_cast<uint4*>(codes + line) = make_uint4(u[0], u[1], u[2], u[3]);
                }
                codes[line + (at & 15)] = (uint8_t)(code >> (8 * k));
            }
        }
    }
}

// grid = (R * per_row, heads), 256 threads.  Bound by how long a workgroup takes (values, their maximum, earlier codes, codes): 16 rows of
// up to 512 tokens, 8 heads of 64, fp32, 21 MB in 12 to 13 us (asked for twice, 19 MB of it come from memory, the rest from L2).
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
    const int eights = a.D >> 3;
    for (int i = threadIdx.x; i < n * eights; i += 256) {
        const int t = (int)((unsigned)i / (unsigned)eights), d = 8 * (i - t * eights);
        float x[8], y[8];
        load_values<TYPE>(a.k, k0 + t * a.kp.token + d, x);
        load_values<TYPE>(a.v, v0 + t * a.vp.token + d, y);
#pragma unroll
        for (int q = 0; q < 8; ++q) { mk = finite_size(mk, x[q]); mv = finite_size(mv, y[q]); }
    }
    mk = wave_max_f32(mk);
    mv = wave_max_f32(mv);
    if (lane_id() == 0) { amax[0][wave_id()] = mk; amax[1][wave_id()] = mv; }
    const int64_t from = (int64_t)src * a.heads + h, to = (int64_t)block * a.heads + h;
    const float before_k = at > 0 ? a.scale_k[from] : 0.f, before_v = at > 0 ? a.scale_v[from] : 0.f;
    __syncthreads();
    const Earlier ek = new_scale(before_k, fmaxf(fmaxf(amax[0][0], amax[0][1]), fmaxf(amax[0][2], amax[0][3])), src == block);
    const Earlier ev = new_scale(before_v, fmaxf(fmaxf(amax[1][0], amax[1][1]), fmaxf(amax[1][2], amax[1][3])), src == block);
    if (threadIdx.x == 0) { a.scale_k[to] = ek.scale; a.scale_v[to] = ev.scale; }
    const int64_t bytes = (int64_t)a.block * a.D;
    // keys: a line of 16 bytes is 16 values of a token
    if (at > 0 && !ek.same) move_keys(a.codes_k + from * bytes, a.codes_k + to * bytes, at, a.block, a.D, ek, threadIdx.x, 256);
    for (int i = threadIdx.x; i < n * eights; i += 256) {
        const int t = (int)((unsigned)i / (unsigned)eights), d = 8 * (i - t * eights);
        float x[8];
        load_values<TYPE>(a.k, k0 + t * a.kp.token + d, x);
#pragma unroll
        for (int q = 0; q < 8; ++q) x[q] *= ek.inverse;
        *reinterpret_cast<uint2*>(a.codes_k + to * bytes + ((int64_t)(d >> 4) * a.block + at + t) * 16 + (d & 15)) =
            make_uint2(to_codes(x[0], x[1], x[2], x[3]), to_codes(x[4], x[5], x[6], x[7]));
    }
    // values: a line of 16 bytes is a value of 16 tokens, some of them earlier ones, some new, some that stay
    for (int i = threadIdx.x; i < ((at + n + 15) >> 4) * a.D; i += 256) {
        const int g = i / a.D, d = i - g * a.D;
        const int64_t line = (int64_t)i * 16;
        const bool same = ev.same;
        if (same && 16 * g + 16 <= at) continue;
        const float ratio = ev.before * ev.inverse;
        const bool all_new = 16 * g >= at && 16 * g + 16 <= at + n;   // (nothing to keep)
        uint4 stay = make_uint4(0, 0, 0, 0);
        if (!all_new) stay = *reinterpret_cast<const uint4*>(a.codes_v + to * bytes + line);
        const uint4 old = at > 16 * g ? *reinterpret_cast<const uint4*>(a.codes_v + from * bytes + line) : stay;
        const uint32_t s[4] = {stay.x, stay.y, stay.z, stay.w}, o[4] = {old.x, old.y, old.z, old.w};
        uint32_t u[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint32_t kept = ev.before == ev.scale ? o[q] : scaled_codes(o[q], ratio);
            float x[4];
            uint32_t is_old = 0, is_new = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int t = 16 * g + 4 * q + j;
                x[j] = 0.f;
                if (t < at) is_old |= 0xffu << (8 * j);
                else if (t < at + n) {
                    is_new |= 0xffu << (8 * j);
                    x[j] = value_at<TYPE>(a.v, v0 + (t - at) * a.vp.token + d) * ev.inverse;
                }
            }
            u[q] = (kept & is_old) | (to_codes(x[0], x[1], x[2], x[3]) & is_new) | (s[q] & ~(is_old | is_new));
        }
        *reinterpret_cast<uint4*>(a.codes_v + to * bytes + line) = make_uint4(u[0], u[1], u[2], u[3]);
    }
}

}  // namespace lshbeam
