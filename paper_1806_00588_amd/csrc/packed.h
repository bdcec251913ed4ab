// Weights of 4 bits (lsh_packed_quantize, lsh_packed_values): their layout, made and read back.
//
// A weight is (code - zero) * scale.  A tile is 16 outputs, a part 128 inputs; the 1 KB of a tile's part lie so that lane l = 16 c + n
// of a wave, loading 16 bytes, has the four operand words of output n that v_mfma_f32_16x16x32 asks of that lane: word w holds inputs
// 32 w + 8 c .. + 7.  The bytes of a word have input i in the lower and i + 4 in the upper four bits, because a byte 0 .. 15 read
// as an e4m3 number is its value times 2^-9, subnormals included: four conversions give the eight codes as bf16 or fp16, exactly.
// The scales of an output's groups in a part lie side by side, one load for all of them.
#pragma once
#include "operands.h"

namespace lshbeam {

constexpr int kPackOutputs = 16, kPackInputs = 128, kPackBytes = 1024;   // of a tile's part

struct PackedRef {
    uint8_t* codes;
    uint16_t* scales;          // [tiles, parts, 16, 128 / group]
    uint8_t* zeros;            // the same, or null
};

template <bool F16> __device__ __forceinline__ float scale_f32(uint32_t bits) {
    return F16 ? __half2float(__ushort_as_half((uint16_t)bits)) : __uint_as_float(bits << 16);
}

struct QuantArgs {
    int N, K, parts, shift;    // log2 of the group
    int64_t units;             // tiles * parts
    const void* w;             // [N, K] (values: the output)
    int64_t ld;
    PackedRef to;
};

// w / s to the nearest whole number, ties to even, of the exact quotient.  From inv, 1 / s rounded, it errs only next to a half;
// there s * (r +- 1/2), 16 bits or fewer, is exact and settles it.
__device__ __forceinline__ float whole_near(float w, float s, float r) {
    const float up = s * (r + 0.5f), down = s * (r - 0.5f);
    const bool odd = ((int)r & 1) != 0;
    if (w > up || (w == up && odd)) r += 1.f;
    else if (w < down || (w == down && odd)) r -= 1.f;
    return r;
}

// A wave for a tile's part: lane 4 n + c has the c-th eights of output n (four neighbouring lanes 32 neighbouring inputs, a group or
// a part of one).  The group's largest and smallest go round its lanes, everything else is a lane's own.  Bound by memory: it reads
// each weight and writes each code once.
template <int TYPE, bool F16, bool ZEROS>
__global__ void __launch_bounds__(256) k_packed_quantize(QuantArgs a) {
    const int64_t unit = (int64_t)blockIdx.x * 4 + wave_id();
    if (unit >= a.units) return;
    const int64_t tile = unit / a.parts;
    const int part = (int)(unit - tile * a.parts), n = lane_id() >> 2, c = lane_id() & 3;
    const int64_t row = tile * kPackOutputs + n;
    float x[4][8];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const int k = part * kPackInputs + 32 * w + 8 * c;
        if (row < a.N && k + 8 <= a.K) load_values<TYPE>(a.w, row * a.ld + k, x[w]);
        else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[w][i] = row < a.N && k + i < a.K ? value_at<TYPE>(a.w, row * a.ld + k + i) : 0.f;
        }
    }
    // smallest (with zeros) and largest
    float lo[4], hi[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        float none = 0.f;                        // 0 times each: no 0 if one of them is not finite
        lo[w] = hi[w] = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            lo[w] = ZEROS ? fminf(lo[w], x[w][i]) : 0.f;
            hi[w] = fmaxf(hi[w], ZEROS ? x[w][i] : fabsf(x[w][i]));
            none = fmaf(x[w][i], 0.f, none);
        }
        if (none != 0.f) hi[w] = INFINITY;       // (says the same to the other lanes)
        hi[w] = fmaxf(hi[w], dpp_f32<0xB1>(hi[w]));
        hi[w] = fmaxf(hi[w], dpp_f32<0x4E>(hi[w]));
        if (ZEROS) {
            lo[w] = fminf(lo[w], dpp_f32<0xB1>(lo[w]));
            lo[w] = fminf(lo[w], dpp_f32<0x4E>(lo[w]));
        }
    }
#pragma unroll
    for (int step = 1; step < 4; step *= 2) {    // groups of 64, of 128
        if (32 * step >= 1 << a.shift) break;
        float h[4], l[4];
#pragma unroll
        for (int w = 0; w < 4; ++w) { h[w] = fmaxf(hi[w], hi[w ^ step]); l[w] = fminf(lo[w], lo[w ^ step]); }
#pragma unroll
        for (int w = 0; w < 4; ++w) { hi[w] = h[w]; lo[w] = l[w]; }
    }
    const int each = kPackInputs >> a.shift;
    const bool edge = (tile + 1) * kPackOutputs > a.N || (part + 1) * kPackInputs > a.K;
    uint32_t words[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const bool nan = !(hi[w] < INFINITY);
        const float wide = nan ? NAN : ZEROS ? (float)(((double)hi[w] - (double)lo[w]) / 15.0) : hi[w] / 7.f;
        uint16_t bits;
        if constexpr (F16) bits = __half_as_ushort(__float2half_rn(wide));
        else put_value<kTypeBf16>(&bits, 0, wide);
        const float s = scale_f32<F16>(bits);
        // (tiny scales, whose inverse is no number of 32 bits, a power of two larger)
        const float f = s < 0x1p-100f ? 0x1p60f : 1.f, inv = s > 0.f ? 1.f / (s * f) : 0.f;
        float zero = 8.f;
        if constexpr (ZEROS) {
            zero = rintf(-lo[w] * f * inv);
            if (s > 0.f) zero = whole_near(-lo[w], s, zero);
            zero = fminf(fmaxf(zero, 0.f), 15.f);
        }
        float q[8], off = 0.f;
        if (f != 1.f) {
#pragma unroll
            for (int i = 0; i < 8; ++i) q[i] = x[w][i] * f * inv;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) q[i] = x[w][i] * inv;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float whole = rintf(q[i]);
            off = fmaxf(off, fabsf(q[i] - whole));
            q[i] = whole;
        }
        if (off > 0.4999f && s > 0.f) {
#pragma unroll
            for (int i = 0; i < 8; ++i) q[i] = whole_near(x[w][i], s, q[i]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = __builtin_amdgcn_fmed3f(q[i] + zero, 0.f, 15.f);
        if (edge || nan) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (nan || row >= a.N || part * kPackInputs + 32 * w + 8 * c + i >= a.K) q[i] = 0.f;
        }
        uint32_t word = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) word = __builtin_amdgcn_cvt_pk_u8_f32(fmaf(q[i + 4], 16.f, q[i]), i, word);
        words[w] = word;
        const int per = 1 << (a.shift - 5);      // words of a group
        if (c == 0 && (w & (per - 1)) == 0) {
            const bool none = row >= a.N || part * kPackInputs + 32 * w >= a.K;
            const int64_t to = (unit * kPackOutputs + n) * each + w / per;
            a.to.scales[to] = none ? (uint16_t)0 : bits;
            if (ZEROS) a.to.zeros[to] = none || nan ? (uint8_t)0 : (uint8_t)zero;
        }
    }
    *reinterpret_cast<uint4*>(a.to.codes + unit * kPackBytes + (16 * c + n) * 16) = make_uint4(words[0], words[1], words[2], words[3]);
}

// The same way back: lane 4 n + c writes the c-th eights of output n.
template <int TYPE, bool F16>
__global__ void __launch_bounds__(256) k_packed_values(QuantArgs a) {
    const int64_t unit = (int64_t)blockIdx.x * 4 + wave_id();
    if (unit >= a.units) return;
    const int64_t tile = unit / a.parts;
    const int part = (int)(unit - tile * a.parts), n = lane_id() >> 2, c = lane_id() & 3;
    const int64_t row = tile * kPackOutputs + n;
    if (row >= a.N) return;
    const int each = kPackInputs >> a.shift;
    const uint4 v = *reinterpret_cast<const uint4*>(a.to.codes + unit * kPackBytes + (16 * c + n) * 16);
    const uint32_t words[4] = {v.x, v.y, v.z, v.w};
    const int64_t from = (unit * kPackOutputs + n) * each;
    void* out = const_cast<void*>(a.w);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const int k = part * kPackInputs + 32 * w + 8 * c, g = w >> (a.shift - 5);
        if (k >= a.K) break;
        const float s = scale_f32<F16>(a.to.scales[from + g]);
        const float zero = a.to.zeros ? (float)a.to.zeros[from + g] : 8.f;
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = ((float)(words[w] >> (8 * (i & 3) + 4 * (i >> 2)) & 15u) - zero) * s;
        if (k + 8 <= a.K) {
            using T = typename WordOf<TYPE>::type;
            T t[8];
            if constexpr (TYPE == kTypeBf16) {   // (nearest even, pairs at once)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const f32x2 v = {x[2 * i], x[2 * i + 1]};
                    const uint32_t two = __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
                    t[2 * i] = (T)(two & 0xffffu);
                    t[2 * i + 1] = (T)(two >> 16);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) put_value<TYPE>(t, i, x[i]);
            }
            T* to = static_cast<T*>(out) + row * a.ld + k;
#pragma unroll
            for (int h = 0; h < (TYPE == kTypeF32 ? 2 : 1); ++h) {
                Chunk16U<T> piece;
                __builtin_memcpy(&piece, t + 4 * h, 16);
                *reinterpret_cast<Chunk16U<T>*>(to + 4 * h) = piece;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (k + i < a.K) put_value<TYPE>(out, row * a.ld + k + i, x[i]);
        }
    }
}

}  // namespace lshbeam
