// Attention over a paged cache of 8-bit codes (lsh_cache_attention):
//   o[r, t, h] = sum_j p_j v_j,   p = softmax_j(scale * q[r, t, h] . k_j)   over the positions j of row r that token t sees.
#pragma once
#include "cache_write.h"

namespace lshbeam {

struct AttnArgs {
    int S, B, T, q_heads, heads, D;
    int n_blocks, block, width;
    int causal, window;
    float scale;
    const void* q;
    RowsPitch qp;
    const uint8_t* codes_k;
    const uint8_t* codes_v;
    const float* scale_k;
    const float* scale_v;
    const int32_t* tables;     // [R, width]
    const int32_t* lengths;    // [R]
    const int32_t* n_new;      // [R] or null
    const int32_t* shared;     // [S] or null
    void* out;
    RowsPitch op;
    float* lse;                // [R, T, q_heads] or null
};

// Positions lo .. hi - 1 that token t of a row of `len` tokens, `n` of them new, sees.
__device__ __forceinline__ void seen(const AttnArgs& a, int len, int n, int t, int* lo, int* hi) {
    *hi = a.causal ? max(0, len - n + t + 1) : len;
    *lo = a.window > 0 ? max(0, *hi - a.window) : 0;
}
__device__ __forceinline__ int row_length(const AttnArgs& a, int r) { return (int)min((int64_t)max(a.lengths[r], 0), (int64_t)a.width * a.block); }
__device__ __forceinline__ int row_new(const AttnArgs& a, int r) { return a.n_new ? min(max(a.n_new[r], 0), a.T) : a.T; }

template <int TYPE> __device__ __forceinline__ void put_value(void* p, int64_t i, float v) {
    if constexpr (TYPE == kTypeF32) static_cast<float*>(p)[i] = v;
    else if constexpr (TYPE == kTypeF16) static_cast<uint16_t*>(p)[i] = __half_as_ushort(__float2half_rn(v));
    else {
        const uint32_t u = __float_as_uint(v);   // nearest even; a NaN stays one
        static_cast<uint16_t*>(p)[i] = v != v ? (uint16_t)0x7fc0 : (uint16_t)((u + 0x7fffu + (u >> 16 & 1u)) >> 16);
    }
}
__device__ __forceinline__ float code_f32(uint8_t c) { return __builtin_amdgcn_cvt_f32_fp8((int)c, 0); }

// grid = (R * T, q_heads), four waves: every wave takes every fourth position, a lane four values of the head at most.
template <int TYPE>
__global__ void __launch_bounds__(256) k_attention(AttnArgs a) {
    __shared__ float ms[4], ls[4], os[4][256];
    const int r = blockIdx.x / a.T, t = blockIdx.x - r * a.T, hq = blockIdx.y, h = hq / (a.q_heads / a.heads);
    const int n = row_new(a, r);
    if (t >= n) return;
    int lo, hi;
    seen(a, row_length(a, r), n, t, &lo, &hi);
    float q[4], o[4], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int d = lane_id() + 64 * i;
        q[i] = d < a.D ? value_at<TYPE>(a.q, r * a.qp.row + t * a.qp.token + hq * a.qp.head + d) : 0.f;
        o[i] = 0.f;
    }
    for (int j = lo + wave_id(); j < hi; j += 4) {
        const int32_t id = a.tables[(int64_t)r * a.width + j / a.block];
        if (id < 0 || id >= a.n_blocks) continue;
        const int at = j % a.block;
        const int64_t head = (int64_t)id * a.heads + h, base = head * a.block * a.D;
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int d = lane_id() + 64 * i;
            if (d < a.D) s += q[i] * code_f32(a.codes_k[base + ((int64_t)(d >> 4) * a.block + at) * 16 + (d & 15)]);
        }
        s = wave_sum_f32(s) * (a.scale_k[head] * a.scale);
        const float now = fmaxf(m, s), was = m > -INFINITY ? expf(m - now) : 0.f, p = expf(s - now);
        l = l * was + p;
        m = now;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int d = lane_id() + 64 * i;
            if (d < a.D) o[i] = o[i] * was + p * (code_f32(a.codes_v[base + ((int64_t)(at >> 4) * a.D + d) * 16 + (at & 15)]) * a.scale_v[head]);
        }
    }
    const int wv = wave_id();
    if (lane_id() == 0) { ms[wv] = m; ls[wv] = l; }
#pragma unroll
    for (int i = 0; i < 4; ++i) os[wv][lane_id() + 64 * i] = o[i];
    __syncthreads();
    const float top = fmaxf(fmaxf(ms[0], ms[1]), fmaxf(ms[2], ms[3]));
    float f[4], sum = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) { f[w] = ms[w] > -INFINITY ? expf(ms[w] - top) : 0.f; sum += ls[w] * f[w]; }
    const int d = threadIdx.x;
    if (d < a.D) {
        const float v = os[0][d] * f[0] + os[1][d] * f[1] + os[2][d] * f[2] + os[3][d] * f[3];
        put_value<TYPE>(a.out, r * a.op.row + t * a.op.token + hq * a.op.head + d, sum > 0.f || sum != sum ? v / sum : 0.f);
    }
    if (d == 0 && a.lse) a.lse[((int64_t)r * a.T + t) * a.q_heads + hq] = sum > 0.f || sum != sum ? top + logf(sum) : -INFINITY;
}

}  // namespace lshbeam
