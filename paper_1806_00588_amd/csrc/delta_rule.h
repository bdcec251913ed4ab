// The gated delta rule (lsh_delta_rule).  For a row and a head, with the state H [Dk, Dv] and of token t the query q, key k, value v,
// a = e^decay, b = beta:
//   u = b (v - a H^T k),   H <- a H + k u^T,   out = scale H^T q
//
// k_delta_tokens: token after token.  The columns of H do not meet, so a workgroup has 64 of them (of a row and head), in registers from the first
// token to the last: a thread four columns and Dk / 16 neighbouring rows.  H^T k and H^T q of the state before the token are summed
// together (out = a H^T q + (q.k) u), so a token costs one exchange: across the 16 threads of a column.  A single token reads and writes
// the state, 8 Dk Dv bytes, for some 8 Dk Dv operations: memory bounds it.
#pragma once
#include "operands.h"

namespace lshbeam {

struct DeltaArgs {
    int S, B, T, heads, k_heads, Dk, Dv;
    float scale;
    const void* q;
    const void* k;
    const void* v;
    RowsPitch qp, kp, vp;
    const float* decay;        // [R, T, heads]
    const float* beta;
    const float* state_in;     // [R, heads, Dk, Dv] or null
    const int32_t* parents;    // [R] or null
    const int32_t* n_new;      // [R] or null
    float* state_out;
    void* out;
    RowsPitch op;
    int slices;                // of a head's columns
};

constexpr int kDeltaColumns = 64;   // of a workgroup
constexpr int kDeltaBlock = 8;      // tokens whose queries and keys are in LDS

__device__ __forceinline__ int delta_new(const DeltaArgs& a, int r) { return a.n_new ? min(max(a.n_new[r], 0), a.T) : a.T; }
// The row whose state row r begins with, -1: zeros.
__device__ __forceinline__ int delta_parent(const DeltaArgs& a, int r) {
    if (!a.state_in) return -1;
    if (!a.parents) return r;
    const int p = a.parents[r];
    return p >= 0 && p < a.B ? r / a.B * a.B + p : -1;
}

// NR: rows of a thread at most.
template <int TYPE, int NR>
__global__ void __launch_bounds__(256) k_delta_tokens(DeltaArgs a) {
    __shared__ float qk[2][kDeltaBlock][256];
    __shared__ f32x4 part[2][4][3][16];
    const int slice = blockIdx.x % (unsigned)a.slices, rh = blockIdx.x / (unsigned)a.slices, h = rh % a.heads, r = rh / a.heads;
    const int hk = h / (a.heads / a.k_heads);
    const int col = threadIdx.x & 15, rg = threadIdx.x >> 4, wave = wave_id();
    const int d = slice * kDeltaColumns + 4 * col, nr = a.Dk >> 4;
    const bool live = d < a.Dv;
    const int n = delta_new(a, r), parent = delta_parent(a, r);
    const int64_t size = (int64_t)a.Dk * a.Dv, first = (int64_t)rg * nr * a.Dv + d;
    f32x4 H[NR];
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        H[i] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (live && parent >= 0 && i < nr) H[i] = *reinterpret_cast<const f32x4*>(a.state_in + ((int64_t)parent * a.heads + h) * size + first + (int64_t)i * a.Dv);
    }
    for (int t0 = 0; t0 < n; t0 += kDeltaBlock) {
        const int here = min(kDeltaBlock, n - t0);
        __syncthreads();
        for (int i = threadIdx.x; i < 2 * here * a.Dk; i += 256) {
            const int which = i >= here * a.Dk, j = i - which * here * a.Dk, t = j / a.Dk, e = j - t * a.Dk;
            const RowsPitch& p = which ? a.kp : a.qp;
            qk[which][t][e] = value_at<TYPE>(which ? a.k : a.q, r * p.row + (t0 + t) * p.token + hk * p.head + e);
        }
        __syncthreads();
        for (int t = 0; t < here; ++t) {
            const int64_t at = ((int64_t)r * a.T + t0 + t) * a.heads + h;
            const float decay = expf(a.decay[at]), beta = a.beta[at];
            f32x4 v = {0.f, 0.f, 0.f, 0.f};
            if (live) {
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = value_at<TYPE>(a.v, r * a.vp.row + (t0 + t) * a.vp.token + h * a.vp.head + d + j);
            }
            f32x4 kh = {0.f, 0.f, 0.f, 0.f}, qh = kh;
            float both = 0.f;
#pragma unroll
            for (int i = 0; i < NR; ++i) {
                if (i >= nr) break;
                const float q = qk[0][t][rg * nr + i], k = qk[1][t][rg * nr + i];
                both = fmaf(q, k, both);
#pragma unroll
                for (int j = 0; j < 4; ++j) { kh[j] = fmaf(k, H[i][j], kh[j]); qh[j] = fmaf(q, H[i][j], qh[j]); }
            }
            // the four row groups of the wave, then the waves
#pragma unroll
            for (int off = 16; off < 64; off *= 2) {
#pragma unroll
                for (int j = 0; j < 4; ++j) { kh[j] += __shfl_xor(kh[j], off, kWave); qh[j] += __shfl_xor(qh[j], off, kWave); }
                both += __shfl_xor(both, off, kWave);
            }
            f32x4 (*to)[3][16] = part[t & 1];
            if (lane_id() < 16) { to[wave][0][col] = kh; to[wave][1][col] = qh; to[wave][2][col] = f32x4{both, 0.f, 0.f, 0.f}; }
            __syncthreads();
            kh = (to[0][0][col] + to[1][0][col]) + (to[2][0][col] + to[3][0][col]);
            f32x4 u;
#pragma unroll
            for (int j = 0; j < 4; ++j) u[j] = beta * (v[j] - decay * kh[j]);
            if (wave == 0 && rg == 0 && live) {
                qh = (to[0][1][col] + to[1][1][col]) + (to[2][1][col] + to[3][1][col]);
                both = (to[0][2][col][0] + to[1][2][col][0]) + (to[2][2][col][0] + to[3][2][col][0]);
                const int64_t o = r * a.op.row + (t0 + t) * a.op.token + h * a.op.head + d;
#pragma unroll
                for (int j = 0; j < 4; ++j) put_value<TYPE>(a.out, o + j, a.scale * (decay * qh[j] + both * u[j]));
            }
#pragma unroll
            for (int i = 0; i < NR; ++i) {
                if (i >= nr) break;
                const float k = qk[1][t][rg * nr + i];
#pragma unroll
                for (int j = 0; j < 4; ++j) H[i][j] = fmaf(k, u[j], decay * H[i][j]);
            }
        }
    }
    if (!live) return;
#pragma unroll
    for (int i = 0; i < NR; ++i)
        if (i < nr) *reinterpret_cast<f32x4*>(a.state_out + ((int64_t)r * a.heads + h) * size + first + (int64_t)i * a.Dv) = H[i];
}

}  // namespace lshbeam
