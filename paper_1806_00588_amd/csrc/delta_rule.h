// The gated delta rule (lsh_delta_rule).  For a row and a head, with the state H [Dk, Dv] and of token t the query q, key k, value v,
// a = e^decay, b = beta:
//   u = b (v - a H^T k),   H <- a H + k u^T,   out = scale H^T q
//
// k_delta_tokens: token after token.  The columns of H do not meet, so a workgroup has 64 of them (of a row and head), in registers from the first
// token to the last: a thread four columns and a sixteenth of the rows.  H^T k and H^T q of the state before the token are summed
// together (out = a H^T q + (q.k) u), so a token costs one exchange, across the 16 threads of a column.  A single token reads and writes
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

// NR: rows of a thread (some of them behind the last); ONE: a single token, whose queries, keys and values are asked for before the state.
template <int TYPE, int NR, bool ONE>
__global__ void __launch_bounds__(256, 4) k_delta_tokens(DeltaArgs a) {
    using Word = typename WordOf<TYPE>::type;
    __shared__ __align__(16) float qk[kDeltaBlock][2][16 * NR];
    __shared__ __align__(16) float vs[kDeltaBlock][kDeltaColumns];
    __shared__ float gate[kDeltaBlock][2];                 // e^decay, beta
    __shared__ f32x4 part[2][4][3][16];
    const int slice = blockIdx.x % (unsigned)a.slices, rh = blockIdx.x / (unsigned)a.slices, h = rh % a.heads, r = rh / a.heads;
    const int hk = h / (a.heads / a.k_heads);
    const int col = threadIdx.x & 15, rg = threadIdx.x >> 4, wave = wave_id(), d = slice * kDeltaColumns + 4 * col;
    const bool live = d < a.Dv;
    const int n = delta_new(a, r), parent = delta_parent(a, r);
    const int64_t q0 = r * a.qp.row + hk * a.qp.head, k0 = r * a.kp.row + hk * a.kp.head, v0 = r * a.vp.row + h * a.vp.head + slice * kDeltaColumns;
    const int64_t g0 = (int64_t)r * a.T * a.heads + h;
    constexpr int kQk = (2 * 16 * NR + 255) / 256;         // of a thread
    // element i of the 2 * 16 NR of a token's query and key, 0 behind their last
    auto qk_at = [&](int t, int i) {
        const int which = i >= 16 * NR, e = i - which * (16 * NR);
        return e < a.Dk && i < 2 * 16 * NR ? static_cast<const Word*>(which ? a.k : a.q)[(which ? k0 + t * a.kp.token : q0 + t * a.qp.token) + e] : (Word)0;
    };
    auto v_at = [&](int t, int i) { return slice * kDeltaColumns + i < a.Dv ? static_cast<const Word*>(a.v)[v0 + t * a.vp.token + i] : (Word)0; };

    Word first_qk[kQk], first_v = (Word)0;
    float first_gate = 0.f;
    if (ONE && n > 0) {
#pragma unroll
        for (int i = 0; i < kQk; ++i) first_qk[i] = qk_at(0, threadIdx.x + 256 * i);
        if (threadIdx.x < kDeltaColumns) first_v = v_at(0, threadIdx.x);
        if (threadIdx.x < 2) first_gate = threadIdx.x ? a.beta[g0] : a.decay[g0];
    }
    f32x4 H[NR];
    const float* from = a.state_in + (parent < 0 ? 0 : ((int64_t)parent * a.heads + h) * a.Dk * a.Dv) + (int64_t)rg * NR * a.Dv + d;
#pragma unroll
    for (int i = 0; i < NR; ++i)
        H[i] = live && parent >= 0 && rg * NR + i < a.Dk ? *reinterpret_cast<const f32x4*>(from + (int64_t)i * a.Dv) : f32x4{0.f, 0.f, 0.f, 0.f};
    for (int t0 = 0; t0 < n; t0 += kDeltaBlock) {
        const int here = ONE ? 1 : min(kDeltaBlock, n - t0);
        if constexpr (ONE) {
#pragma unroll
            for (int i = 0; i < kQk; ++i) {
                const int at = threadIdx.x + 256 * i;
                if (at < 2 * 16 * NR) (&qk[0][0][0])[at] = word_f32<TYPE>(first_qk[i]);
            }
            if (threadIdx.x < kDeltaColumns) vs[0][threadIdx.x] = word_f32<TYPE>(first_v);
            if (threadIdx.x < 2) gate[0][threadIdx.x] = threadIdx.x ? first_gate : expf(first_gate);
        } else {
            __syncthreads();
            for (int i = threadIdx.x; i < here * 2 * 16 * NR; i += 256) {
                const int t = i / (2 * 16 * NR), e = i - t * (2 * 16 * NR);
                (&qk[t][0][0])[e] = word_f32<TYPE>(qk_at(t0 + t, e));
            }
            for (int i = threadIdx.x; i < here * kDeltaColumns; i += 256) vs[i / kDeltaColumns][i % kDeltaColumns] = word_f32<TYPE>(v_at(t0 + i / kDeltaColumns, i % kDeltaColumns));
            if (threadIdx.x < 2 * here) {
                const int t = threadIdx.x >> 1;
                const int64_t at = g0 + (int64_t)(t0 + t) * a.heads;
                gate[t][threadIdx.x & 1] = threadIdx.x & 1 ? a.beta[at] : expf(a.decay[at]);
            }
        }
        lds_barrier();
        for (int t = 0; t < here; ++t) {
            const float decay = gate[t][0], beta = gate[t][1];
            f32x4 kh = {0.f, 0.f, 0.f, 0.f}, qh = kh;
            float both = 0.f, k[NR];
#pragma unroll
            for (int i = 0; i < NR; ++i) {
                const float q = qk[t][0][rg * NR + i];
                k[i] = qk[t][1][rg * NR + i];
                both = fmaf(q, k[i], both);
#pragma unroll
                for (int j = 0; j < 4; ++j) { kh[j] = fmaf(k[i], H[i][j], kh[j]); qh[j] = fmaf(q, H[i][j], qh[j]); }
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
            lds_barrier();
            kh = (to[0][0][col] + to[1][0][col]) + (to[2][0][col] + to[3][0][col]);
            const f32x4 v = *reinterpret_cast<const f32x4*>(&vs[t][4 * col]);
            f32x4 u;
#pragma unroll
            for (int j = 0; j < 4; ++j) u[j] = beta * (v[j] - decay * kh[j]);
#pragma unroll
            for (int i = 0; i < NR; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) H[i][j] = fmaf(k[i], u[j], decay * H[i][j]);
            if (rg == 0 && live) {
                qh = (to[0][1][col] + to[1][1][col]) + (to[2][1][col] + to[3][1][col]);
                both = (to[0][2][col][0] + to[1][2][col][0]) + (to[2][2][col][0] + to[3][2][col][0]);
                const int64_t o = r * a.op.row + (t0 + t) * a.op.token + h * a.op.head + d;
#pragma unroll
                for (int j = 0; j < 4; ++j) put_value<TYPE>(a.out, o + j, a.scale * (decay * qh[j] + both * u[j]));
            }
        }
        if constexpr (ONE) break;
    }
    if (!live) return;
    float* to = a.state_out + ((int64_t)r * a.heads + h) * a.Dk * a.Dv + (int64_t)rg * NR * a.Dv + d;
#pragma unroll
    for (int i = 0; i < NR; ++i)
        if (rg * NR + i < a.Dk) *reinterpret_cast<f32x4*>(to + (int64_t)i * a.Dv) = H[i];
}

}  // namespace lshbeam
