// The gated delta rule over many tokens, 64 at a time.  In a chunk, with c_i the sum of the decays of its tokens up to i, S the state before it and
// e_i = e^(c_i):
//   (1 + L) U = diag(b) (V - e K S),     L_ij = b_i e^(c_i - c_j) k_i.k_j  for j < i
//   out = scale (e Q S + A U),           A_ij = e^(c_i - c_j) q_i.k_j      for j <= i
//   S <- e^(c_last) S + K^T (e^(c_last - c_j) u_j)_j
//
// What does not depend on the state -- T = (1 + L)^-1 diag(b), A, and K, Q, K^T, V in the order of the matrix operands -- is made for all chunks at once
// by k_delta_prepare and goes through the workspace; k_delta_chain goes through a row's chunks in order.  The state's columns do not meet: a wave
// has 16 of them in registers, four waves share what comes through LDS.
//
// v_mfma_f32_16x16x32_bf16 everywhere, numbers of 32 bits as three planes of bf16 that add up to them (keys of 16 bits: one plane of bf16, two for
// fp16), with the products of planes down to 2^-16 of the first, so that what is left out is 2^-24 of a product; of results of 16 bits
// down to 2^-8, 2^-16 left out, a sixteenth of their own rounding at least.  A result D of an instruction has rows 4 c + i in lane (n, c), an
// operand rows 8 c + j: rows of the K, Q and T operands are in the order row_of below, so that two results' registers are the next
// product's operand as they are, and nothing is exchanged between lanes.
#pragma once
#include "delta_rule.h"

namespace lshbeam {

constexpr int kChunk = 64;            // tokens
constexpr int kStageBlocks = 8;       // operands of 1 KB that the waves of k_delta_chain wait for together

// Row of row m of tile t: of two tiles, lane c's 4 + 4 rows are neighbours.
__host__ __device__ constexpr int row_of(int t, int m) { return 32 * (t >> 1) + 8 * (m >> 2) + 4 * (t & 1) + (m & 3); }
__device__ __forceinline__ int tile_of_row(int r) { return 2 * (r >> 5) + (r >> 2 & 1); }
__device__ __forceinline__ int place_of_row(int r) { return 4 * (r >> 3 & 3) + (r & 3); }

// Operands of a chunk and head in the workspace, NK = ceil(k_dim / 32):
//   for each 32 of k_dim: K and Q [4 tiles of tokens][planes]; then e and e^(c_last - c_j) [2][64] fp32; T [6][3], A [6][its planes]; K^T [2][2 NK tiles][planes]
// in blocks of 1 KB, and V [64 columns at a time][parts of two blocks][4 tiles of columns][2].  k_delta_chain takes them in this order, V behind K and Q.  Of T and A those (tile of rows, 32 columns) that are not zero: (0, 0), (1, 0),
// (2, 0), (2, 1), (3, 0), (3, 1).
template <int TYPE, int NK> struct ChunkPlan {
    static constexpr int P = TYPE == kTypeBf16 ? 1 : TYPE == kTypeF16 ? 2 : 3;    // planes of K and Q
    static constexpr int PA = TYPE == kTypeF32 ? 3 : 2;                           // of A, and of what it meets
    static constexpr int kScalars = NK * 8 * P, kT = kScalars + 1, kA = kT + 18, kKt = kA + 6 * PA, kBlocks = kKt + 4 * NK * P;
    static constexpr int kStages = (kBlocks + kStageBlocks - 1) / kStageBlocks;   // without V's
    static constexpr int kVStages = TYPE == kTypeF32 ? 2 : 1;                     // V of 64 columns
    static constexpr int kBeforeV = NK * P;                                       // stages before V's
    static_assert(kScalars == kBeforeV * kStageBlocks && kStageBlocks == 8, "V's stages come between two others");
    static constexpr size_t bytes(int Dv) { return ((size_t)kStages + (Dv + 63) / 64 * kVStages) * kStageBlocks * 1024; }
};
__host__ __device__ constexpr int block_of(int t, int s) { return t < 2 ? t : 2 * t - 2 + s; }

struct ChunkArgs {
    DeltaArgs d;
    char* room;                // workspace: [pairs][chunks of the segment] of pair_bytes
    size_t bytes;              // of a chunk
    int64_t pair0;             // first pair of a row and a head of the launch
    int chunk0, chunks;        // the segment
    bool first;                // the state comes from the parent, else from state_out
};

__device__ __forceinline__ f32x4 mfma_bf16(uint4 a, uint4 b, f32x4 acc) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
}
// Products of planes i of a and j of b with i + j < ORDER, the smallest first.
template <int ORDER, int PA, int PB> __device__ __forceinline__ f32x4 mfma_planes(const uint4 (&a)[PA], const uint4 (&b)[PB], f32x4 acc) {
#pragma unroll
    for (int sum = ORDER - 1; sum >= 0; --sum)
#pragma unroll
        for (int i = 0; i < PA; ++i)
            if (sum - i >= 0 && sum - i < PB) acc = mfma_bf16(a[i], b[sum - i], acc);
    return acc;
}

constexpr int kMatrixPitch = 68;   // floats
// acc + a b of 16 x 16 each in LDS, all 32 bits.
__device__ __forceinline__ f32x4 mfma_f32(const float* a, const float* b, f32x4 acc) {
    const int ln = lane_id();
#pragma unroll
    for (int k = 0; k < 4; ++k)
        acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a[(ln & 15) * kMatrixPitch + 4 * k + (ln >> 4)], b[(4 * k + (ln >> 4)) * kMatrixPitch + (ln & 15)], acc, 0, 0, 0);
    return acc;
}
__device__ __forceinline__ void put_tile(float* to, f32x4 v) {
    const int ln = lane_id();
#pragma unroll
    for (int i = 0; i < 4; ++i) to[(4 * (ln >> 4) + i) * kMatrixPitch + (ln & 15)] = v[i];
}

template <int TYPE, int NK> constexpr int kPrepareLds = ChunkPlan<TYPE, NK>::P * 4 * NK * 1024 + (2 * 64 * kMatrixPitch + 4 * 64) * 4;

// A workgroup of four waves for a chunk of a row and head.
template <int TYPE, int NK>
__global__ void __launch_bounds__(256) k_delta_prepare(ChunkArgs ca) {
    using Plan = ChunkPlan<TYPE, NK>;
    constexpr int P = Plan::P;
    extern __shared__ __align__(16) char lds[];
    const DeltaArgs& a = ca.d;
    float* L = reinterpret_cast<float*>(lds + P * 4 * NK * 1024);
    float* T = L + 64 * kMatrixPitch;
    float* chi = T + 64 * kMatrixPitch;
    float *clo = chi + 64, *beta = clo + 64;
    const int64_t pair = ca.pair0 + blockIdx.x / (unsigned)ca.chunks;
    const int at = blockIdx.x % (unsigned)ca.chunks;
    const int r = (int)(pair / a.heads), h = (int)(pair - (int64_t)r * a.heads), hk = h / (a.heads / a.k_heads);
    const int t0 = (ca.chunk0 + at) * kChunk, n = min(kChunk, delta_new(a, r) - t0);
    if (n <= 0) return;
    char* to = ca.room + (size_t)blockIdx.x * ca.bytes;
    const int wave = __builtin_amdgcn_readfirstlane(wave_id()), ln = lane_id(), c = ln >> 4, m = ln & 15;

    // the decays' sums, in 64 bits, kept as two numbers of 32
    if (wave == 0) {
        const int64_t i = ((int64_t)r * a.T + t0 + ln) * a.heads + h;
        const float g = ln < n ? a.decay[i] : 0.f;
        double sum = g < -1e4f ? -1e4 : (double)g;      // (e^-infinity and e^-10000 are both 0; infinities have no differences)
#pragma unroll
        for (int off = 1; off < 64; off *= 2) {
            const double other = __shfl_up(sum, off, kWave);
            if (ln >= off) sum += other;
        }
        const double last = __shfl(sum, 63, kWave);
        chi[ln] = (float)sum;
        clo[ln] = (float)(sum - (double)(float)sum);
        beta[ln] = ln < n ? a.beta[i] : 0.f;
        float* scalars = reinterpret_cast<float*>(to + Plan::kScalars * 1024);
        scalars[ln] = (float)exp(sum);
        scalars[64 + ln] = (float)exp(last - sum);
    }
    // keys: planes as operands
    for (int u = threadIdx.x; u < kChunk * NK * 4; u += 256) {
        const int piece = u % (NK * 4), t = u / (NK * 4);
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = 0.f;
        if (t < n && 8 * piece < a.Dk) load_values<TYPE>(a.k, r * a.kp.row + (int64_t)(t0 + t) * a.kp.token + hk * a.kp.head + 8 * piece, x);
        uint4 op[P];
        planes_of<P>(x, op);
#pragma unroll
        for (int p = 0; p < P; ++p)
            *reinterpret_cast<uint4*>(lds + (((p * 4 + tile_of_row(t)) * NK + (piece >> 2)) * 64 + 16 * (piece & 3) + place_of_row(t)) * 16) = op[p];
    }
    for (int i = threadIdx.x; i < 64 * kMatrixPitch; i += 256) { L[i] = 0.f; T[i] = 0.f; }
    __syncthreads();

    auto key = [&](int p, int t, int s) { return *reinterpret_cast<const uint4*>(lds + (((p * 4 + t) * NK + s) * 64 + ln) * 16); };
    // a wave for a tile of rows: K K^T, and Q K^T with its own tile of Q
    f32x4 kk[4], qk[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) kk[j] = qk[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int tiles = 2 * (wave >> 1) + 2;
    for (int s = 0; s < NK; ++s) {
        float x[8];
        const int t = row_of(wave, m), d = 32 * s + 8 * c;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = 0.f;
        if (t < n && d < a.Dk) load_values<TYPE>(a.q, r * a.qp.row + (int64_t)(t0 + t) * a.qp.token + hk * a.qp.head + d, x);
        uint4 q[P], k[P];
        planes_of<P>(x, q);
#pragma unroll
        for (int p = 0; p < P; ++p) {
            k[p] = key(p, wave, s);
            char* block = to + (size_t)(s * 8 * P + wave * P + p) * 1024 + 16 * ln;
            *reinterpret_cast<uint4*>(block) = k[p];
            *reinterpret_cast<uint4*>(block + 4 * P * 1024) = q[p];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (j >= tiles) break;
            uint4 other[P];
#pragma unroll
            for (int p = 0; p < P; ++p) other[p] = key(p, j, s);
            kk[j] = mfma_planes<3>(k, other, kk[j]);
            qk[j] = mfma_planes<3>(q, other, qk[j]);
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (j >= tiles) break;
        const int col = row_of(j, m);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = row_of(wave, 4 * c + i);
            const float e = row >= col ? expf((chi[row] - chi[col]) + (clo[row] - clo[col])) : 0.f;
            if (row > col) L[row * kMatrixPitch + col] = beta[row] * (e * kk[j][i]);
            qk[j][i] = row >= col ? e * qk[j][i] : 0.f;
        }
    }
    // the keys' other way round: 8 tokens of one of k_dim
    for (int b = wave; b < 4 * NK * P; b += 4) {
        const int p = b % P, t = b / P % (2 * NK), s = b / (P * 2 * NK);
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t v = *reinterpret_cast<const uint16_t*>(lds + (((p * 4 + 2 * s + (j >> 2)) * NK + (t >> 1)) * 64 + 16 * (m >> 2) + 4 * c + (j & 3)) * 16 + 2 * (4 * (t & 1) + (m & 3)));
            if (j & 1) w[j >> 1] |= v << 16;
            else w[j >> 1] = v;
        }
        *reinterpret_cast<uint4*>(to + (size_t)(Plan::kKt + b) * 1024 + 16 * ln) = make_uint4(w[0], w[1], w[2], w[3]);
    }
    // values: 16-bit as they are, eight tokens of a column; fp32 four
    const int groups = (a.Dv + 63) / 64;
    char* values = to + (size_t)Plan::kStages * kStageBlocks * 1024;
    for (int b = wave; b < groups * Plan::kVStages * kStageBlocks; b += 4) {
        const int part = b / kStageBlocks % Plan::kVStages * 2 + (b & 1), tile = b / (kStageBlocks * Plan::kVStages) * 4 + (b >> 1 & 3);
        const int col = 16 * tile + m;
        if (16 * tile >= a.Dv) continue;
        const int64_t from = r * a.vp.row + (int64_t)t0 * a.vp.token + h * a.vp.head + col;
        uint32_t w[4];
        if constexpr (TYPE == kTypeF32) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int t = row_of(part, 4 * c + i);
                w[i] = t < n ? __float_as_uint(value_at<TYPE>(a.v, from + t * a.vp.token)) : 0u;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int t = 32 * part + 8 * c + i;
                const uint32_t v = t < n ? (uint32_t)static_cast<const uint16_t*>(a.v)[from + t * a.vp.token] : 0u;
                if (i & 1) w[i >> 1] |= v << 16;
                else w[i >> 1] = v;
            }
        }
        *reinterpret_cast<uint4*>(values + (size_t)b * 1024 + 16 * ln) = make_uint4(w[0], w[1], w[2], w[3]);
    }
    __syncthreads();

    // (1 + L)^-1: blocks of 16 on the diagonal by substitution, a lane a column; blocks below them by X21 = -X22 L21 X11, twice
    if (wave == 0) {
        const float* block = L + 16 * c * kMatrixPitch + 16 * c;
        float x[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float v = i == m ? 1.f : 0.f;
#pragma unroll
            for (int j = 0; j < i; ++j) v = fmaf(-block[i * kMatrixPitch + j], x[j], v);
            x[i] = v;
            T[(16 * c + i) * kMatrixPitch + 16 * c + m] = v;
        }
    }
    __syncthreads();
    const f32x4 none = {0.f, 0.f, 0.f, 0.f};
    if (wave < 2) {
        const int at32 = 32 * wave * kMatrixPitch + 32 * wave, below = at32 + 16 * kMatrixPitch;
        put_tile(L + below, mfma_f32(L + below, T + at32, none));
        put_tile(T + below, -mfma_f32(T + below + 16, L + below, none));
    }
    __syncthreads();
    const int ti = wave >> 1, tj = wave & 1, mine = (32 + 16 * ti) * kMatrixPitch + 16 * tj;
    f32x4 part = mfma_f32(L + (32 + 16 * ti) * kMatrixPitch, T + 16 * tj, none);
    part = mfma_f32(L + (32 + 16 * ti) * kMatrixPitch + 16, T + 16 * kMatrixPitch + 16 * tj, part);
    __syncthreads();
    put_tile(L + mine, part);
    __syncthreads();
    part = mfma_f32(T + (32 + 16 * ti) * kMatrixPitch + 32, L + 32 * kMatrixPitch + 16 * tj, none);
    part = mfma_f32(T + (32 + 16 * ti) * kMatrixPitch + 48, L + 48 * kMatrixPitch + 16 * tj, part);
    put_tile(T + mine, -part);
    __syncthreads();
    // T and A as operands
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (j >= tiles) break;
#pragma unroll
        for (int i = 0; i < 4; ++i) L[row_of(wave, 4 * c + i) * kMatrixPitch + row_of(j, m)] = qk[j][i];
    }
    __syncthreads();
    for (int s = 0; s <= wave >> 1; ++s) {
        const int b = block_of(wave, s), from = row_of(wave, m) * kMatrixPitch + 32 * s + 8 * c;
        float x[8];
        uint4 tp[3], ap[Plan::PA];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = T[from + i] * beta[32 * s + 8 * c + i];
        planes_of<3>(x, tp);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = L[from + i];
        planes_of<Plan::PA>(x, ap);
#pragma unroll
        for (int p = 0; p < 3; ++p) *reinterpret_cast<uint4*>(to + (size_t)(Plan::kT + 3 * b + p) * 1024 + 16 * ln) = tp[p];
#pragma unroll
        for (int p = 0; p < Plan::PA; ++p) *reinterpret_cast<uint4*>(to + (size_t)(Plan::kA + Plan::PA * b + p) * 1024 + 16 * ln) = ap[p];
    }
}

// Stages of k_delta_chain that are in LDS or on their way.
constexpr int kRing = 8;
constexpr int kChainLds = kRing * kStageBlocks * 1024;

// A workgroup of four waves for 64 columns of a row's and head's state.
template <int TYPE, int NK>
__global__ void __launch_bounds__(256) k_delta_chain(ChunkArgs ca) {
    using Plan = ChunkPlan<TYPE, NK>;
    constexpr int P = Plan::P, PA = Plan::PA, ORDER = TYPE == kTypeF32 ? 3 : 2;
    extern __shared__ __align__(16) char lds[];
    const DeltaArgs& a = ca.d;
    const int64_t pairs = gridDim.x / (unsigned)a.slices;
    const int64_t local = blockIdx.x % pairs, pair = ca.pair0 + local;     // (a head's workgroups on one XCD, if the pairs are a multiple of eight)
    const int slice = (int)(blockIdx.x / pairs);
    const int r = (int)(pair / a.heads), h = (int)(pair - (int64_t)r * a.heads);
    const int wave = __builtin_amdgcn_readfirstlane(wave_id()), ln = lane_id(), c = ln >> 4, n = ln & 15;
    const int n_new = delta_new(a, r), begin = ca.chunk0 * kChunk;
    const int chunks = min(ca.chunks, (n_new - begin + kChunk - 1) / kChunk);
    if (!ca.first && chunks <= 0) return;
    const int col = slice * kDeltaColumns + 16 * wave + n;
    const bool live = slice * kDeltaColumns + 16 * wave < a.Dv;
    const int64_t size = (int64_t)a.Dk * a.Dv;

    f32x4 S[2 * NK];
    const int parent = delta_parent(a, r);
    const float* from = ca.first ? a.state_in + (parent < 0 ? 0 : ((int64_t)parent * a.heads + h) * size) : a.state_out + pair * size;
    const bool any = live && (!ca.first || parent >= 0);
#pragma unroll
    for (int t = 0; t < 2 * NK; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int d = row_of(t, 4 * c + i);
            S[t][i] = any && d < a.Dk ? from[(int64_t)d * a.Dv + col] : 0.f;
        }
    // (the compiler's own wait for these loads: here, not with every stage)
#pragma unroll
    for (int t = 0; t < 2 * NK; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(S[t][i]));

    if (chunks > 0) {
        constexpr int kStages = Plan::kStages + Plan::kVStages;
        const char* room = ca.room + (size_t)local * ca.chunks * ca.bytes;
        int ask_chunk = 0, ask_stage = 0, ask_slot = 0, slot = 0;
        auto ask = [&]() {                     // the next stage to its slot: two operands a wave
            const char* of = room + (size_t)ask_chunk * ca.bytes;
            const int v = ask_stage - Plan::kBeforeV;
            if (v >= 0 && v < Plan::kVStages) of += ((size_t)Plan::kStages + slice * Plan::kVStages + v) * (kStageBlocks * 1024);
            else of += (size_t)(v < 0 ? ask_stage : ask_stage - Plan::kVStages) * (kStageBlocks * 1024);
            of += wave * 2048 + ln * 16;
            char* to = lds + ask_slot * (kStageBlocks * 1024) + wave * 2048;
            load_to_lds16(of, to);
            load_to_lds16(of + 1024, to + 1024);
            ask_slot = ask_slot + 1 == kRing ? 0 : ask_slot + 1;
            if (++ask_stage == kStages) { ask_stage = 0; ask_chunk = min(ask_chunk + 1, chunks - 1); }   // (behind the end the last chunk once more)
        };
        const char* stage = lds;
        auto next_stage = [&]() {
            wait_vmem<2 * (kRing - 2)>();
            lds_barrier();
            stage = lds + slot * (kStageBlocks * 1024);
            slot = slot + 1 == kRing ? 0 : slot + 1;
            ask();
        };
        for (int i = 0; i < kRing - 1; ++i) ask();
        for (int chunk = 0; chunk < chunks; ++chunk) {
            auto block = [&](int b) {          // asked for one after the other
                if (b % kStageBlocks == 0) next_stage();
                return stage + b % kStageBlocks * 1024;
            };
            auto operand = [&](int b) { return *reinterpret_cast<const uint4*>(block(b) + 16 * ln); };
            f32x4 ks[4], qs[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) ks[t] = qs[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < NK; ++s) {
                float x[8];
                uint4 sp[3];
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = S[2 * s + (i >> 2)][i & 3];
                planes_of<3>(x, sp);
#pragma unroll
                for (int which = 0; which < 2; ++which)
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        uint4 op[P];
#pragma unroll
                        for (int p = 0; p < P; ++p) op[p] = operand(s * 8 * P + (which * 4 + t) * P + p);
                        if (which == 0) ks[t] = mfma_planes<3>(op, sp, ks[t]);
                        else qs[t] = mfma_planes<ORDER>(op, sp, qs[t]);
                    }
            }
            f32x4 v[4], e[4], last[4];
#pragma unroll
            for (int part = 0; part < 2 * Plan::kVStages; ++part) {
                if (part % 2 == 0) next_stage();
                const uint4 w = *reinterpret_cast<const uint4*>(stage + (2 * wave + part % 2) * 1024 + 16 * ln);
                const uint32_t words[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if constexpr (TYPE == kTypeF32) v[part][i] = __uint_as_float(words[i]);
                    else {
                        v[2 * part + (i >> 1)][2 * (i & 1)] = word_f32<TYPE>((uint16_t)(words[i] & 0xffffu));
                        v[2 * part + (i >> 1)][2 * (i & 1) + 1] = word_f32<TYPE>((uint16_t)(words[i] >> 16));
                    }
                }
            }
            const float* scalars = reinterpret_cast<const float*>(block(Plan::kScalars));
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                e[t] = *reinterpret_cast<const f32x4*>(scalars + row_of(t, 4 * c));
                last[t] = *reinterpret_cast<const f32x4*>(scalars + 64 + row_of(t, 4 * c));
            }
            const float all = scalars[63];
            // U = T (V - e K S)
            uint4 rp[2][3];
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                float x[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int t = 2 * s + (i >> 2);
                    x[i] = fmaf(-e[t][i & 3], ks[t][i & 3], v[t][i & 3]);
                }
                planes_of<3>(x, rp[s]);
            }
            f32x4 u[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                u[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int s = 0; s <= t >> 1; ++s) {
                    uint4 op[3];
#pragma unroll
                    for (int p = 0; p < 3; ++p) op[p] = operand(Plan::kT + 3 * block_of(t, s) + p);
                    u[t] = mfma_planes<3>(op, rp[s], u[t]);
                }
            }
            // out = scale (e Q S + A U), and what the state gets
            uint4 up[2][PA], lp[2][3];
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                float x[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = u[2 * s + (i >> 2)][i & 3];
                planes_of<PA>(x, up[s]);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] *= last[2 * s + (i >> 2)][i & 3];
                planes_of<3>(x, lp[s]);
            }
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                f32x4 o;
#pragma unroll
                for (int i = 0; i < 4; ++i) o[i] = e[t][i] * qs[t][i];
#pragma unroll
                for (int s = 0; s <= t >> 1; ++s) {
                    uint4 op[PA];
#pragma unroll
                    for (int p = 0; p < PA; ++p) op[p] = operand(Plan::kA + PA * block_of(t, s) + p);
                    o = mfma_planes<ORDER>(op, up[s], o);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int token = begin + chunk * kChunk + row_of(t, 4 * c + i);
                    if (live && token < n_new) put_value<TYPE>(a.out, r * a.op.row + (int64_t)token * a.op.token + h * a.op.head + col, a.scale * o[i]);
                }
            }
#pragma unroll
            for (int t = 0; t < 2 * NK; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) S[t][i] *= all;
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int t = 0; t < 2 * NK; ++t) {
                    uint4 op[P];
#pragma unroll
                    for (int p = 0; p < P; ++p) op[p] = operand(Plan::kKt + (s * 2 * NK + t) * P + p);
                    S[t] = mfma_planes<3>(op, lp[s], S[t]);
                }
        }
        wait_vmem<0>();                        // (what was asked for behind the end must not come into another workgroup's LDS)
    }
    if (!live) return;
    float* to = a.state_out + pair * size;
#pragma unroll
    for (int t = 0; t < 2 * NK; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int d = row_of(t, 4 * c + i);
            if (d < a.Dk) to[(int64_t)d * a.Dv + col] = S[t][i];
        }
}

}  // namespace lshbeam
