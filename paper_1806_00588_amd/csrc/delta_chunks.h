// The gated delta rule over many tokens, 64 at a time.  In a chunk, with c_i the sum of the decays of its tokens up to i, S the state before it and
// e_i = e^(c_i):
//   (1 + L) U = diag(b) (V - e K S),     L_ij = b_i e^(c_i - c_j) k_i.k_j  for j < i
//   out = scale (e Q S + A U),           A_ij = e^(c_i - c_j) q_i.k_j      for j <= i
//   S <- e^(c_last) S + K^T (e^(c_last - c_j) u_j)_j
//
// What does not depend on the state -- T = (1 + L)^-1 diag(b), A, and K, Q, K^T in the order of the matrix operands -- is made for all chunks at once
// by k_delta_prepare and goes through the workspace; k_delta_chain goes through a row's chunks in order.  The state's columns do not meet: a wave
// has 16 of them in registers, four waves share what comes through LDS.
//
// v_mfma_f32_16x16x32_bf16 everywhere, numbers of 32 bits as three planes of bf16 that add up to them (queries and keys of 16 bits: one plane of bf16,
// two for fp16), whatever the results' type.  A plane is what the ones before it leave, rounded to nearest: at most 2^-8 and 2^-17 of the number, of either
// sign.  Of the products of planes those of a second and a third, and of two thirds, are left out: 2^-24 of a product at most, 2^-28 in the mean, as
// often of one sign as of the other.  A result D of an instruction has rows 4 c + i in lane (n, c), an
// operand rows 8 c + j: rows of the K, Q and T operands are in the order row_of below, so that two results' registers are the next
// product's operand as they are, and nothing is exchanged between lanes.
#pragma once
#include "delta_rule.h"

namespace lshbeam {

constexpr int kChunk = 64;            // tokens

// Row of row m of tile t: of two tiles, lane c's 4 + 4 rows are neighbours.
__host__ __device__ constexpr int row_of(int t, int m) { return 32 * (t >> 1) + 8 * (m >> 2) + 4 * (t & 1) + (m & 3); }
__device__ __forceinline__ int tile_of_row(int r) { return 2 * (r >> 5) + (r >> 2 & 1); }
__device__ __forceinline__ int place_of_row(int r) { return 4 * (r >> 3 & 3) + (r & 3); }

// Operands of a chunk and head in the workspace, NK = ceil(k_dim / 32):
//   for each 32 of k_dim: K and Q [4 tiles of tokens][planes]; then e and e^(c_last - c_j) [2][64] fp32; T and A [6][3]; K^T [2][2 NK tiles][planes]
// in blocks of 1 KB.  Of T and A those (tile of rows, 32 columns) that are not zero: (0, 0), (1, 0),
// (2, 0), (2, 1), (3, 0), (3, 1).
template <int TYPE, int NK> struct ChunkPlan {
    static constexpr int P = TYPE == kTypeBf16 ? 1 : TYPE == kTypeF16 ? 2 : 3;    // planes of K and Q
    static constexpr int kScalars = NK * 8 * P, kT = kScalars + 1, kA = kT + 18, kKt = kA + 18, kBlocks = kKt + 4 * NK * P;
};
__host__ __device__ constexpr int block_of(int t, int s) { return t < 2 ? t : 2 * t - 2 + s; }

struct ChunkArgs {
    DeltaArgs d;
    char* room;                // workspace: [pairs][chunks of the segment] of pair_bytes
    size_t bytes;              // of a chunk
    int64_t pair0, pairs;      // pairs of a row and a head of the launch
    int chunk0, chunks;        // the segment
    bool first;                // the state comes from the parent, else from state_out
};

__device__ __forceinline__ f32x4 mfma_bf16(uint4 a, uint4 b, f32x4 acc) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
}
// Eight values as NP operands that add up to them: each the bf16 nearest to what is left (from 3.39e38 on, which is that type's largest, infinite).
template <int NP> __device__ __forceinline__ void near_planes(const float (&x)[8], uint4 (&out)[NP]) {
    float rest[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) rest[i] = x[i];
#pragma unroll
    for (int p = 0; p < NP; ++p) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f32x2 v = {rest[2 * i], rest[2 * i + 1]};
            w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
            if (p + 1 < NP) { rest[2 * i] -= __uint_as_float(w[i] << 16); rest[2 * i + 1] -= __uint_as_float(w[i] & 0xffff0000u); }
        }
        out[p] = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// N products of planes i of a and j of b with i + j < 3, the smallest first; one after the other of the N, each waiting for its own sum
// alone (an instruction that adds to the one before it waits for that).
template <int N, int PA, int PB> __device__ __forceinline__ void mfma_planes(const uint4 (&a)[N][PA], const uint4 (&b)[PB], f32x4 (&acc)[N]) {
#pragma unroll
    for (int sum = 2; sum >= 0; --sum)
#pragma unroll
        for (int i = 0; i < PA; ++i)
            if (sum - i >= 0 && sum - i < PB) {
#pragma unroll
                for (int n = 0; n < N; ++n) acc[n] = mfma_bf16(a[n][i], b[sum - i], acc[n]);
            }
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

// LDS: the keys and later T in their place, L, small things.
template <int TYPE, int NK> constexpr int kPrepareKeys = ChunkPlan<TYPE, NK>::P * 4 * NK * 1024 > 64 * kMatrixPitch * 4 ? ChunkPlan<TYPE, NK>::P * 4 * NK * 1024 : 64 * kMatrixPitch * 4;
template <int TYPE, int NK> constexpr int kPrepareLds = kPrepareKeys<TYPE, NK> + (64 * kMatrixPitch + 3 * 64) * 4;

// A workgroup of four waves for a chunk of a row and head.
template <int TYPE, int NK>
__global__ void __launch_bounds__(256) k_delta_prepare(ChunkArgs ca) {
    using Plan = ChunkPlan<TYPE, NK>;
    constexpr int P = Plan::P;
    extern __shared__ __align__(16) char lds[];
    const DeltaArgs& a = ca.d;
    float* T = reinterpret_cast<float*>(lds);
    float* L = reinterpret_cast<float*>(lds + kPrepareKeys<TYPE, NK>);
    float* chi = L + 64 * kMatrixPitch;
    float *clo = chi + 64, *beta = clo + 64;
    const int64_t pair = ca.pair0 + blockIdx.x / (unsigned)ca.chunks;
    const int at = blockIdx.x % (unsigned)ca.chunks;
    const int r = (int)(pair / a.heads), h = (int)(pair - (int64_t)r * a.heads), hk = h / (a.heads / a.k_heads);
    const int t0 = (ca.chunk0 + at) * kChunk, n = min(kChunk, delta_new(a, r) - t0);
    if (n <= 0) return;
    char* to = ca.room + (size_t)blockIdx.x * ca.bytes;
    const int wave = __builtin_amdgcn_readfirstlane(wave_id()), ln = lane_id(), c = ln >> 4, m = ln & 15;

    // queries of the wave's tile: asked for before anything waits
    float xq[NK][8];
    {
        const int t = row_of(wave, m);
        const int64_t q0 = r * a.qp.row + (int64_t)(t0 + t) * a.qp.token + hk * a.qp.head + 8 * c;
#pragma unroll
        for (int s = 0; s < NK; ++s) {
#pragma unroll
            for (int i = 0; i < 8; ++i) xq[s][i] = 0.f;
            if (t < n && 32 * s + 8 * c < a.Dk) load_values<TYPE>(a.q, q0 + 32 * s, xq[s]);
        }
    }
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
        const double rest = last - sum;          // (e^(h + l) = e^h (1 + l), l being some 2^-24 of h at most)
        scalars[ln] = expf((float)sum) * (1.f + (float)(sum - (double)(float)sum));
        scalars[64 + ln] = expf((float)rest) * (1.f + (float)(rest - (double)(float)rest));
    }
    // keys: planes as operands
    for (int u = threadIdx.x; u < kChunk * NK * 4; u += 256) {
        const int piece = u % (NK * 4), t = u / (NK * 4);
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = 0.f;
        if (t < n && 8 * piece < a.Dk) load_values<TYPE>(a.k, r * a.kp.row + (int64_t)(t0 + t) * a.kp.token + hk * a.kp.head + 8 * piece, x);
        uint4 op[P];
        near_planes<P>(x, op);
#pragma unroll
        for (int p = 0; p < P; ++p)
            *reinterpret_cast<uint4*>(lds + (((p * 4 + tile_of_row(t)) * NK + (piece >> 2)) * 64 + 16 * (piece & 3) + place_of_row(t)) * 16) = op[p];
    }
    for (int i = threadIdx.x; i < 64 * kMatrixPitch; i += 256) L[i] = 0.f;
    __syncthreads();

    auto key = [&](int p, int t, int s) { return *reinterpret_cast<const uint4*>(lds + (((p * 4 + t) * NK + s) * 64 + ln) * 16); };
    // a wave for a tile of rows: K K^T, and Q K^T with its own tile of Q
    f32x4 kk[4], qk[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) kk[j] = qk[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int tiles = 2 * (wave >> 1) + 2;
#pragma unroll
    for (int s = 0; s < NK; ++s) {
        uint4 kq[2][P];
        near_planes<P>(xq[s], kq[1]);
#pragma unroll
        for (int p = 0; p < P; ++p) {
            kq[0][p] = key(p, wave, s);
            char* block = to + (size_t)(s * 8 * P + wave * P + p) * 1024 + 16 * ln;
            *reinterpret_cast<uint4*>(block) = kq[0][p];
            *reinterpret_cast<uint4*>(block + 4 * P * 1024) = kq[1][p];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (j >= tiles) break;
            uint4 other[P];
#pragma unroll
            for (int p = 0; p < P; ++p) other[p] = key(p, j, s);
            f32x4 both[2] = {kk[j], qk[j]};
            mfma_planes(kq, other, both);
            kk[j] = both[0];
            qk[j] = both[1];
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
    __syncthreads();
    for (int i = threadIdx.x; i < 64 * kMatrixPitch; i += 256) T[i] = 0.f;
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
        uint4 tp[3], ap[3];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = T[from + i] * beta[32 * s + 8 * c + i];
        near_planes<3>(x, tp);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = L[from + i];
        near_planes<3>(x, ap);
#pragma unroll
        for (int p = 0; p < 3; ++p) *reinterpret_cast<uint4*>(to + (size_t)(Plan::kT + 3 * b + p) * 1024 + 16 * ln) = tp[p];
#pragma unroll
        for (int p = 0; p < 3; ++p) *reinterpret_cast<uint4*>(to + (size_t)(Plan::kA + 3 * b + p) * 1024 + 16 * ln) = ap[p];
    }
}

// LDS of k_delta_chain: K S and Q S of each wave's rows of the state; V - e K S, U, and e^(c_last - c_j) U as operands.  OVER: U lies over the sums.
template <bool OVER, int TILES> struct ChainLds {
    static constexpr int kR = TILES * 4 * 8 * 1024, kU = OVER ? 0 : kR + TILES * 2 * 3 * 1024, kLast = kU + TILES * 2 * 3 * 1024;
    static constexpr int kBytes = OVER ? kR + TILES * 2 * 3 * 1024 : kLast + TILES * 2 * 3 * 1024;
};

// Planes of a tile's four values a lane: its half of the operand that two tiles make.
__device__ __forceinline__ void put_half(char* to, int tile, const f32x4& v) {
    const float x[8] = {v[0], v[1], v[2], v[3], 0.f, 0.f, 0.f, 0.f};
    uint4 op[3];
    near_planes<3>(x, op);
#pragma unroll
    for (int p = 0; p < 3; ++p) *reinterpret_cast<uint2*>(to + ((tile >> 1) * 3 + p) * 1024 + 16 * lane_id() + 8 * (tile & 1)) = make_uint2(op[p].x, op[p].y);
}
// One tile's sum of products of planes, in two accumulators (an instruction that adds to the one before it waits for that).
template <int PA, int PB> __device__ __forceinline__ void mfma_two(const uint4 (&a)[PA], const uint4 (&b)[PB], f32x4 (&acc)[2]) {
    int turn = 0;
#pragma unroll
    for (int sum = 2; sum >= 0; --sum)
#pragma unroll
        for (int i = 0; i < PA; ++i)
            if (sum - i >= 0 && sum - i < PB) { acc[turn & 1] = mfma_bf16(a[i], b[sum - i], acc[turn & 1]); ++turn; }
}

// A workgroup of four waves for 16 columns of a row's and head's state, or 32.  Wave w has the state's rows of every fourth 32 of k_dim in registers, and of what
// is made for tokens the tile w; K S, V - e K S and U are exchanged through LDS, three barriers a chunk.  So an operand is loaded by one wave, straight
// to registers.  Bound by the chain of a chunk: some 430 instructions a wave and tile of columns, 54 of them matrix ones, four phases that wait for each other.
// 16 heads of 128 x 128 in bf16, 128 workgroups, operands asked for a chunk ahead: 2.16 us a chunk; k_delta_apart 1.85.  (Four waves with columns of their own,
// operands through LDS: each goes through all of a chunk's 182 matrix and 1200 other instructions, 4.0 us a chunk, and a wave alone on its CU 4.5.)
// Where there are more than 512 workgroups of 16 columns, 32 columns and two workgroups a CU that ask when they need it: 144 heads of 96 x 160 in fp16,
// up to 700 tokens, with what comes before 119 us; asking ahead 125, 16 columns 124, asking ahead 145.
// AHEAD: operands are asked for a chunk ahead, for which a workgroup has a CU for itself, or when they are needed.  TILES: times 16 columns.
template <int TYPE, int NK, bool AHEAD, int TILES>
__global__ void __launch_bounds__(256, TILES) k_delta_chain(ChunkArgs ca) {
    using Plan = ChunkPlan<TYPE, NK>;
    constexpr int P = Plan::P, MINE = (NK + 3) / 4;
    constexpr bool OVER = TILES == 2;                      // (two workgroups a CU)
    using Lds = ChainLds<OVER, TILES>;
    __shared__ __align__(16) char lds[Lds::kBytes];
    const DeltaArgs& a = ca.d;
    // workgroups go round the eight XCDs one by one: those of a pair follow each other on one of them, so that its operands come from there but once
    const unsigned tiles = (((unsigned)a.Dv >> 4) + TILES - 1) / TILES, on_xcd = blockIdx.x >> 3;
    const int64_t local = (int64_t)(on_xcd / tiles) * 8 + (blockIdx.x & 7), pair = ca.pair0 + local;
    const int tile = (int)(on_xcd % tiles) * TILES;
    if (local >= ca.pairs) return;
    const int r = (int)(pair / a.heads), h = (int)(pair - (int64_t)r * a.heads);
    const int wave = __builtin_amdgcn_readfirstlane(wave_id()), ln = lane_id(), c = ln >> 4, n = ln & 15;
    const int n_new = delta_new(a, r), begin = ca.chunk0 * kChunk;
    const int chunks = min(ca.chunks, (n_new - begin + kChunk - 1) / kChunk);
    if (!ca.first && chunks <= 0) return;
    int col[TILES];            // (tiles behind the last: the last one once more, without results)
    bool live[TILES];
#pragma unroll
    for (int k = 0; k < TILES; ++k) {
        live[k] = 16 * (tile + k) < a.Dv;
        col[k] = min(16 * (tile + k), a.Dv - 16) + n;
    }
    const int64_t size = (int64_t)a.Dk * a.Dv;

    f32x4 S[TILES][MINE][2];
    const int parent = delta_parent(a, r);
    const float* from = ca.first ? a.state_in + (parent < 0 ? 0 : ((int64_t)parent * a.heads + h) * size) : a.state_out + pair * size;
    const bool any = !ca.first || parent >= 0;
#pragma unroll
    for (int k = 0; k < TILES; ++k)
#pragma unroll
        for (int j = 0; j < MINE; ++j)
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int d = row_of(2 * (wave + 4 * j) + t, 4 * c + i);
                    S[k][j][t][i] = any && d < a.Dk ? from[(int64_t)d * a.Dv + col[k]] : 0.f;
                }

    // Operands.  What a wave has no work for it asks for all the same (another's): the number of loads under way is known to the compiler then.
    struct Operands {
        uint4 kq[MINE][8][P], kt[MINE][4][P], tp[2][3], ap[2][3];
        f32x4 e, last;
        float all;
        typename WordOf<TYPE>::type v[TILES][4];
    } set;
    const char* room = ca.room + (size_t)local * ca.chunks * ca.bytes;       // (the same for all lanes, and stays in scalar registers)
    const int64_t v_from = r * a.vp.row + h * a.vp.head;
    auto block = [&](int chunk, int b) { return reinterpret_cast<const uint4*>(room + (size_t)chunk * ca.bytes + (size_t)b * 1024)[(unsigned)ln]; };
    auto ask_kq = [&](Operands& to, int chunk) {
#pragma unroll
        for (int j = 0; j < MINE; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int p = 0; p < P; ++p) to.kq[j][i][p] = block(chunk, (min(wave + 4 * j, NK - 1) * 8 + i) * P + p);
    };
    auto ask_values = [&](Operands& to, int chunk) {
        const float* scalars = reinterpret_cast<const float*>(room + (size_t)chunk * ca.bytes + Plan::kScalars * 1024);
        to.e = *reinterpret_cast<const f32x4*>(scalars + row_of(wave, 4 * c));
        to.last = *reinterpret_cast<const f32x4*>(scalars + 64 + row_of(wave, 4 * c));
        to.all = scalars[63];
#pragma unroll
        for (int i = 0; i < 4; ++i) {                                        // (tokens behind the last count as if they were it: T has zeros there)
            const int token = min(begin + chunk * kChunk + row_of(wave, 4 * c + i), n_new - 1);
#pragma unroll
            for (int k = 0; k < TILES; ++k) to.v[k][i] = static_cast<const typename WordOf<TYPE>::type*>(a.v)[v_from + token * a.vp.token + col[k]];
        }
    };
    auto ask_t = [&](Operands& to, int chunk) {
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int p = 0; p < 3; ++p) to.tp[s][p] = block(chunk, Plan::kT + 3 * block_of(wave, min(s, wave >> 1)) + p);
    };
    auto ask_a = [&](Operands& to, int chunk) {
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int p = 0; p < 3; ++p) to.ap[s][p] = block(chunk, Plan::kA + 3 * block_of(wave, min(s, wave >> 1)) + p);
    };
    auto ask_kt = [&](Operands& to, int chunk) {
#pragma unroll
        for (int j = 0; j < MINE; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i)                                      // [32 tokens][tile of the state's rows]
#pragma unroll
                for (int p = 0; p < P; ++p) to.kt[j][i][p] = block(chunk, Plan::kKt + ((i >> 1) * 2 * NK + 2 * min(wave + 4 * j, NK - 1) + (i & 1)) * P + p);
    };
    if (AHEAD && chunks > 0) { ask_kq(set, 0); ask_values(set, 0); ask_t(set, 0); ask_a(set, 0); ask_kt(set, 0); }

    const f32x4 none = {0.f, 0.f, 0.f, 0.f};
    f32x4* part = reinterpret_cast<f32x4*>(lds);
    auto read = [&](int at, int b) { return *reinterpret_cast<const uint4*>(lds + at + b * 1024 + 16 * ln); };
    auto work = [&](Operands& of, int chunk) __attribute__((always_inline)) {
        const int after = min(chunk + AHEAD, chunks - 1);                    // (behind the end the last chunk once more)
        if constexpr (!AHEAD) { ask_kq(of, chunk); ask_values(of, chunk); }
        // K S and Q S: of the wave's rows of the state
        f32x4 ks[TILES][4], qs[TILES][4];
#pragma unroll
        for (int k = 0; k < TILES; ++k)
#pragma unroll
            for (int t = 0; t < 4; ++t) ks[k][t] = qs[k][t] = none;
#pragma unroll
        for (int j = 0; j < MINE; ++j)
            if (wave + 4 * j < NK) {
                uint4 op[2][4][P];
#pragma unroll
                for (int t = 0; t < 8; ++t)
#pragma unroll
                    for (int p = 0; p < P; ++p) op[t >> 2][t & 3][p] = of.kq[j][t][p];
#pragma unroll
                for (int k = 0; k < TILES; ++k) {
                    float x[8];
                    uint4 sp[3];
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = S[k][j][i >> 2][i & 3];
                    near_planes<3>(x, sp);
                    mfma_planes(op[0], sp, ks[k]);
                    mfma_planes(op[1], sp, qs[k]);
                }
            }
        if constexpr (AHEAD) ask_kq(of, after);
        else ask_t(of, chunk);
#pragma unroll
        for (int k = 0; k < TILES; ++k)
#pragma unroll
            for (int t = 0; t < 4; ++t) { part[((k * 4 + wave) * 8 + t) * 64 + ln] = ks[k][t]; part[((k * 4 + wave) * 8 + 4 + t) * 64 + ln] = qs[k][t]; }
        lds_barrier();
        // V - e K S of the wave's tile of tokens
        f32x4 q_sum[TILES];
#pragma unroll
        for (int k = 0; k < TILES; ++k) {
            f32x4 k_sum = none, v;
#pragma unroll
            for (int w = 0; w < 4; ++w)
                if (w < NK) k_sum += part[((k * 4 + w) * 8 + wave) * 64 + ln];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = fmaf(-of.e[i], k_sum[i], word_f32<TYPE>(of.v[k][i]));
            put_half(lds + Lds::kR + k * (2 * 3 * 1024), wave, v);
            q_sum[k] = none;
#pragma unroll
            for (int w = 0; w < 4; ++w)
                if (w < NK) q_sum[k] += part[((k * 4 + w) * 8 + 4 + wave) * 64 + ln];
            q_sum[k] *= of.e;
        }
        lds_barrier();
        // U = T (V - e K S)
#pragma unroll
        for (int k = 0; k < TILES; ++k) {
            f32x4 two[2] = {none, none};
#pragma unroll
            for (int s = 0; s < 2; ++s)
                if (s <= wave >> 1) {
                    const int at = Lds::kR + k * (2 * 3 * 1024);
                    const uint4 rp[3] = {read(at, 3 * s), read(at, 3 * s + 1), read(at, 3 * s + 2)};
                    mfma_two(of.tp[s], rp, two);
                }
            const f32x4 u = two[0] + two[1];
            put_half(lds + Lds::kU + k * (2 * 3 * 1024), wave, u);
            put_half(lds + Lds::kLast + k * (2 * 3 * 1024), wave, u * of.last);
        }
        if constexpr (AHEAD) ask_t(of, after);
        else { ask_a(of, chunk); ask_kt(of, chunk); }
        const float decay = of.all;
        if constexpr (AHEAD) ask_values(of, after);
        lds_barrier();
        // the state
#pragma unroll
        for (int k = 0; k < TILES; ++k) {
            uint4 lp[2][3];
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int p = 0; p < 3; ++p) lp[s][p] = read(Lds::kLast + k * (2 * 3 * 1024), 3 * s + p);
#pragma unroll
            for (int j = 0; j < MINE; ++j)
                if (wave + 4 * j < NK) {
                    S[k][j][0] *= decay;
                    S[k][j][1] *= decay;
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        uint4 op[2][P];
#pragma unroll
                        for (int t = 0; t < 2; ++t)
#pragma unroll
                            for (int p = 0; p < P; ++p) op[t][p] = of.kt[j][2 * s + t][p];
                        mfma_planes(op, lp[s], S[k][j]);
                    }
                }
        }
        if constexpr (AHEAD) ask_kt(of, after);
        // out = scale (e Q S + A U)
        f32x4 o[TILES][2];
#pragma unroll
        for (int k = 0; k < TILES; ++k) {
            o[k][0] = q_sum[k];
            o[k][1] = none;
#pragma unroll
            for (int s = 0; s < 2; ++s)
                if (s <= wave >> 1) {
                    uint4 up[3];
#pragma unroll
                    for (int p = 0; p < 3; ++p) up[p] = read(Lds::kU + k * (2 * 3 * 1024), 3 * s + p);
                    mfma_two(of.ap[s], up, o[k]);
                }
        }
        if constexpr (AHEAD) ask_a(of, after);
        if constexpr (OVER) lds_barrier();                                   // (the next sums go where U is)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int token = begin + chunk * kChunk + row_of(wave, 4 * c + i);
            if (token < n_new) {
                const int64_t at = r * a.op.row + (int64_t)token * a.op.token + h * a.op.head;
#pragma unroll
                for (int k = 0; k < TILES; ++k)
                    if (live[k]) put_value<TYPE>(a.out, at + col[k], a.scale * (o[k][0][i] + o[k][1][i]));
            }
        }
    };
    for (int chunk = 0; chunk < chunks; ++chunk) work(set, chunk);
    float* to = a.state_out + pair * size;
#pragma unroll
    for (int k = 0; k < TILES; ++k)
#pragma unroll
        for (int j = 0; j < MINE; ++j)
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int d = row_of(2 * (wave + 4 * j) + t, 4 * c + i);
                    if (live[k] && d < a.Dk) to[(int64_t)d * a.Dv + col[k]] = S[k][j][t][i];
                }
}

// Eight waves for 16 columns: four of them as in k_delta_chain, which have the state and make U, and four that make the results, a tile of tokens each, while
// the others go on: these give the state's planes and U to them through LDS, so that Q S, A U and the results are out of the chunk's chain.  16 heads of
// 128 x 128 in bf16, 8192 tokens: 237 us, 1.85 a chunk (k_delta_chain 277; keys and queries straight from where they lie, rows a few KB apart, 30 more when tried).  A workgroup has a CU for itself; of more than two rounds of them k_delta_chain is quicker
// (144 heads of 96 x 160 in fp16, up to 700 tokens: with what comes before 119 us, this 133).
// AHEAD: chunks that operands are asked for ahead, what there are registers for.
template <int TYPE, int NK, int AHEAD>
__global__ void __launch_bounds__(512, 1) k_delta_apart(ChunkArgs ca) {
    using Plan = ChunkPlan<TYPE, NK>;
    constexpr int P = Plan::P, MINE = (NK + 3) / 4;
    // LDS: K S of each wave's rows of the state; the state; V - e K S, U, and e^(c_last - c_j) U as operands
    constexpr int kState = 4 * 4 * 1024, kR = kState + NK * 3 * 1024, kU = kR + 2 * 3 * 1024, kLast = kU + 2 * 3 * 1024;
    __shared__ __align__(16) char lds[kLast + 2 * 3 * 1024];
    const DeltaArgs& a = ca.d;
    const unsigned tiles = (unsigned)a.Dv >> 4, on_xcd = blockIdx.x >> 3;
    const int64_t local = (int64_t)(on_xcd / tiles) * 8 + (blockIdx.x & 7), pair = ca.pair0 + local;
    if (local >= ca.pairs) return;
    const int r = (int)(pair / a.heads), h = (int)(pair - (int64_t)r * a.heads);
    const int wave = __builtin_amdgcn_readfirstlane(wave_id()) & 3, ln = lane_id(), c = ln >> 4, n = ln & 15;
    const bool results = __builtin_amdgcn_readfirstlane(wave_id()) >= 4;
    const int n_new = delta_new(a, r), begin = ca.chunk0 * kChunk, col = 16 * (int)(on_xcd % tiles) + n;
    const int chunks = min(ca.chunks, (n_new - begin + kChunk - 1) / kChunk);
    if (!ca.first && chunks <= 0) return;
    const char* room = ca.room + (size_t)local * ca.chunks * ca.bytes;       // (the same for all lanes, and stays in scalar registers)
    auto block = [&](int chunk, int b) { return reinterpret_cast<const uint4*>(room + (size_t)chunk * ca.bytes + (size_t)b * 1024)[(unsigned)ln]; };
    auto scalars = [&](int chunk) { return reinterpret_cast<const float*>(room + (size_t)chunk * ca.bytes + Plan::kScalars * 1024); };
    auto read = [&](int at, int b) { return *reinterpret_cast<const uint4*>(lds + at + b * 1024 + 16 * ln); };
    const f32x4 none = {0.f, 0.f, 0.f, 0.f};

    if (results) {
        struct Operands { uint4 q[NK][P], ap[2][3]; f32x4 e; } sets[AHEAD];
        auto ask_q = [&](Operands& to, int chunk) {
#pragma unroll
            for (int s = 0; s < NK; ++s)
#pragma unroll
                for (int p = 0; p < P; ++p) to.q[s][p] = block(chunk, (s * 8 + 4 + wave) * P + p);
            to.e = *reinterpret_cast<const f32x4*>(scalars(chunk) + row_of(wave, 4 * c));
        };
        auto ask_a = [&](Operands& to, int chunk) {
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int p = 0; p < 3; ++p) to.ap[s][p] = block(chunk, Plan::kA + 3 * block_of(wave, min(s, wave >> 1)) + p);
        };
        if (chunks > 0) {
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) { ask_q(sets[i], min(i, chunks - 1)); ask_a(sets[i], min(i, chunks - 1)); }
        }
        auto work = [&](Operands& of, int chunk) __attribute__((always_inline)) {
            const int after = min(chunk + AHEAD, chunks - 1);                // (behind the end the last chunk once more)
            lds_barrier();
            f32x4 o[2] = {none, none};
#pragma unroll
            for (int s = 0; s < NK; ++s) {
                uint4 sp[3];
#pragma unroll
                for (int p = 0; p < 3; ++p) sp[p] = read(kState, s * 3 + p);
                mfma_two(of.q[s], sp, o);
            }
            o[0] = (o[0] + o[1]) * of.e;
            o[1] = none;
            ask_q(of, after);
            lds_barrier();
            lds_barrier();
#pragma unroll
            for (int s = 0; s < 2; ++s)
                if (s <= wave >> 1) {
                    uint4 up[3];
#pragma unroll
                    for (int p = 0; p < 3; ++p) up[p] = read(kU, 3 * s + p);
                    mfma_two(of.ap[s], up, o);
                }
            ask_a(of, after);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int token = begin + chunk * kChunk + row_of(wave, 4 * c + i);
                if (token < n_new) put_value<TYPE>(a.out, r * a.op.row + (int64_t)token * a.op.token + h * a.op.head + col, a.scale * (o[0][i] + o[1][i]));
            }
        };
        for (int chunk = 0; chunk < chunks; chunk += AHEAD) {
            work(sets[0], chunk);
            if (AHEAD == 2 && chunk + 1 < chunks) work(sets[AHEAD - 1], chunk + 1);
        }
        return;
    }

    const int64_t size = (int64_t)a.Dk * a.Dv;
    const int parent = delta_parent(a, r);
    const float* from = ca.first ? a.state_in + (parent < 0 ? 0 : ((int64_t)parent * a.heads + h) * size) : a.state_out + pair * size;
    const bool any = !ca.first || parent >= 0;
    f32x4 S[MINE][2];
#pragma unroll
    for (int j = 0; j < MINE; ++j)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int d = row_of(2 * (wave + 4 * j) + t, 4 * c + i);
                S[j][t][i] = any && d < a.Dk ? from[(int64_t)d * a.Dv + col] : 0.f;
            }
    // (what a wave has no work for it asks for all the same, another's: the number of loads under way is known to the compiler then)
    struct Operands {
        uint4 k[MINE][4][P], kt[MINE][4][P], tp[2][3];
        f32x4 e, last;
        float all;
        typename WordOf<TYPE>::type v[4];
    } sets[AHEAD];
    const int64_t v_from = r * a.vp.row + h * a.vp.head + col;
    auto ask_k = [&](Operands& to, int chunk) {
#pragma unroll
        for (int j = 0; j < MINE; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int p = 0; p < P; ++p) to.k[j][i][p] = block(chunk, (min(wave + 4 * j, NK - 1) * 8 + i) * P + p);
    };
    auto ask_values = [&](Operands& to, int chunk) {
        to.e = *reinterpret_cast<const f32x4*>(scalars(chunk) + row_of(wave, 4 * c));
        to.last = *reinterpret_cast<const f32x4*>(scalars(chunk) + 64 + row_of(wave, 4 * c));
        to.all = scalars(chunk)[63];
#pragma unroll
        for (int i = 0; i < 4; ++i) {                                        // (tokens behind the last count as if they were it: T has zeros there)
            const int token = min(begin + chunk * kChunk + row_of(wave, 4 * c + i), n_new - 1);
            to.v[i] = static_cast<const typename WordOf<TYPE>::type*>(a.v)[v_from + token * a.vp.token];
        }
    };
    auto ask_t = [&](Operands& to, int chunk) {
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int p = 0; p < 3; ++p) to.tp[s][p] = block(chunk, Plan::kT + 3 * block_of(wave, min(s, wave >> 1)) + p);
    };
    auto ask_kt = [&](Operands& to, int chunk) {
#pragma unroll
        for (int j = 0; j < MINE; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i)                                      // [32 tokens][tile of the state's rows]
#pragma unroll
                for (int p = 0; p < P; ++p) to.kt[j][i][p] = block(chunk, Plan::kKt + ((i >> 1) * 2 * NK + 2 * min(wave + 4 * j, NK - 1) + (i & 1)) * P + p);
    };
    if (chunks > 0) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int chunk = min(i, chunks - 1);
            ask_k(sets[i], chunk); ask_values(sets[i], chunk); ask_t(sets[i], chunk); ask_kt(sets[i], chunk);
        }
    }
    f32x4* part = reinterpret_cast<f32x4*>(lds);
    auto work = [&](Operands& of, int chunk) __attribute__((always_inline)) {
        const int after = min(chunk + AHEAD, chunks - 1);
        // K S of the wave's rows of the state, and these for the results
        f32x4 ks[4] = {none, none, none, none};
#pragma unroll
        for (int j = 0; j < MINE; ++j)
            if (wave + 4 * j < NK) {
                float x[8];
                uint4 sp[3];
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = S[j][i >> 2][i & 3];
                near_planes<3>(x, sp);
#pragma unroll
                for (int p = 0; p < 3; ++p) *reinterpret_cast<uint4*>(lds + kState + ((wave + 4 * j) * 3 + p) * 1024 + 16 * ln) = sp[p];
                mfma_planes(of.k[j], sp, ks);
            }
        ask_k(of, after);
#pragma unroll
        for (int t = 0; t < 4; ++t) part[(wave * 4 + t) * 64 + ln] = ks[t];
        lds_barrier();
        // V - e K S of the wave's tile of tokens
        f32x4 k_sum = none, v;
#pragma unroll
        for (int w = 0; w < 4; ++w)
            if (w < NK) k_sum += part[(w * 4 + wave) * 64 + ln];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = fmaf(-of.e[i], k_sum[i], word_f32<TYPE>(of.v[i]));
        put_half(lds + kR, wave, v);
        lds_barrier();
        // U = T (V - e K S)
        f32x4 two[2] = {none, none};
#pragma unroll
        for (int s = 0; s < 2; ++s)
            if (s <= wave >> 1) {
                const uint4 rp[3] = {read(kR, 3 * s), read(kR, 3 * s + 1), read(kR, 3 * s + 2)};
                mfma_two(of.tp[s], rp, two);
            }
        const f32x4 u = two[0] + two[1];
        put_half(lds + kU, wave, u);
        put_half(lds + kLast, wave, u * of.last);
        const float decay = of.all;
        ask_t(of, after);
        ask_values(of, after);
        lds_barrier();
        // the state
        uint4 lp[2][3];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int p = 0; p < 3; ++p) lp[s][p] = read(kLast, 3 * s + p);
#pragma unroll
        for (int j = 0; j < MINE; ++j)
            if (wave + 4 * j < NK) {
                S[j][0] *= decay;
                S[j][1] *= decay;
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    uint4 op[2][P];
#pragma unroll
                    for (int t = 0; t < 2; ++t)
#pragma unroll
                        for (int p = 0; p < P; ++p) op[t][p] = of.kt[j][2 * s + t][p];
                    mfma_planes(op, lp[s], S[j]);
                }
            }
        ask_kt(of, after);
    };
    for (int chunk = 0; chunk < chunks; chunk += AHEAD) {
        work(sets[0], chunk);
        if (AHEAD == 2 && chunk + 1 < chunks) work(sets[AHEAD - 1], chunk + 1);
    }
    float* to = a.state_out + pair * size;
#pragma unroll
    for (int j = 0; j < MINE; ++j)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int d = row_of(2 * (wave + 4 * j) + t, 4 * c + i);
                if (d < a.Dk) to[(int64_t)d * a.Dv + col] = S[j][t][i];
            }
}

}  // namespace lshbeam
