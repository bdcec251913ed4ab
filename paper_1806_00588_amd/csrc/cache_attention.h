// Attention over a paged cache of 8-bit codes (lsh_cache_attention):
//   o[r, t, h] = sum_j p_j v_j,   p = softmax_j(scale * q[r, t, h] . k_j)   over the positions j of row r that token t sees.
//
// Single tokens: two operations per byte of the cache and query head, so the bytes bound it.  Everything that reads the same keys
// is therefore worked on together: the query heads of a key head, the new tokens of a row, and -- where `shared` says that a
// sentence's beams have their first blocks in common -- the beams.  Those are the columns of v_mfma_f32_16x16x32_bf16:
//   S^T [tokens, rows] = K Q^T      O^T [values, rows] += V^T P^T
// A code is exact in bf16.  Queries of 16 or 32 bits are taken apart into bf16 planes whose sum they are (bf16 1, fp16 2, fp32 3),
// and so are the probabilities (bf16: rounded, half a step of 2^-8; fp16: the first 16 bits; fp32: all 24), products and sums are fp32.
//
// A wave takes tiles of 64 tokens.  Row m of the K operand of sub-tile i is token 16 (m / 4) + 4 i + m % 4, so that lane (n, c) of the
// result holds, for row n of the queries, tokens 16 c + 4 i + j: the sixteen neighbours 16 c .. 16 c + 15, which are its part of the
// P^T operand as they are and lie in one block -- one scale of k and one of v for each lane.  Nothing is exchanged between lanes
// but the rows' maximum.  The cache's layout gives the operands' 16 bytes per lane in pieces of 64 (k) and 256 (v) bytes at least.
//
// k_attention_few   up to 16 rows of queries: the four waves of a workgroup take every fourth tile, straight from memory into
//                   registers (values of this tile asked for, products with its keys, keys of the next tile asked for, softmax,
//                   products with the values), and join through LDS.
// k_attention_rows  17 to 64 rows: a wave per 16 rows, all on the same tiles, which come through LDS two tiles ahead.
// The rows of a row set are split along the tokens into chunks, a workgroup's work.  Chunks leave (max, sum, products) in the
// workspace, k_attention_join adds them up in order.
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
    // of a launch: all beams of a sentence over the blocks that they have in common, or each row over the rest of its own
    int common;
    int has_common;            // there is a launch of the first kind
    int chunk;                 // tiles of a chunk
    int groups, splits;        // groups of rows; workgroups along the tokens
    int part0;                 // the first part that this launch writes
    int parts;                 // in all; 1: results are written at once
    float2* ml;                // workspace [R * T * q_heads, parts]: max of the products (times log2 e), sum of the exponentials; sum -1: done
    float* acc;                // workspace [R * T * q_heads, parts, D]
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

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

template <int TYPE> constexpr int kPlanes = TYPE == kTypeBf16 ? 1 : TYPE == kTypeF16 ? 2 : 3;
constexpr int kAttnTile = 64;    // tokens of a wave at a time

// Eight codes as an operand.
__device__ __forceinline__ bf16x8 codes_to_operand(uint32_t a, uint32_t b) {
    const bf16x2 r0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, false), r1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, true);
    const bf16x2 r2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, false), r3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, true);
    return bf16x8{r0.x, r0.y, r1.x, r1.y, r2.x, r2.y, r3.x, r3.y};
}

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

// Bytes of a word whose low seven bits are all ones (the code NaN), each as 0xff.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) {
    const uint32_t hit = ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
    return hit | (hit - (hit >> 7));
}

// What a row of the queries is and sees.
struct AttnRow { int r, t, head, lo, hi; bool valid; };
__device__ __forceinline__ AttnRow attn_row(const AttnArgs& a, int s_or_r, int h, int i) {
    const int g = a.q_heads / a.heads, per = a.T * g;
    AttnRow w{0, 0, 0, 0, 0, false};
    if (i >= (a.common ? a.B * per : per)) return w;
    const int b = a.common ? i / per : 0, at = i - b * per;
    w.r = a.common ? s_or_r * a.B + b : s_or_r;
    w.t = at / g;
    w.head = h * g + at - w.t * g;
    const int n = row_new(a, w.r);
    w.valid = w.t < n;
    if (w.valid) seen(a, row_length(a, w.r), n, w.t, &w.lo, &w.hi);
    return w;
}
// Tokens that the rows of sentence s have in common.
__device__ __forceinline__ int common_tokens(const AttnArgs& a, int s) {
    return a.has_common ? min(max(a.shared[s], 0), a.width) * a.block : 0;
}

// A workgroup's place and what is found out once for it.
constexpr int kMaxChunk = 32;                        // tiles
struct AttnShared {
    AttnRow row[64];
    int id[4 * kMaxChunk];                           // block of each 16 tokens of the chunk, -1: none that anybody here sees
    float k_scale[4 * kMaxChunk], v_scale[4 * kMaxChunk];   // times scale * log2 e; as it is
    int vlo, vhi, lo_most, hi_least, first_lo, table_row;
};
struct AttnPlace {
    int split, group, h, sr;                         // sr: sentence or row
    int shared_tokens;
    int tile0, tiles, chunks;                        // of the positions that any row sees here
    bool direct;                                     // nobody else has a part of these rows
};

// Rows, positions: by all threads, ends with a barrier.
template <int ROWS> __device__ __forceinline__ AttnPlace attn_place(const AttnArgs& a, AttnShared& sh) {
    AttnPlace p;
    int u = blockIdx.x;
    p.split = u % a.splits;
    u /= a.splits;
    p.group = u % a.groups;
    u /= a.groups;
    p.h = u % a.heads;
    p.sr = u / a.heads;
    const int s = a.common ? p.sr : p.sr / a.B;
    p.shared_tokens = common_tokens(a, s);
    const int from = a.common ? 0 : p.shared_tokens, to = a.common ? p.shared_tokens : INT32_MAX;
    if (wave_id() == 0) {
        const int i = lane_id();
        AttnRow w{0, 0, 0, 0, 0, false};
        if (i < ROWS) w = attn_row(a, p.sr, p.h, p.group * ROWS + i);
        int first = w.valid && w.lo < w.hi ? w.lo : INT32_MAX;
        w.lo = max(w.lo, from);
        w.hi = min(w.hi, to);
        const bool live = w.valid && w.lo < w.hi;
        int vlo = live ? w.lo : INT32_MAX, vhi = live ? w.hi : 0;
        // a row without a position here is worked on like the rest and left out at the end
        if (!live) { w.lo = INT32_MIN; w.hi = INT32_MAX; }
        int lo_most = w.lo, hi_least = w.hi, table_row = p.sr;
        if (i < ROWS) sh.row[i] = w;
        if (a.common) {                              // the sentence's first row with tokens
            int b0 = INT32_MAX;
            for (int b = i; b < a.B; b += kWave)
                if (b0 == INT32_MAX && a.lengths[p.sr * a.B + b] > 0) b0 = b;
#pragma unroll
            for (int off = 32; off > 0; off >>= 1) b0 = min(b0, __shfl_xor(b0, off, kWave));
            table_row = p.sr * a.B + min(b0, a.B - 1);
        }
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) {
            vlo = min(vlo, __shfl_xor(vlo, off, kWave));
            vhi = max(vhi, __shfl_xor(vhi, off, kWave));
            lo_most = max(lo_most, __shfl_xor(lo_most, off, kWave));
            hi_least = min(hi_least, __shfl_xor(hi_least, off, kWave));
            first = min(first, __shfl_xor(first, off, kWave));
        }
        if (i == 0) { sh.vlo = vlo; sh.vhi = vhi; sh.lo_most = lo_most; sh.hi_least = hi_least; sh.first_lo = first; sh.table_row = table_row; }
    }
    __syncthreads();
    const int vhi = __builtin_amdgcn_readfirstlane(sh.vhi);
    p.tile0 = vhi > 0 ? __builtin_amdgcn_readfirstlane(sh.vlo) / kAttnTile : 0;
    p.tiles = vhi > 0 ? (vhi + kAttnTile - 1) / kAttnTile - p.tile0 : 0;
    p.chunks = (p.tiles + a.chunk - 1) / a.chunk;
    p.direct = a.parts == 1 || (!a.common && p.chunks <= 1 && __builtin_amdgcn_readfirstlane(sh.first_lo) >= p.shared_tokens);
    return p;
}

// Queries to LDS as operands [plane, row tile, kk, half, lane].
template <int TYPE, int DP, int MT>
__device__ __forceinline__ void stage_queries(const AttnArgs& a, const AttnShared& sh, uint4* to, int threads) {
    using T = typename WordOf<TYPE>::type;
    constexpr int NP = kPlanes<TYPE>, KK = DP / 64;
    for (int e = threadIdx.x; e < 16 * MT * (DP / 8); e += threads) {
        const int cd = e % (DP / 8), row = e / (DP / 8);
        const AttnRow& w = sh.row[row];
        float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (w.valid && 8 * cd < a.D) {
            const T* p = static_cast<const T*>(a.q) + w.r * a.qp.row + w.t * a.qp.token + w.head * a.qp.head + 8 * cd;
            if constexpr (TYPE == kTypeF32) {
                const Float4U u = *reinterpret_cast<const Float4U*>(p), v = *reinterpret_cast<const Float4U*>(p + 4);
                x[0] = u.x; x[1] = u.y; x[2] = u.z; x[3] = u.w; x[4] = v.x; x[5] = v.y; x[6] = v.z; x[7] = v.w;
            } else {
                const Chunk16U<T> v = *reinterpret_cast<const Chunk16U<T>*>(p);
#pragma unroll
                for (int i = 0; i < 4; ++i) { x[2 * i] = word_f32<TYPE>((T)(v.w[i] & 0xffffu)); x[2 * i + 1] = word_f32<TYPE>((T)(v.w[i] >> 16)); }
            }
        }
        uint4 planes[NP];
        planes_of<NP>(x, planes);
        const int piece = cd >> 1, kk = piece >> 2, lane = (piece & 3) * 16 + (row & 15);
#pragma unroll
        for (int p = 0; p < NP; ++p) to[(((p * MT + (row >> 4)) * KK + kk) * 2 + (cd & 1)) * 64 + lane] = planes[p];
    }
}

// Blocks and scales of chunk `chunk`'s tokens, 16 at a time: thread i the i-th of them.
__device__ __forceinline__ void load_chunk(const AttnArgs& a, AttnShared& sh, const AttnPlace& p, int chunk) {
    const int i = threadIdx.x;
    if (i >= 4 * a.chunk) return;
    const int64_t pos = ((int64_t)p.tile0 + (int64_t)chunk * a.chunk) * kAttnTile + 16 * i;
    int32_t id = -1;
    if (pos < sh.vhi && pos + 15 >= sh.vlo && pos / a.block < a.width) {
        id = a.tables[(int64_t)sh.table_row * a.width + pos / a.block];
        id = id < a.n_blocks ? max(id, -1) : -1;
    }
    const int64_t at = (int64_t)max(id, 0) * a.heads + p.h;
    sh.id[i] = id;
    sh.k_scale[i] = id >= 0 ? a.scale_k[at] * (a.scale * 1.44269504f) : 0.f;
    sh.v_scale[i] = id >= 0 ? a.scale_v[at] : 0.f;
}

// A wave's sums for one row tile: lane (n, c) has values 16 dt + 4 c + j of row n, its maximum, and of its sum what its tokens give.
template <int DP> struct RowSums {
    float m = -INFINITY, l = 0.f;
    f32x4 acc[DP / 16];
    __device__ __forceinline__ RowSums() {
#pragma unroll
        for (int dt = 0; dt < DP / 16; ++dt) acc[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
};

// One tile: products with the keys (k(kk, i): 16 codes of a token), then `between()`, softmax, products with the values
// (v(dt): a value's codes of 16 tokens).  rel: the tile's number in the chunk, pos its first token.
template <int TYPE, int DP, int MT, bool EXACT, typename K, typename V, typename F>
__device__ __forceinline__ void attend_tile(const AttnArgs& a, const AttnShared& sh, const uint4* queries, int row_tile, int rel, int pos,
                                            int lo, int hi, RowSums<DP>& to, K k, V v, F between) {
    constexpr int NP = kPlanes<TYPE>, KK = DP / 64, DT = DP / 16;
    const int ln = lane_id(), c = ln >> 4, pieces = a.D >> 4;
    f32x4 sc[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) sc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
        if (EXACT || 4 * kk < pieces) {
            uint4 w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = k(kk, i);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                bf16x8 key[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) key[i] = half ? codes_to_operand(w[i].z, w[i].w) : codes_to_operand(w[i].x, w[i].y);
#pragma unroll
                for (int p = 0; p < NP; ++p) {
                    const bf16x8 q = __builtin_bit_cast(bf16x8, queries[(((p * MT + row_tile) * KK + kk) * 2 + half) * 64 + ln]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) sc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(key[i], q, sc[i], 0, 0, 0);
                }
            }
        }
    }
    between();
    const bool has = sh.id[4 * rel + c] >= 0;
    const float k_scale = sh.k_scale[4 * rel + c], v_scale = sh.v_scale[4 * rel + c];
    // which tokens the rows see: all of a tile but at the ends
    const bool whole = __builtin_amdgcn_readfirstlane(pos >= sh.lo_most && pos + kAttnTile <= sh.hi_least && __ballot(!has) == 0);
    const int first = pos + 16 * c;
    float x[16], top = -INFINITY;
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = sc[i >> 2][i & 3] * k_scale;
    if (!whole) {
        const int vhi = sh.vhi;
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = has && first + i >= lo && first + i < hi && first + i < vhi ? x[i] : -INFINITY;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) top = fmaxf(top, x[i]);
    top = fmaxf(top, __shfl_xor(top, 16, kWave));
    top = fmaxf(top, __shfl_xor(top, 32, kWave));
    if (__ballot(top > to.m)) {
        const float was = to.m;
        to.m = fmaxf(was, top);
        const float f = was > -INFINITY ? __builtin_amdgcn_exp2f(was - to.m) : 0.f;
        to.l *= f;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) to.acc[dt] *= f;
    }
    const float base = to.m > -INFINITY ? to.m : 0.f;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        x[i] = __builtin_amdgcn_exp2f(x[i] - base);
        sum += x[i];
        x[i] *= v_scale;
    }
    to.l += sum;
    uint4 prob[2][NP];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = x[8 * half + i];
        planes_of<NP>(y, prob[half]);
    }
    if (whole) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
            if (EXACT || dt < pieces) {
                const uint4 w = v(dt);
                const bf16x8 v0 = codes_to_operand(w.x, w.y), v1 = codes_to_operand(w.z, w.w);
#pragma unroll
                for (int p = 0; p < NP; ++p) {
                    to.acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, __builtin_bit_cast(bf16x8, prob[0][p]), to.acc[dt], 0, 0, 0);
                    to.acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, __builtin_bit_cast(bf16x8, prob[1][p]), to.acc[dt], 0, 0, 0);
                }
            }
        }
        return;
    }
    // values that no row sees count as 0, whatever lies there, and a NaN among the others counts for the rows that see it
    const int vlo = sh.vlo, vhi = sh.vhi;
    uint32_t keep[4];
    bf16x8 sees[2];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int t = first + i;
        const uint32_t byte = has && t >= vlo && t < vhi ? 0xffu << (8 * (i & 3)) : 0u;
        keep[i >> 2] = i & 3 ? keep[i >> 2] | byte : byte;
        sees[i >> 3][i & 7] = t >= lo && t < hi ? (__bf16)1.f : (__bf16)0.f;
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
        if (EXACT || dt < pieces) {
            uint4 w = v(dt);
            w = make_uint4(w.x & keep[0], w.y & keep[1], w.z & keep[2], w.w & keep[3]);
            const uint4 bad = make_uint4(nan_bytes(w.x), nan_bytes(w.y), nan_bytes(w.z), nan_bytes(w.w));
            if (__ballot((bad.x | bad.y | bad.z | bad.w) != 0)) {   // the code 1.0 (0x38) in the place of each NaN
                f32x4 hits = {0.f, 0.f, 0.f, 0.f};
                hits = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes_to_operand(bad.x & 0x38383838u, bad.y & 0x38383838u), sees[0], hits, 0, 0, 0);
                hits = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes_to_operand(bad.z & 0x38383838u, bad.w & 0x38383838u), sees[1], hits, 0, 0, 0);
#pragma unroll
                for (int j = 0; j < 4; ++j) to.acc[dt][j] = hits[j] > 0.f ? __builtin_nanf("") : to.acc[dt][j];
                w = make_uint4(w.x & ~bad.x, w.y & ~bad.y, w.z & ~bad.z, w.w & ~bad.w);
            }
            const bf16x8 v0 = codes_to_operand(w.x, w.y), v1 = codes_to_operand(w.z, w.w);
#pragma unroll
            for (int p = 0; p < NP; ++p) {
                to.acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, __builtin_bit_cast(bf16x8, prob[0][p]), to.acc[dt], 0, 0, 0);
                to.acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, __builtin_bit_cast(bf16x8, prob[1][p]), to.acc[dt], 0, 0, 0);
            }
        }
    }
}

// Four values of a row from d on, their sum's maximum and the sum: a result, or a chunk's part of one.
template <int TYPE>
__device__ __forceinline__ void put_row(const AttnArgs& a, const AttnPlace& p, const AttnRow& w, int d, f32x4 v, float top, float sum) {
    const bool none = sum == 0.f;
    const int64_t at = ((int64_t)w.r * a.T + w.t) * a.q_heads + w.head;
    if (p.direct) {
        if (p.split == 0) {
            const int64_t o = w.r * a.op.row + w.t * a.op.token + w.head * a.op.head + d;
#pragma unroll
            for (int i = 0; i < 4; ++i) put_value<TYPE>(a.out, o + i, none ? 0.f : v[i] / sum);
            if (d == 0 && a.lse) a.lse[at] = none ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * 0.693147181f;
        }
        if (a.parts > 1 && d == 0) a.ml[at * a.parts + a.part0 + p.split] = make_float2(-INFINITY, p.split == 0 ? -1.f : 0.f);
    } else {
        if (!none) *reinterpret_cast<f32x4*>(a.acc + (at * a.parts + a.part0 + p.split) * a.D + d) = v;
        if (d == 0) a.ml[at * a.parts + a.part0 + p.split] = make_float2(top, sum);
    }
}

template <int TYPE, int DP> constexpr int kFewLds = (4 * 16 * (DP + 4) * 4 > kPlanes<TYPE> * DP * 32 ? 4 * 16 * (DP + 4) * 4 : kPlanes<TYPE> * DP * 32);

// grid = (sentences or rows) * heads * groups * splits workgroups of four waves; D <= DP, EXACT: D == DP.
template <int TYPE, int DP, bool EXACT>
__global__ void __launch_bounds__(256, DP > 128 ? 1 : 2) k_attention_few(AttnArgs a) {
    constexpr int KK = DP / 64, DT = DP / 16, PITCH = DP + 4;
    extern __shared__ uint4 lds[];                       // queries as operands; then each wave's sums [wave, row, PITCH]
    __shared__ AttnShared sh;
    __shared__ float wave_m[4][16], wave_l[4][16];
    const int ln = lane_id(), wv = __builtin_amdgcn_readfirstlane(wave_id()), n16 = ln & 15, c = ln >> 4, pieces = a.D >> 4;
    const AttnPlace p = attn_place<16>(a, sh);
    RowSums<DP> sums;
    const bool some = p.split < p.chunks;
    if (some) stage_queries<TYPE, DP, 1>(a, sh, lds, 256);
    const int lo = sh.row[n16].lo, hi = sh.row[n16].hi;
    const int64_t head_bytes = (int64_t)a.block * a.D;
    for (int chunk = p.split; chunk < p.chunks; chunk += a.splits) {
        if (chunk != p.split) __syncthreads();
        load_chunk(a, sh, p, chunk);
        __syncthreads();
        const int rel0 = chunk * a.chunk, n = min(a.chunk, p.tiles - rel0);
        uint4 kw[KK][4], vw[DT];
        auto load_k = [&](int rel) {
            const int group = n16 >> 2, in_block = ((p.tile0 + rel0 + rel) * kAttnTile + 16 * group) & (a.block - 1);
            const uint8_t* at = a.codes_k + ((int64_t)max(sh.id[4 * rel + group], 0) * a.heads + p.h) * head_bytes + (c * a.block + in_block + (n16 & 3)) * 16;
#pragma unroll
            for (int kk = 0; kk < KK; ++kk)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if constexpr (!EXACT) kw[kk][i] = make_uint4(0, 0, 0, 0);
                    if (EXACT || c + 4 * kk < pieces) kw[kk][i] = *reinterpret_cast<const uint4*>(at + (kk * 4 * a.block + i * 4) * 16);
                }
        };
        if (wv < n) load_k(wv);
        for (int rel = wv; rel < n; rel += 4) {
            {
                const int in_block = ((p.tile0 + rel0 + rel) * kAttnTile + 16 * c) & (a.block - 1);
                const uint8_t* at = a.codes_v + ((int64_t)max(sh.id[4 * rel + c], 0) * a.heads + p.h) * head_bytes + ((in_block >> 4) * a.D + n16) * 16;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt)
                    if (EXACT || dt < pieces) vw[dt] = *reinterpret_cast<const uint4*>(at + dt * 256);
            }
            attend_tile<TYPE, DP, 1, EXACT>(a, sh, lds, 0, rel, (p.tile0 + rel0 + rel) * kAttnTile, lo, hi, sums,
                                            [&](int kk, int i) { return kw[kk][i]; }, [&](int dt) { return vw[dt]; },
                                            [&] { if (rel + 4 < n) load_k(rel + 4); });
        }
    }
    // the four waves' results together
    const bool live = sh.row[n16].lo != INT32_MIN;
    sums.l += __shfl_xor(sums.l, 16, kWave);
    sums.l += __shfl_xor(sums.l, 32, kWave);
    if (c == 0) { wave_m[wv][n16] = live ? sums.m : -INFINITY; wave_l[wv][n16] = live ? sums.l : 0.f; }
    __syncthreads();
    float* red = reinterpret_cast<float*>(lds);
    if (some) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
            if (EXACT || dt < pieces) *reinterpret_cast<f32x4*>(red + (wv * 16 + n16) * PITCH + dt * 16 + 4 * c) = sums.acc[dt];
        __syncthreads();
    }
    const int quads = a.D >> 2;
    for (int e = threadIdx.x; e < 16 * quads; e += 256) {
        const int row = e / quads, d = 4 * (e - row * quads);
        if (!sh.row[row].valid) continue;
        const float top = fmaxf(fmaxf(wave_m[0][row], wave_m[1][row]), fmaxf(wave_m[2][row], wave_m[3][row]));
        float sum = 0.f;
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float m = wave_m[w][row], l = wave_l[w][row];
            if (l == 0.f) continue;                      // (nothing, or not this row)
            const float f = m > -INFINITY ? __builtin_amdgcn_exp2f(m - top) : 1.f;   // (no maximum: nothing but NaN, which stays)
            sum += l * f;
            v += *reinterpret_cast<const f32x4*>(red + (w * 16 + row) * PITCH + d) * f;
        }
        put_row<TYPE>(a, p, sh.row[row], d, v, top, sum);
    }
}

template <int DP> constexpr int kRowsStages = DP > 128 ? 2 : 3;
template <int TYPE, int DP, int MT> constexpr int kRowsLds = kRowsStages<DP> * DP * 128 + kPlanes<TYPE> * MT * DP * 32;

// The same grid, MT waves: wave w has rows 16 w .. 16 w + 15 of the group.
template <int TYPE, int DP, int MT, bool EXACT>
__global__ void __launch_bounds__(64 * MT, 2) k_attention_rows(AttnArgs a) {
    constexpr int DT = DP / 16, STAGES = kRowsStages<DP>, TILE = 2 * DT * 64;   // uint4 of a tile: keys [kk, i, lane], values [dt, lane]
    constexpr int LOADS = (2 * DT + MT - 1) / MT;                               // of a wave for a tile, 1 KB each
    extern __shared__ uint4 lds[];
    uint4* queries = lds + STAGES * TILE;
    __shared__ AttnShared sh;
    const int ln = lane_id(), wv = __builtin_amdgcn_readfirstlane(wave_id()), n16 = ln & 15, c = ln >> 4, pieces = a.D >> 4;
    const AttnPlace p = attn_place<16 * MT>(a, sh);
    RowSums<DP> sums;
    if (p.split < p.chunks) stage_queries<TYPE, DP, MT>(a, sh, queries, 64 * MT);
    const AttnRow row = sh.row[16 * wv + n16];
    const int64_t head_bytes = (int64_t)a.block * a.D;
    for (int chunk = p.split; chunk < p.chunks; chunk += a.splits) {
        if (chunk != p.split) __syncthreads();
        load_chunk(a, sh, p, chunk);
        __syncthreads();
        const int rel0 = chunk * a.chunk, n = min(a.chunk, p.tiles - rel0);
        // every wave asks for LOADS kilobytes of a tile, the last of them twice where they do not come out even
        auto ask = [&](int rel) {
            const int group = n16 >> 2, base = (p.tile0 + rel0 + rel) * kAttnTile;
            const int in_k = (base + 16 * group) & (a.block - 1), in_v = (base + 16 * c) & (a.block - 1);
            const uint8_t* at_k = a.codes_k + ((int64_t)max(sh.id[4 * rel + group], 0) * a.heads + p.h) * head_bytes + (in_k + (n16 & 3)) * 16;
            const uint8_t* at_v = a.codes_v + ((int64_t)max(sh.id[4 * rel + c], 0) * a.heads + p.h) * head_bytes + ((in_v >> 4) * a.D + n16) * 16;
            uint4* stage = lds + (rel % STAGES) * TILE;
#pragma unroll
            for (int j = 0; j < LOADS; ++j) {
                const int load = min(wv + j * MT, 2 * DT - 1);
                if (load < DT) {   // (pieces that a head does not have: the last that it has)
                    const int kk = load >> 2, i = load & 3, piece = EXACT ? c + 4 * kk : min(c + 4 * kk, pieces - 1);
                    load_to_lds16(at_k + (piece * a.block + i * 4) * 16, stage + load * 64);
                } else {
                    const int dt = EXACT ? load - DT : min(load - DT, pieces - 1);
                    load_to_lds16(at_v + dt * 256, stage + load * 64);
                }
            }
        };
        wait_vmem<0>();   // (what was asked for before is not counted below)
#pragma unroll
        for (int i = 0; i < STAGES - 1; ++i)
            if (i < n) ask(i);
        for (int rel = 0; rel < n; ++rel) {
            if (STAGES > 2 && rel + 1 < n) wait_vmem<LOADS>();
            else wait_vmem<0>();
            lds_barrier();
            if (rel + STAGES - 1 < n) ask(rel + STAGES - 1);
            const uint4* stage = lds + (rel % STAGES) * TILE;
            attend_tile<TYPE, DP, MT, EXACT>(a, sh, queries, wv, rel, (p.tile0 + rel0 + rel) * kAttnTile, row.lo, row.hi, sums,
                                             [&](int kk, int i) {
                                                 const uint4 w = stage[(kk * 4 + i) * 64 + ln];
                                                 return EXACT || c + 4 * kk < pieces ? w : make_uint4(0, 0, 0, 0);
                                             },
                                             [&](int dt) { return stage[(DT + dt) * 64 + ln]; }, [] {});
        }
    }
    if (!row.valid) return;
    const bool live = row.lo != INT32_MIN;
    sums.l += __shfl_xor(sums.l, 16, kWave);
    sums.l += __shfl_xor(sums.l, 32, kWave);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
        if (EXACT || dt < pieces) put_row<TYPE>(a, p, row, dt * 16 + 4 * c, sums.acc[dt], live ? sums.m : -INFINITY, live ? sums.l : 0.f);
}

// A wave per row of the queries adds up its parts, in order: D / 4 lanes (up to the next power of two) take every so many-th part.
template <int TYPE>
__global__ void __launch_bounds__(256) k_attention_join(AttnArgs a) {
    const int64_t at = (int64_t)blockIdx.x * 4 + wave_id(), rt = at / a.q_heads;
    if (at >= (int64_t)a.S * a.B * a.T * a.q_heads) return;
    const int ln = lane_id(), head = (int)(at - rt * a.q_heads), r = (int)(rt / a.T), t = (int)(rt - (int64_t)r * a.T);
    if (t >= row_new(a, r)) return;
    const int per = a.D > 128 ? 64 : a.D > 64 ? 32 : 16, d = 4 * (ln & (per - 1)), side = ln / per, sides = kWave / per;
    const float2* ml = a.ml + at * a.parts;
    const float* acc = a.acc + at * a.parts * a.D + d;
    float top = -INFINITY, sum = 0.f;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    for (int i0 = 0; i0 < a.parts; i0 += kWave) {        // 64 parts' maxima and sums at a time, a lane each
        float2 p = i0 + ln < a.parts ? ml[i0 + ln] : make_float2(-INFINITY, 0.f);
        if (__ballot(p.y < 0.f)) return;                 // done already
        const float now = fmaxf(top, wave_max_f32(p.x)), was = top > -INFINITY ? __builtin_amdgcn_exp2f(top - now) : 1.f;
        top = now;
        // (never 0 for a part that is one: a NaN in it stays)
        const float f = p.y == 0.f ? 0.f : p.x > -INFINITY ? fmaxf(__builtin_amdgcn_exp2f(p.x - now), 1e-37f) : 1.f;
        sum = sum * was + wave_sum_f32(p.y * f);
        v *= was;
        const int n = min(a.parts - i0, kWave);
        for (int j = 0; j < n; j += 4 * sides) {
            f32x4 x[4];
            float g[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int part = j + q * sides + side;
                g[q] = __shfl(f, min(part, kWave - 1), kWave);
                const bool some = part < n && g[q] != 0.f && d < a.D;   // (a NaN is some)
                x[q] = f32x4{0.f, 0.f, 0.f, 0.f};
                if (some) x[q] = *reinterpret_cast<const f32x4*>(acc + (int64_t)(i0 + part) * a.D);
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const bool some = j + q * sides + side < n && g[q] != 0.f;
                v += some ? x[q] * g[q] : f32x4{0.f, 0.f, 0.f, 0.f};
            }
        }
    }
    for (int off = per; off < kWave; off <<= 1)
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] += __shfl_xor(v[i], off, kWave);
    const bool none = sum == 0.f;
    if (ln < per && d < a.D) {
        const int64_t o = r * a.op.row + t * a.op.token + head * a.op.head + d;
#pragma unroll
        for (int i = 0; i < 4; ++i) put_value<TYPE>(a.out, o + i, none ? 0.f : v[i] / sum);
    }
    if (ln == 0 && a.lse) a.lse[at] = none ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * 0.693147181f;
}

}  // namespace lshbeam
