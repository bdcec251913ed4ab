// Attention over a paged cache of 8-bit codes (lsh_cache_attention):
//   o[r, t, h] = sum_j p_j v_j,   p = softmax_j(scale * q[r, t, h] . k_j)   over the positions j of row r that token t sees.
//
// Single tokens: two operations per byte of the cache and query head, so the bytes bound it.  Everything that reads the same keys
// is therefore worked on together: the query heads of a key head, the new tokens of a row, and -- where `shared` says that a
// sentence's beams have their first blocks in common -- the beams.  Those are the columns of v_mfma_f32_16x16x32_bf16:
//   S^T [tokens, rows] = K Q^T      O^T [values, rows] += V^T P^T
// A code is exact in bf16.  Queries of 16 or 32 bits are taken apart into bf16 planes whose sum they are (bf16 1, fp16 2, fp32 3),
// and so are the probabilities, products and sums are fp32.  What the probabilities lose, and why no more is kept:
//   bf16  rounded, at most 2^-8 of each.  Many of them add up, and the result is rounded to bf16 itself: 1.2e-3 off 64 bits in the mean,
//         3e-4 off what probabilities of 32 bits give.  A second plane (16 bits) costs, 16 sentences of 12 beams over 8000 common
//         tokens, 126 us against 114, a prompt of 4096 tokens 368 against 328.
//   fp16  cut behind 16 bits: up to 2^-16 too small, where the result's own rounding is 2^-12 to 2^-11.  fp32: all 24 bits.
// log2 e is one fp32 number, 1.3e-8 of it off; rounding its product with the scale can cost 6e-8.
//
// A wave takes tiles of 64 tokens.  Row m of the K operand of sub-tile i is token 16 (m / 4) + 4 i + m % 4, so that lane (n, c) of the
// result holds, for row n of the queries, tokens 16 c + 4 i + j: the sixteen neighbours 16 c .. 16 c + 15, which are its part of the
// P^T operand as they are and lie in one block -- one scale of k and one of v for each lane.  Nothing is exchanged between lanes
// but the rows' maximum.  The cache's layout gives the operands' 16 bytes per lane in pieces of 64 (k) and 256 (v) bytes at least.
//
// k_attention_few   up to 16 rows of queries (of a row, or of all beams over what they have in common): the four waves of a workgroup
//                   take every fourth tile, straight from memory into registers (values of this tile asked for, products with its
//                   keys, keys of the next tile asked for, softmax, products with the values), and join through LDS.  Bound by
//                   memory: 64 rows of 8192, 32 heads on 8 of 128, fp16 190 us, 5.6 TB/s; 4 rows of 60 7.3 us, a chain of trips.
// k_attention_rows  17 to 64 rows (48 of fp32 in the code for heads of 256): a wave per 16 rows, all on the same tiles, which come through LDS two
//                   tiles ahead.
// k_attention_both  the common blocks' workgroups of either kind and the rows' own in one launch.
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
    int chunk;                 // tiles of a chunk at least
    int sets, groups, splits;  // sentences or rows; groups of their rows; workgroups along the tokens
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

constexpr int kAttnTile = 64;    // tokens of a wave at a time

// Eight codes as an operand.
__device__ __forceinline__ bf16x8 codes_to_operand(uint32_t a, uint32_t b) {
    const bf16x2 r0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, false), r1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, true);
    const bf16x2 r2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, false), r3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, true);
    return bf16x8{r0.x, r0.y, r1.x, r1.y, r2.x, r2.y, r3.x, r3.y};
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
    const int b = a.common ? (int)((unsigned)i / (unsigned)per) : 0, at = i - b * per;
    w.r = a.common ? s_or_r * a.B + b : s_or_r;
    w.t = (int)((unsigned)at / (unsigned)g);
    w.head = h * g + at - w.t * g;
    const int n = row_new(a, w.r);
    w.valid = w.t < n;
    seen(a, row_length(a, w.r), n, w.t, &w.lo, &w.hi);
    return w;
}

// A workgroup's place, and what is found out once for it: the same in all lanes.
struct AttnPlace {
    int split, group, h, sr;                         // sr: sentence or row
    int shared_tokens;                               // that the rows of the sentence have in common
    int vlo, vhi;                                    // positions that any row sees here
    int lo_most, hi_least;                           // ... and that all do
    int tile0, tiles, chunk, chunks;                 // of the former; tiles of a chunk
    int table_row;
    bool direct;                                     // nobody else has a part of these rows
};
__device__ __forceinline__ AttnPlace attn_place(const AttnArgs& a, unsigned u) {   // u: the workgroup's number in its launch
    AttnPlace p;
    // (heads first: workgroups go round the eight XCDs one by one, and chunks next to each other in that order -- which short rows do
    // not have -- would leave some of them idle)
    p.h = u % (unsigned)a.heads;
    u /= (unsigned)a.heads;
    p.group = u % (unsigned)a.groups;
    u /= (unsigned)a.groups;
    p.sr = u % (unsigned)a.sets;
    p.split = u / (unsigned)a.sets;
    p.shared_tokens = 0;
    if (a.has_common) p.shared_tokens = min(max(a.shared[a.common ? p.sr : p.sr / a.B], 0), a.width) * a.block;
    p.table_row = a.common ? p.sr * a.B : p.sr;
    return p;
}

constexpr int kLookup = 32;                          // tiles whose blocks are looked up at a time
struct AttnShared {
    int id[4 * kLookup];                             // block of each 16 tokens, -1: none that anybody here sees
    float k_scale[4 * kLookup], v_scale[4 * kLookup];   // times scale * log2 e; as it is
};

// The rest of the place, by every wave for itself: w is its lane's row (the rows of 64 lanes hold those of the workgroup), whose
// positions are cut to what belongs to this launch.
__device__ __forceinline__ void find_positions(const AttnArgs& a, AttnPlace& p, AttnRow& w) {
    int first = w.valid && w.lo < w.hi ? w.lo : INT32_MAX;
    w.lo = max(w.lo, a.common ? 0 : p.shared_tokens);
    w.hi = min(w.hi, a.common ? p.shared_tokens : INT32_MAX);
    const bool live = w.valid && w.lo < w.hi;
    int vlo = live ? w.lo : INT32_MAX, vhi = live ? w.hi : 0;
    // a row without a position here is worked on like the rest and left out at the end
    if (!live) { w.lo = 0; w.hi = INT32_MAX; }
    int lo_most = w.lo, hi_least = w.hi;
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
        vlo = min(vlo, __shfl_xor(vlo, off, kWave));
        vhi = max(vhi, __shfl_xor(vhi, off, kWave));
        lo_most = max(lo_most, __shfl_xor(lo_most, off, kWave));
        hi_least = min(hi_least, __shfl_xor(hi_least, off, kWave));
        first = min(first, __shfl_xor(first, off, kWave));
    }
    p.vlo = __builtin_amdgcn_readfirstlane(vlo);
    p.vhi = __builtin_amdgcn_readfirstlane(vhi);
    p.lo_most = __builtin_amdgcn_readfirstlane(lo_most);
    p.hi_least = __builtin_amdgcn_readfirstlane(hi_least);
    p.tile0 = p.vhi > 0 ? p.vlo / kAttnTile : 0;
    p.tiles = p.vhi > 0 ? (p.vhi + kAttnTile - 1) / kAttnTile - p.tile0 : 0;
    p.chunk = max(a.chunk, (p.tiles + a.splits - 1) / a.splits);
    p.chunks = (p.tiles + p.chunk - 1) / p.chunk;
    p.direct = a.parts == 1 || (!a.common && p.chunks <= 1 && __builtin_amdgcn_readfirstlane(first) >= p.shared_tokens);
    if (a.common) {                                  // the table of the sentence's first row with tokens
        int b0 = INT32_MAX;
        for (int b = lane_id(); b < a.B; b += kWave)
            if (b0 == INT32_MAX && a.lengths[p.sr * a.B + b] > 0) b0 = b;
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) b0 = min(b0, __shfl_xor(b0, off, kWave));
        p.table_row = p.sr * a.B + min(__builtin_amdgcn_readfirstlane(b0), a.B - 1);
    }
}

// A table entry for the 16 tokens from `pos` on, any row's if there is none.
__device__ __forceinline__ int32_t table_entry(const AttnArgs& a, int table_row, int64_t pos) {
    return a.tables[(int64_t)table_row * a.width + min(pos >> __builtin_ctz(a.block), (int64_t)a.width - 1)];
}
// Blocks and scales of n tiles (kLookup at most) from `tile` on, 16 tokens at a time: thread i the i-th of them.  `entry` is its table
// entry.  ids() puts the blocks to LDS and asks for the scales, put() puts those there: what the blocks alone are needed for can be
// asked for in between.
struct Lookup {
    float k, v;
    __device__ __forceinline__ void ids(const AttnArgs& a, AttnShared& sh, const AttnPlace& p, int64_t tile, int n, int32_t entry) {
        const int i = threadIdx.x;
        k = v = 0.f;
        if (i >= 4 * n) return;
        const int64_t pos = tile * kAttnTile + 16 * i;
        const int32_t id = pos < p.vhi && pos + 15 >= p.vlo && entry >= 0 && entry < a.n_blocks && pos < (int64_t)a.width * a.block ? entry : -1;
        const int64_t at = (int64_t)max(id, 0) * a.heads + p.h;
        sh.id[i] = id;
        if (id >= 0) { k = a.scale_k[at]; v = a.scale_v[at]; }
    }
    __device__ __forceinline__ void put(const AttnArgs& a, AttnShared& sh, int n) const {
        const int i = threadIdx.x;
        if (i >= 4 * n) return;
        sh.k_scale[i] = k * (a.scale * 1.44269504f);
        sh.v_scale[i] = v;
    }
};

// Queries: asked for (whatever the row's tokens: they are there), then put to LDS as operands [plane, row tile, kk, half, lane].
template <int TYPE, int DP, int MT, int THREADS> struct Queries {
    using T = typename WordOf<TYPE>::type;
    static constexpr int NP = kPlanes<TYPE>, KK = DP / 64, ALL = 16 * MT * (DP / 8), OWN = (ALL + THREADS - 1) / THREADS;
    struct Eight { uint32_t w[TYPE == kTypeF32 ? 8 : 4]; };
    Eight x[OWN];
    __device__ __forceinline__ void ask(const AttnArgs& a, const AttnPlace& p) {
        const int g = a.q_heads / a.heads, per = a.T * g, rows = a.common ? a.B * per : per;
#pragma unroll
        for (int j = 0; j < OWN; ++j) {
            const int e = threadIdx.x + j * THREADS, cd = e % (DP / 8), i = p.group * 16 * MT + e / (DP / 8);
            x[j] = Eight{};
            if (e >= ALL || i >= rows || 8 * cd >= a.D) continue;
            const int b = a.common ? (int)((unsigned)i / (unsigned)per) : 0, at = i - b * per, t = (int)((unsigned)at / (unsigned)g);
            const int r = a.common ? p.sr * a.B + b : p.sr;
            const T* from = static_cast<const T*>(a.q) + r * a.qp.row + t * a.qp.token + (p.h * g + at - t * g) * a.qp.head + 8 * cd;
            const Chunk16U<T> u = *reinterpret_cast<const Chunk16U<T>*>(from);
#pragma unroll
            for (int q = 0; q < 4; ++q) x[j].w[q] = u.w[q];
            if constexpr (TYPE == kTypeF32) {
                const Chunk16U<T> v = *reinterpret_cast<const Chunk16U<T>*>(from + 4);
#pragma unroll
                for (int q = 0; q < 4; ++q) x[j].w[4 + q] = v.w[q];
            }
        }
    }
    __device__ __forceinline__ void put(uint4* to) const {
#pragma unroll
        for (int j = 0; j < OWN; ++j) {
            const int e = threadIdx.x + j * THREADS, cd = e % (DP / 8), row = e / (DP / 8);
            if (e >= ALL) continue;
            float f[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                if constexpr (TYPE == kTypeF32) f[q] = __uint_as_float(x[j].w[q]);
                else f[q] = word_f32<TYPE>((T)(x[j].w[q >> 1] >> (16 * (q & 1)) & 0xffffu));
            }
            uint4 planes[NP];
            planes_of<NP>(f, planes);
            const int piece = cd >> 1, kk = piece >> 2, lane = (piece & 3) * 16 + (row & 15);
#pragma unroll
            for (int p = 0; p < NP; ++p) to[(((p * MT + (row >> 4)) * KK + kk) * 2 + (cd & 1)) * 64 + lane] = planes[p];
        }
    }
};

// A wave's sums for 16 rows: lane (n, c) has values 16 dt + 4 c + j of row n, its maximum, and of its sum what its tokens give.
template <int DP> struct RowSums {
    float m = -INFINITY, l = 0.f;
    f32x4 acc[DP / 16];
    __device__ __forceinline__ RowSums() {
#pragma unroll
        for (int dt = 0; dt < DP / 16; ++dt) acc[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
};

// One tile: products of the queries (q(plane, kk, half): an operand) with the keys (k(kk, i): 16 codes of a token), then `between()`,
// softmax, products with the values (v(dt): a value's codes of 16 tokens).  rel: the tile's number among those looked up, pos its
// first token.
template <int TYPE, int DP, bool EXACT, typename Q, typename K, typename V, typename F>
__device__ __forceinline__ void attend_tile(const AttnArgs& a, const AttnPlace& p, const AttnShared& sh, int rel, int pos,
                                            int lo, int hi, RowSums<DP>& to, Q q, K k, V v, F between) {
    constexpr int NP = kPlanes<TYPE>, KK = DP / 64, DT = DP / 16;
    const int c = lane_id() >> 4, pieces = a.D >> 4;
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
                for (int pl = 0; pl < NP; ++pl) {
                    const bf16x8 query = __builtin_bit_cast(bf16x8, q(pl, kk, half));
#pragma unroll
                    for (int i = 0; i < 4; ++i) sc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(key[i], query, sc[i], 0, 0, 0);
                }
                if constexpr (DP > 64) __builtin_amdgcn_sched_barrier(0);   // (or all codes are widened before they are used, and the registers do not last)
            }
        }
    }
    between();
    const bool has = sh.id[4 * rel + c] >= 0;
    const float k_scale = sh.k_scale[4 * rel + c];
    float v_scale = sh.v_scale[4 * rel + c];
    // which tokens the rows see: all of a tile but at the ends
    const bool whole = __builtin_amdgcn_readfirstlane(pos >= p.lo_most && pos + kAttnTile <= p.hi_least && __ballot(!has) == 0);
    const int first = pos + 16 * c;
    float x[16], top = -INFINITY;
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = sc[i >> 2][i & 3] * k_scale;
    if (!whole) {   // the row sees tokens from .. end - 1 of the lane's
        const int from = max(lo - first, 0), end = has ? min(hi, p.vhi) - first : 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = i >= from && i < end ? x[i] : -INFINITY;
        if (from >= min(end, 16)) v_scale = 0.f;   // (none of them: 0 times a scale that is not finite would be NaN)
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
    if constexpr (DP > 64) __builtin_amdgcn_sched_barrier(0);
    if (whole) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
            if (EXACT || dt < pieces) {
                const uint4 both = v(dt);
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const bf16x8 value = half ? codes_to_operand(both.z, both.w) : codes_to_operand(both.x, both.y);
#pragma unroll
                    for (int pl = 0; pl < NP; ++pl)
                        to.acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(value, __builtin_bit_cast(bf16x8, prob[half][pl]), to.acc[dt], 0, 0, 0);
                }
                if constexpr (DP > 64) { if (dt & 1) __builtin_amdgcn_sched_barrier(0); }
            }
        }
        return;
    }
    // values that no row sees count as 0, whatever lies there, and a NaN among the others counts for the rows that see it
    uint32_t keep[2][2];
    bf16x8 sees[2];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const uint32_t byte = has && first + i >= p.vlo && first + i < p.vhi ? 0xffu << (8 * (i & 3)) : 0u;
        uint32_t& at = keep[i >> 3][i >> 2 & 1];
        at = i & 3 ? at | byte : byte;
        sees[i >> 3][i & 7] = first + i >= lo && first + i < hi ? (__bf16)1.f : (__bf16)0.f;
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
        if (EXACT || dt < pieces) {
            const uint4 both = v(dt);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                uint2 w = half ? make_uint2(both.z, both.w) : make_uint2(both.x, both.y);
                w = make_uint2(w.x & keep[half][0], w.y & keep[half][1]);
                const uint2 bad = make_uint2(nan_bytes(w.x), nan_bytes(w.y));
                if (__ballot((bad.x | bad.y) != 0)) {   // the code 1.0 (0x38) in the place of each NaN
                    f32x4 hits = {0.f, 0.f, 0.f, 0.f};
                    hits = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes_to_operand(bad.x & 0x38383838u, bad.y & 0x38383838u), sees[half], hits, 0, 0, 0);
#pragma unroll
                    for (int j = 0; j < 4; ++j) to.acc[dt][j] = hits[j] > 0.f ? __builtin_nanf("") : to.acc[dt][j];
                    w = make_uint2(w.x & ~bad.x, w.y & ~bad.y);
                }
                const bf16x8 value = codes_to_operand(w.x, w.y);
#pragma unroll
                for (int pl = 0; pl < NP; ++pl)
                    to.acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(value, __builtin_bit_cast(bf16x8, prob[half][pl]), to.acc[dt], 0, 0, 0);
            }
        }
        if constexpr (DP > 64) { if (dt & 1) __builtin_amdgcn_sched_barrier(0); }
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

template <int TYPE, int DP, int MT> constexpr int kQueriesLds = kPlanes<TYPE> * MT * DP * 32;
template <int DP, int SUMS> constexpr int kSumsLds = SUMS * 16 * (DP + 4) * 4;
constexpr int larger(int a, int b) { return a > b ? a : b; }
constexpr int kCuLds = 160 * 1024;   // what a workgroup can have, of its own and asked for at launch together

template <int TYPE, int DP> constexpr int kFewLds = larger(kQueriesLds<TYPE, DP, 1>, kSumsLds<DP, 4>);

struct FewShared {
    AttnShared sh;
    AttnRow row[16];
    float wave_m[4][16], wave_l[4][16];
};
// heads * groups * sets * splits workgroups of four waves; D <= DP, EXACT: D == DP.  lds: queries as operands, then each wave's sums
// [wave, row, PITCH].
template <int TYPE, int DP, bool EXACT>
__device__ __forceinline__ void attend_few(const AttnArgs& a, unsigned unit, uint4* lds, FewShared& few) {
    constexpr int KK = DP / 64, DT = DP / 16, PITCH = DP + 4;
    AttnShared& sh = few.sh;
    auto& wave_m = few.wave_m;
    auto& wave_l = few.wave_l;
    const int ln = lane_id(), wv = __builtin_amdgcn_readfirstlane(wave_id()), n16 = ln & 15, c = ln >> 4, pieces = a.D >> 4;
    AttnPlace p = attn_place(a, unit);
    Queries<TYPE, DP, 1, 256> queries;
    queries.ask(a, p);
    // without a window the first tile is known before the lengths are
    const int64_t tile_guess = p.shared_tokens / kAttnTile * (a.common ? 0 : 1) + (int64_t)p.split * a.chunk;
    const int table_guess = p.table_row;
    int32_t entry = table_entry(a, p.table_row, tile_guess * kAttnTile + 16 * threadIdx.x);
    AttnRow row = attn_row(a, p.sr, p.h, p.group * 16 + n16);
    find_positions(a, p, row);
    if (threadIdx.x < 16) few.row[threadIdx.x] = row;
    const int lo = row.lo, hi = row.hi;
    RowSums<DP> sums;
    const bool some = p.split < p.chunks;
    if (some) queries.put(lds);
    const int64_t head_bytes = (int64_t)a.block * a.D;
    const int last = min(p.tiles, (p.split + 1) * p.chunk);
    for (int rel0 = p.split * p.chunk; rel0 < last; rel0 += kLookup) {
        const int n = min(kLookup, last - rel0);
        if (rel0 != p.split * p.chunk) __syncthreads();
        if (p.tile0 + rel0 != tile_guess || p.table_row != table_guess)
            entry = table_entry(a, p.table_row, ((int64_t)p.tile0 + rel0) * kAttnTile + 16 * threadIdx.x);
        Lookup lookup;
        lookup.ids(a, sh, p, (int64_t)p.tile0 + rel0, n, entry);
        lds_barrier();                                   // (the scales are on their way)
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
        lookup.put(a, sh, n);
        lds_barrier();
        for (int rel = wv; rel < n; rel += 4) {
            {
                const int in_block = ((p.tile0 + rel0 + rel) * kAttnTile + 16 * c) & (a.block - 1);
                const uint8_t* at = a.codes_v + ((int64_t)max(sh.id[4 * rel + c], 0) * a.heads + p.h) * head_bytes + ((in_block >> 4) * a.D + n16) * 16;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt)
                    if (EXACT || dt < pieces) vw[dt] = *reinterpret_cast<const uint4*>(at + dt * 256);
            }
            attend_tile<TYPE, DP, EXACT>(a, p, sh, rel, (p.tile0 + rel0 + rel) * kAttnTile, lo, hi, sums,
                                            [&](int pl, int kk, int half) { return lds[((pl * KK + kk) * 2 + half) * 64 + ln]; },
                                            [&](int kk, int i) { return kw[kk][i]; },
                                            [&](int dt) { return vw[dt]; },
                                            [&] { if (rel + 4 < n) load_k(rel + 4); });
        }
    }
    // the four waves' results together
    const bool live = hi != INT32_MAX;
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
        const int at = (int)((unsigned)e / (unsigned)quads), d = 4 * (e - at * quads);
        if (!few.row[at].valid) continue;
        const float top = fmaxf(fmaxf(wave_m[0][at], wave_m[1][at]), fmaxf(wave_m[2][at], wave_m[3][at]));
        float sum = 0.f;
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float m = wave_m[w][at], l = wave_l[w][at];
            if (l == 0.f) continue;                      // (nothing, or not this row)
            const float f = m > -INFINITY ? __builtin_amdgcn_exp2f(m - top) : 1.f;   // (no maximum: nothing but NaN, which stays)
            sum += l * f;
            v += *reinterpret_cast<const f32x4*>(red + (w * 16 + at) * PITCH + d) * f;
        }
        put_row<TYPE>(a, p, few.row[at], d, v, top, sum);
    }
}
// Two waves on a SIMD at least, with 256 registers each; with heads of 256, and of 192 with fp32 queries, what would not fit costs more
// than the second wave gives.  64 rows of 4096, 32 heads on 8 of 192, two waves against one: bf16 161 us against 173, fp16 177 against 176,
// fp32 241 against 186; 378 rows of 14 tokens, bf16 24 against 39, fp16 27 against 41.
template <int TYPE, int DP> constexpr int kFewWaves = DP > 192 || (DP > 128 && TYPE == kTypeF32) ? 1 : 2;
template <int TYPE, int DP, bool EXACT>
__global__ void __launch_bounds__(256, (kFewWaves<TYPE, DP>)) k_attention_few(AttnArgs a) {
    static_assert(kFewLds<TYPE, DP> + sizeof(FewShared) <= kCuLds, "LDS of a CU");
    extern __shared__ uint4 lds[];
    __shared__ FewShared few;
    attend_few<TYPE, DP, EXACT>(a, blockIdx.x, lds, few);
}

template <int DP> constexpr int kRowsStages = DP > 128 ? 2 : 3;
template <int TYPE, int DP, int MT> constexpr int kRowsLds = kRowsStages<DP> * DP * 128 + kQueriesLds<TYPE, DP, MT>;
// Waves that it can have: four, but three where two tiles of 256 values and 64 rows of fp32 queries (three planes: 160 KB) are all LDS there is.
template <int TYPE, int DP> constexpr int kRowsMost = kRowsLds<TYPE, DP, 4> + (int)sizeof(AttnShared) <= kCuLds ? 4 : 3;

// The same grid, MT waves: wave w has rows 16 w .. 16 w + 15 of the group.  Bound by how many workgroups a CU holds and by what each of
// them does one thing after the other (about 1.3 us a tile): 16 sentences of 12 beams over 8000 common tokens of 8 heads, D = 128, bf16, 264 MB
// in 80 us as a launch of its own.  Of the time of its waves half is waiting (for tiles and at barriers), a quarter vector instructions, a
// hundredth waiting for LDS.  Measured against those 80 and not kept: two waves per 16 rows, each for half the tokens (108); queries in
// registers and a third workgroup on a CU (81); all rows in each wave and tiles in registers as above (some 500 registers, which do not last).
template <int TYPE, int DP, int MT, bool EXACT>
__device__ __forceinline__ void attend_rows(const AttnArgs& a, unsigned unit, uint4* lds, AttnShared& sh) {
    constexpr int KK = DP / 64, DT = DP / 16, STAGES = kRowsStages<DP>, TILE = 2 * DT * 64;   // uint4 of a tile: keys [kk, i, lane], values [dt, lane]
    constexpr int LOADS = (2 * DT + MT - 1) / MT;                                             // of a wave for a tile, 1 KB each
    uint4* queries = lds + STAGES * TILE;                // (lds: tiles [stage, TILE], queries as operands)
    const int ln = lane_id(), wv = __builtin_amdgcn_readfirstlane(wave_id()), n16 = ln & 15, c = ln >> 4, pieces = a.D >> 4;
    AttnPlace p = attn_place(a, unit);
    RowSums<DP> sums;
    const int64_t tile_guess = p.shared_tokens / kAttnTile * (a.common ? 0 : 1) + (int64_t)p.split * a.chunk;
    const int table_guess = p.table_row;
    int32_t entry;
    AttnRow row;
    {
        Queries<TYPE, DP, MT, 64 * MT> q;
        q.ask(a, p);
        entry = table_entry(a, p.table_row, tile_guess * kAttnTile + 16 * threadIdx.x);
        row = attn_row(a, p.sr, p.h, ln < 16 * MT ? p.group * 16 * MT + ln : INT32_MAX);
        find_positions(a, p, row);
        const int from = 16 * wv + n16;                  // the lane's own row of those
        row.r = __shfl(row.r, from, kWave);
        row.t = __shfl(row.t, from, kWave);
        row.head = __shfl(row.head, from, kWave);
        row.lo = __shfl(row.lo, from, kWave);
        row.hi = __shfl(row.hi, from, kWave);
        row.valid = __shfl((int)row.valid, from, kWave) != 0;
        if (p.split < p.chunks) q.put(queries);
    }
    const int64_t head_bytes = (int64_t)a.block * a.D;
    const int last = min(p.tiles, (p.split + 1) * p.chunk);
    for (int rel0 = p.split * p.chunk; rel0 < last; rel0 += kLookup) {
        const int n = min(kLookup, last - rel0);
        if (rel0 != p.split * p.chunk) __syncthreads();
        if (p.tile0 + rel0 != tile_guess || p.table_row != table_guess)
            entry = table_entry(a, p.table_row, ((int64_t)p.tile0 + rel0) * kAttnTile + 16 * threadIdx.x);
        Lookup lookup;
        lookup.ids(a, sh, p, (int64_t)p.tile0 + rel0, n, entry);
        lookup.put(a, sh, n);
        __syncthreads();
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
            attend_tile<TYPE, DP, EXACT>(a, p, sh, rel, (p.tile0 + rel0 + rel) * kAttnTile, row.lo, row.hi, sums,
                                         [&](int pl, int kk, int half) { return queries[(((pl * MT + wv) * KK + kk) * 2 + half) * 64 + ln]; },
                                         [&](int kk, int i) {
                                             const uint4 w = stage[(kk * 4 + i) * 64 + ln];
                                             return EXACT || c + 4 * kk < pieces ? w : make_uint4(0, 0, 0, 0);
                                         },
                                         [&](int dt) { return stage[(DT + dt) * 64 + ln]; }, [] {});
        }
    }
    if (!row.valid) return;
    const bool live = row.hi != INT32_MAX;
    float l = sums.l;
    l += __shfl_xor(l, 16, kWave);
    l += __shfl_xor(l, 32, kWave);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
        if (EXACT || dt < pieces) put_row<TYPE>(a, p, row, dt * 16 + 4 * c, sums.acc[dt], live ? sums.m : -INFINITY, live ? l : 0.f);
}
template <int TYPE, int DP, int MT, bool EXACT>
__global__ void __launch_bounds__(64 * MT, 2) k_attention_rows(AttnArgs a) {
    static_assert(kRowsLds<TYPE, DP, MT> + sizeof(AttnShared) <= kCuLds, "LDS of a CU");
    extern __shared__ uint4 lds[];
    __shared__ AttnShared sh;
    attend_rows<TYPE, DP, MT, EXACT>(a, blockIdx.x, lds, sh);
}

// 4 sentences of 12 beams over 8192 common tokens, 32 heads on 8 of 128, bf16: 37 us a call, 40 as two launches (26 and 10); 16 sentences of 12
// beams, 8000 of 8192 tokens common, 338 MB: 104 us, the join 9.
// What a sentence's beams have in common (the first `units` workgroups; MT: waves of each, 1: all four with at most 16 rows) and each
// row's own part in one launch: neither waits for the other.  The waves behind the MT-th end at once, and a barrier does not wait for
// waves that have ended.
template <int TYPE, int DP, int MT> constexpr int kBothLds = MT == 1 ? kFewLds<TYPE, DP> : larger(kRowsLds<TYPE, DP, MT>, kFewLds<TYPE, DP>);
struct BothArgs { AttnArgs common, own; unsigned units; };
template <int TYPE, int DP, int MT, bool EXACT>
__global__ void __launch_bounds__(256, 2) k_attention_both(BothArgs b) {
    static_assert(kBothLds<TYPE, DP, MT> + sizeof(FewShared) <= kCuLds, "LDS of a CU");
    extern __shared__ uint4 lds[];
    __shared__ FewShared few;
    if (blockIdx.x >= b.units) return attend_few<TYPE, DP, EXACT>(b.own, blockIdx.x - b.units, lds, few);
    if constexpr (MT == 1) attend_few<TYPE, DP, EXACT>(b.common, blockIdx.x, lds, few);
    else if (__builtin_amdgcn_readfirstlane(wave_id()) < MT) attend_rows<TYPE, DP, MT, EXACT>(b.common, blockIdx.x, lds, few.sh);
}

// Bound by latency: 5 to 6 us for 1500 to 2000 rows of some parts each.  A wave per row of the queries adds up its parts, in order: D / 4 lanes (up to the next power of two) take every so many-th part.
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
        for (int j = 0; j < n; j += 8 * sides) {
            f32x4 x[8];
            float g[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const int part = j + q * sides + side;
                g[q] = __shfl(f, min(part, kWave - 1), kWave);
                const bool some = part < n && g[q] != 0.f && d < a.D;   // (a NaN is some)
                x[q] = f32x4{0.f, 0.f, 0.f, 0.f};
                if (some) x[q] = *reinterpret_cast<const f32x4*>(acc + (int64_t)(i0 + part) * a.D);
            }
#pragma unroll
            for (int q = 0; q < 8; ++q) {
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
