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
// Order of a wave's work: values of this tile asked for, products with its keys, keys of the next tile asked for, softmax, products
// with the values: 8 to 16 KB under way all the time at D = 128, block numbers one tile earlier still.
//
// The rows of a row set are split along the tokens into chunks; a chunk is a workgroup's, its tiles go round its four waves, which
// join through LDS.  Chunks leave (max, sum, products) in the workspace, k_attention_join adds them up in order.
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
    int chunk;                 // tiles of a chunk
    int rows;                  // rows of a workgroup: 16 times its MT
    int common_groups, common_splits, common_units;   // beams together: groups of rows, workgroups along the tokens, workgroups in all
    int own_groups, own_splits;                       // each row by itself
    int parts;                 // common_splits + own_splits; 1: results are written at once
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
__device__ __forceinline__ AttnRow attn_row(const AttnArgs& a, bool common, int s_or_r, int h, int i) {
    const int g = a.q_heads / a.heads, per = a.T * g;
    AttnRow w{0, 0, 0, 0, 0, false};
    if (i >= (common ? a.B * per : per)) return w;
    const int b = common ? i / per : 0, at = i - b * per;
    w.r = common ? s_or_r * a.B + b : s_or_r;
    w.t = at / g;
    w.head = h * g + at - w.t * g;
    const int n = row_new(a, w.r);
    w.valid = w.t < n;
    if (w.valid) seen(a, row_length(a, w.r), n, w.t, &w.lo, &w.hi);
    return w;
}
// Tokens that the rows of sentence s have in common.
__device__ __forceinline__ int common_tokens(const AttnArgs& a, int s) {
    return a.common_splits > 0 ? min(max(a.shared[s], 0), a.width) * a.block : 0;
}

__device__ __forceinline__ int row16_all_min(int v) { return __builtin_amdgcn_readfirstlane(row16_min_i32(v)); }

// grid = common_units + R * heads * own_groups * own_splits workgroups of four waves; D <= DP, EXACT: D == DP.
template <int TYPE, int DP, int MT, bool EXACT>
__global__ void __launch_bounds__(256, DP * MT > 256 ? 1 : 2) k_attention_tiles(AttnArgs a) {
    constexpr int NP = kPlanes<TYPE>, KK = DP / 64, DT = DP / 16, ROWS = 16 * MT, PITCH = DP + 4;
    constexpr int QS = NP * MT * KK * 2 * 64, RED = ROWS * PITCH / 4;
    __shared__ uint4 lds[QS > RED ? QS : RED];          // queries as operands [plane, mt, kk, half, lane]; then the rows' sums [row, PITCH]
    __shared__ float wave_m[4][ROWS], wave_l[4][ROWS];
    const int ln = lane_id(), wv = __builtin_amdgcn_readfirstlane(wave_id()), n16 = ln & 15, c = ln >> 4;
    const bool common = (int)blockIdx.x < a.common_units;
    int u = common ? blockIdx.x : blockIdx.x - a.common_units;
    const int splits = common ? a.common_splits : a.own_splits, groups = common ? a.common_groups : a.own_groups;
    const int split = u % splits;
    u /= splits;
    const int group = u % groups;
    u /= groups;
    const int h = u % a.heads, sr = u / a.heads;        // sentence or row
    const int s = common ? sr : sr / a.B;
    const int shared_tokens = common_tokens(a, s);
    const int from = common ? 0 : shared_tokens, to = common ? shared_tokens : INT32_MAX;

    // the rows' positions here; a row without any is worked on like the rest and left out at the end
    int lo[MT], hi[MT];
    bool live[MT];
    int vlo = INT32_MAX, vhi_neg = 0, lo_most = INT32_MIN, hi_least = INT32_MAX, common_lo = INT32_MAX;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const AttnRow w = attn_row(a, common, sr, h, group * ROWS + mt * 16 + n16);
        const int l = max(w.lo, from), e = min(w.hi, to);
        live[mt] = w.valid && l < e;
        lo[mt] = live[mt] ? l : INT32_MIN;
        hi[mt] = live[mt] ? e : INT32_MAX;
        if (live[mt]) { vlo = min(vlo, l); vhi_neg = min(vhi_neg, -e); }
        if (w.valid && w.lo < w.hi) common_lo = min(common_lo, w.lo);
        lo_most = max(lo_most, lo[mt]);
        hi_least = min(hi_least, hi[mt]);
    }
    vlo = row16_all_min(vlo);
    const int vhi = -row16_all_min(vhi_neg);
    lo_most = lo_most == INT32_MIN ? INT32_MIN + 1 : lo_most;
    lo_most = -row16_all_min(-lo_most);
    hi_least = row16_all_min(hi_least);
    common_lo = row16_all_min(common_lo);
    const int row_tiles = min(MT, ((common ? a.B : 1) * a.T * (a.q_heads / a.heads) - group * ROWS + 15) >> 4);   // those that hold rows
    const int tile0 = vhi > 0 ? vlo / kAttnTile : 0, tiles = vhi > 0 ? (vhi + kAttnTile - 1) / kAttnTile - tile0 : 0;
    const int chunks = (tiles + a.chunk - 1) / a.chunk;
    const bool direct = a.parts == 1 || (!common && chunks <= 1 && common_lo >= shared_tokens);   // nobody else has a part of these rows
    float m[MT], l[MT];
    f32x4 acc[MT][DT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        m[mt] = -INFINITY;
        l[mt] = 0.f;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) acc[mt][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    if (split < chunks) {
        // queries to LDS, as operands
        for (int e = threadIdx.x; e < ROWS * (DP / 8); e += 256) {
            const int cd = e % (DP / 8), row = e / (DP / 8);
            const AttnRow w = attn_row(a, common, sr, h, group * ROWS + row);
            float x[8];
            const int64_t at = w.r * a.qp.row + w.t * a.qp.token + w.head * a.qp.head + 8 * cd;
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = w.valid && 8 * cd < a.D ? value_at<TYPE>(a.q, at + i) : 0.f;
            uint4 planes[NP];
            planes_of<NP>(x, planes);
            const int piece = cd >> 1, kk = piece >> 2, lane = (piece & 3) * 16 + (row & 15);
#pragma unroll
            for (int p = 0; p < NP; ++p) lds[(((p * MT + (row >> 4)) * KK + kk) * 2 + (cd & 1)) * 64 + lane] = planes[p];
        }
        int table_row = sr;
        if (common) {                                   // the sentence's first row with tokens
            int first = INT32_MAX;
            for (int b = ln; b < a.B; b += kWave) if (a.lengths[sr * a.B + b] > 0) first = min(first, b);
#pragma unroll
            for (int off = 32; off > 0; off >>= 1) first = min(first, __shfl_xor(first, off, kWave));
            table_row = sr * a.B + min(__builtin_amdgcn_readfirstlane(first), a.B - 1);
        }
        const int32_t* table = a.tables + (int64_t)table_row * a.width;
        __syncthreads();

        const int block_bits = __builtin_ctz(a.block), pieces = a.D >> 4;
        const int64_t head_bytes = (int64_t)a.block * a.D;
        // block of the 16 tokens from `pos` on, -1: none that anybody here sees
        auto block_at = [&](int pos) -> int32_t {
            if (pos >= vhi || pos + 15 < vlo || (pos >> block_bits) >= a.width) return -1;
            const int32_t id = table[pos >> block_bits];
            return id < a.n_blocks ? id : -1;
        };
        const int group_k = n16 >> 2;
        struct Tile { int index; int32_t id_k, id_v; };
        // the wave's tiles: tile k of its chunks split, split + splits, ...
        const int per_chunk = a.chunk >> 2;             // a multiple of 4 tiles a chunk: as many for each wave
        const int n_mine = ((chunks - split + splits - 1) / splits) * per_chunk;
        auto tile_at = [&](int k) -> Tile {
            Tile t;
            const int chunk = split + (k / per_chunk) * splits;
            const int rel = chunk * a.chunk + (k % per_chunk) * 4 + wv;
            t.index = k < n_mine && rel < tiles ? tile0 + rel : -1;
            const int pos = t.index < 0 ? INT32_MAX - 1024 : t.index * kAttnTile;
            t.id_k = block_at(pos + 16 * group_k);
            t.id_v = block_at(pos + 16 * c);
            return t;
        };
        uint4 kw[KK][4], vw[DT];
        auto load_k = [&](const Tile& t) {
            const int in_block = (t.index * kAttnTile + 16 * group_k) & (a.block - 1);
            const uint8_t* p = a.codes_k + ((int64_t)max(t.id_k, 0) * a.heads + h) * head_bytes + (c * a.block + in_block + (n16 & 3)) * 16;
#pragma unroll
            for (int kk = 0; kk < KK; ++kk)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if constexpr (EXACT) kw[kk][i] = *reinterpret_cast<const uint4*>(p + (kk * 4 * a.block + i * 4) * 16);
                    else {
                        kw[kk][i] = make_uint4(0, 0, 0, 0);
                        if (c + 4 * kk < pieces) kw[kk][i] = *reinterpret_cast<const uint4*>(p + (kk * 4 * a.block + i * 4) * 16);
                    }
                }
        };
        auto load_v = [&](const Tile& t) {
            const int in_block = (t.index * kAttnTile + 16 * c) & (a.block - 1);
            const uint8_t* p = a.codes_v + ((int64_t)max(t.id_v, 0) * a.heads + h) * head_bytes + ((in_block >> 4) * a.D + n16) * 16;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
                if (EXACT || dt < pieces) vw[dt] = *reinterpret_cast<const uint4*>(p + dt * 256);
        };
        const float to_log2 = a.scale * 1.44269504f;
        Tile now = tile_at(0), next = tile_at(1);
        if (now.index >= 0) load_k(now);
        for (int k = 0; k < n_mine; ++k) {
            if (now.index >= 0) {
                load_v(now);
                const int64_t scale_at = (int64_t)max(now.id_v, 0) * a.heads + h;
                const bool has = now.id_v >= 0;
                const float k_scale = has ? a.scale_k[scale_at] * to_log2 : 0.f, v_scale = has ? a.scale_v[scale_at] : 0.f;
                const Tile after = tile_at(k + 2);
                const int pos = now.index * kAttnTile;
                // products
                f32x4 sc[MT][4];
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) sc[mt][i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int kk = 0; kk < KK; ++kk) {
                    if (!EXACT && 4 * kk >= pieces) continue;
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        bf16x8 key[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            key[i] = half ? codes_to_operand(kw[kk][i].z, kw[kk][i].w) : codes_to_operand(kw[kk][i].x, kw[kk][i].y);
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt)
                          if (mt == 0 || mt < row_tiles)
#pragma unroll
                            for (int p = 0; p < NP; ++p) {
                                const bf16x8 q = __builtin_bit_cast(bf16x8, lds[(((p * MT + mt) * KK + kk) * 2 + half) * 64 + ln]);
#pragma unroll
                                for (int i = 0; i < 4; ++i) sc[mt][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(key[i], q, sc[mt][i], 0, 0, 0);
                            }
                    }
                }
                if (next.index >= 0) load_k(next);
                // which tokens the rows see: all of a tile but at the ends
                const bool whole = pos >= lo_most && pos + kAttnTile <= hi_least && __ballot(!has) == 0;
                uint4 prob[MT][NP][2];
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    if (mt > 0 && mt >= row_tiles) continue;
                    float x[16], top = -INFINITY;
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        x[i] = sc[mt][i >> 2][i & 3] * k_scale;
                        if (!whole) {
                            const int t = pos + 16 * c + i;
                            x[i] = has && t >= lo[mt] && t < hi[mt] && t < vhi ? x[i] : -INFINITY;
                        }
                        top = fmaxf(top, x[i]);
                    }
                    top = fmaxf(top, __shfl_xor(top, 16, kWave));
                    top = fmaxf(top, __shfl_xor(top, 32, kWave));
                    const float was = m[mt];
                    if (__ballot(top > was)) {
                        m[mt] = fmaxf(was, top);
                        const float f = was > -INFINITY ? __builtin_amdgcn_exp2f(was - m[mt]) : 0.f;
                        l[mt] *= f;
#pragma unroll
                        for (int dt = 0; dt < DT; ++dt) acc[mt][dt] *= f;
                    }
                    const float base = m[mt] > -INFINITY ? m[mt] : 0.f;
                    float sum = 0.f;
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        x[i] = __builtin_amdgcn_exp2f(x[i] - base);
                        sum += x[i];
                        x[i] *= v_scale;
                    }
                    l[mt] += sum;
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        float y[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) y[i] = x[8 * half + i];
                        uint4 planes[NP];
                        planes_of<NP>(y, planes);
#pragma unroll
                        for (int p = 0; p < NP; ++p) prob[mt][p][half] = planes[p];
                    }
                }
                if (!whole) {
                    // values that no row sees count as 0, whatever lies there; and a NaN among the others counts for those who see it
                    uint32_t any = 0;
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        uint32_t keep = 0;
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int t = pos + 16 * c + 4 * q + j;
                            keep |= has && t >= vlo && t < vhi ? 0xffu << (8 * j) : 0u;
                        }
#pragma unroll
                        for (int dt = 0; dt < DT; ++dt)
                            if (EXACT || dt < pieces) {
                                uint32_t& w = q == 0 ? vw[dt].x : q == 1 ? vw[dt].y : q == 2 ? vw[dt].z : vw[dt].w;
                                w &= keep;
                                any |= nan_bytes(w);
                            }
                    }
                    if (__ballot(any != 0)) {
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) {
                            bf16x8 sees[2];
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                const int t = pos + 16 * c + i;
                                sees[i >> 3][i & 7] = t >= lo[mt] && t < hi[mt] ? (__bf16)1.f : (__bf16)0.f;
                            }
#pragma unroll
                            for (int dt = 0; dt < DT; ++dt)
                                if (EXACT || dt < pieces) {   // the code 1.0 (0x38) in the place of each NaN
                                    const uint4 w = vw[dt];
                                    f32x4 hits = {0.f, 0.f, 0.f, 0.f};
                                    hits = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes_to_operand(nan_bytes(w.x) & 0x38383838u, nan_bytes(w.y) & 0x38383838u), sees[0], hits, 0, 0, 0);
                                    hits = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes_to_operand(nan_bytes(w.z) & 0x38383838u, nan_bytes(w.w) & 0x38383838u), sees[1], hits, 0, 0, 0);
#pragma unroll
                                    for (int j = 0; j < 4; ++j) acc[mt][dt][j] = hits[j] > 0.f ? __builtin_nanf("") : acc[mt][dt][j];
                                }
                        }
#pragma unroll
                        for (int dt = 0; dt < DT; ++dt)
                            if (EXACT || dt < pieces) {
                                vw[dt].x &= ~nan_bytes(vw[dt].x);
                                vw[dt].y &= ~nan_bytes(vw[dt].y);
                                vw[dt].z &= ~nan_bytes(vw[dt].z);
                                vw[dt].w &= ~nan_bytes(vw[dt].w);
                            }
                    }
                }
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    if (!EXACT && dt >= pieces) continue;
                    const bf16x8 v0 = codes_to_operand(vw[dt].x, vw[dt].y), v1 = codes_to_operand(vw[dt].z, vw[dt].w);
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt)
                      if (mt == 0 || mt < row_tiles)
#pragma unroll
                        for (int p = 0; p < NP; ++p) {
                            acc[mt][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, __builtin_bit_cast(bf16x8, prob[mt][p][0]), acc[mt][dt], 0, 0, 0);
                            acc[mt][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, __builtin_bit_cast(bf16x8, prob[mt][p][1]), acc[mt][dt], 0, 0, 0);
                        }
                }
                now = next;
                next = after;
            } else {
                now = next;                             // (a chunk's last tiles: the next chunk's may follow)
                if (now.index >= 0) load_k(now);
                next = tile_at(k + 2);
            }
        }
    }

    // the four waves' results together, in order
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        l[mt] += __shfl_xor(l[mt], 16, kWave);
        l[mt] += __shfl_xor(l[mt], 32, kWave);
        if (c == 0) { wave_m[wv][mt * 16 + n16] = live[mt] ? m[mt] : -INFINITY; wave_l[wv][mt * 16 + n16] = live[mt] ? l[mt] : 0.f; }
    }
    __syncthreads();
    float* red = reinterpret_cast<float*>(lds);
    const bool some = split < chunks;
    if (some) {
        for (int w = 0; w < 4; ++w) {
            if (wv == w) {
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    const int row = mt * 16 + n16;
                    const float top = fmaxf(fmaxf(wave_m[0][row], wave_m[1][row]), fmaxf(wave_m[2][row], wave_m[3][row]));
                    const float f = m[mt] > -INFINITY && top > -INFINITY ? __builtin_amdgcn_exp2f(m[mt] - top) : 0.f;
                    // (a row of nothing but NaN has no maximum: its sums are NaN and stay)
                    const float g = m[mt] > -INFINITY ? f : l[mt] != l[mt] ? 1.f : 0.f;
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) {
                        f32x4* at = reinterpret_cast<f32x4*>(red + row * PITCH + dt * 16 + 4 * c);
                        const f32x4 v = acc[mt][dt] * g;
                        *at = w == 0 ? v : *at + v;
                    }
                }
            }
            __syncthreads();
        }
    }
    // results, or this chunk's part of them
    const int part = common ? split : a.common_splits + split;
    const int quads = a.D >> 2;
    for (int e = threadIdx.x; e < ROWS * quads; e += 256) {
        const int row = e / quads, d = 4 * (e - row * quads);
        const AttnRow w = attn_row(a, common, sr, h, group * ROWS + row);
        if (!w.valid) continue;
        float top = -INFINITY, sum = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, wave_m[i][row]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float x = wave_l[i][row];
            sum += wave_m[i][row] > -INFINITY ? x * __builtin_amdgcn_exp2f(wave_m[i][row] - top) : x;
        }
        const bool none = sum == 0.f;
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
        if (!none && some) v = *reinterpret_cast<const f32x4*>(red + row * PITCH + d);
        const int64_t at = ((int64_t)w.r * a.T + w.t) * a.q_heads + w.head;
        if (direct) {
            if (split == 0) {
                const int64_t o = w.r * a.op.row + w.t * a.op.token + w.head * a.op.head + d;
#pragma unroll
                for (int i = 0; i < 4; ++i) put_value<TYPE>(a.out, o + i, none ? 0.f : v[i] / sum);
                if (d == 0 && a.lse) a.lse[at] = none ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * 0.693147181f;
            }
            if (a.parts > 1 && d == 0) a.ml[at * a.parts + part] = make_float2(-INFINITY, split == 0 ? -1.f : 0.f);
        } else {
            if (!none) *reinterpret_cast<f32x4*>(a.acc + (at * a.parts + part) * a.D + d) = v;
            if (d == 0) a.ml[at * a.parts + part] = make_float2(top, sum);
        }
    }
}

// A wave per row of the queries adds up its parts, in order.
template <int TYPE>
__global__ void __launch_bounds__(256) k_attention_join(AttnArgs a) {
    const int64_t at = (int64_t)blockIdx.x * 4 + wave_id(), rt = at / a.q_heads;
    if (at >= (int64_t)a.S * a.B * a.T * a.q_heads) return;
    const int ln = lane_id(), head = (int)(at - rt * a.q_heads), r = (int)(rt / a.T), t = (int)(rt - (int64_t)r * a.T);
    if (t >= row_new(a, r)) return;
    const float2* ml = a.ml + at * a.parts;
    float top = -INFINITY;
    bool done = false;
    for (int i = ln; i < a.parts; i += kWave) {
        const float2 p = ml[i];
        top = fmaxf(top, p.x);
        done |= p.y < 0.f;
    }
    if (__ballot(done)) return;
    top = wave_max_f32(top);
    float sum = 0.f;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    const int d = 4 * ln;
    for (int i = 0; i < a.parts; ++i) {
        const float2 p = ml[i];
        if (p.y == 0.f) continue;
        const float f = p.x > -INFINITY ? __builtin_amdgcn_exp2f(p.x - top) : 1.f;
        sum += p.y * f;
        if (d < a.D) v += *reinterpret_cast<const f32x4*>(a.acc + (at * a.parts + i) * a.D + d) * f;
    }
    const bool none = sum == 0.f;
    if (d < a.D) {
        const int64_t o = r * a.op.row + t * a.op.token + head * a.op.head + d;
#pragma unroll
        for (int i = 0; i < 4; ++i) put_value<TYPE>(a.out, o + i, none ? 0.f : v[i] / sum);
    }
    if (ln == 0 && a.lse) a.lse[at] = none ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * 0.693147181f;
}

}  // namespace lshbeam
