// Rows times weights of 4 bits (lsh_packed_linear, lsh_packed_gated):
//   y[m, n] = sum_k x[m, k] (code[n, k] - zero[n, g]) scale[n, g] = sum_g scale[n, g] (sum_{k in g} x[m, k] code[n, k] - zero[n, g] X[m, g])
// with X[m, g] the sum of a row's inputs of group g.  Codes 0 .. 15 are exact in bf16 and fp16, rows of fp32 are taken apart into three planes of
// bf16 that add up to them, so every product is exact and nothing but the fp32 sums rounds.
//
// Few rows: two operations a weight and row, so the weights' bytes bound it.
#pragma once
#include "packed.h"

namespace lshbeam {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

struct PackedArgs {
    int M, N, K, tiles, parts;
    int shift;                 // log2 of the group
    bool scale_f16;
    const void* x;
    int64_t ldx;
    PackedRef w[2];            // gated: gate, up
    const float* bias;
    const void* add;
    int64_t ld_add;
    void* out;
    int64_t ld_out;
    int out_type;
    int activation;
    // of the launch
    int rows;                  // of a workgroup
    int across;                // waves side by side along the outputs; the others share their inputs
    int chunk;                 // parts whose rows are in LDS at a time
    int sets;                  // groups of tiles
    int join_at;               // where in LDS waves that share inputs add up; 0: over the rows, which nothing asks for again
};

constexpr int kRowsPlanesF32 = 3;
template <int TYPE> constexpr int kRowPlanes = TYPE == kTypeF32 ? kRowsPlanesF32 : 1;
constexpr int kPackedWaves = 8;
// LDS: operands of 32 inputs: [plane][of the chunk][c][row] 16 bytes, the c's 32 bytes apart so that four neighbouring lanes write to banks
// of their own; sums of the rows' groups; what the waves that share inputs add up.
template <int MT> constexpr int kRowsOfC = 16 * MT * 16 + 32;
template <int MT> constexpr int packed_plane(int chunk) { return chunk * 4 * 4 * kRowsOfC<MT>; }
template <int MT> constexpr int packed_sums(int chunk) { return chunk * 4 * 16 * MT * 4; }

template <int TYPE> struct OperandOf { using type = bf16x8; };
template <> struct OperandOf<kTypeF16> { using type = f16x8; };

// Eight codes, as they are, as an operand.
template <int TYPE> __device__ __forceinline__ typename OperandOf<TYPE>::type codes_operand(uint32_t word) {
    const uint32_t lo = word & 0x0f0f0f0fu, hi = word >> 4 & 0x0f0f0f0fu;
    if constexpr (TYPE == kTypeF16) {
        const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 512.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 512.f, true);
        const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 512.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 512.f, true);
        return f16x8{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
    } else {
        const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 512.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 512.f, true);
        const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 512.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 512.f, true);
        return bf16x8{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
    }
}
template <int TYPE> __device__ __forceinline__ f32x4 product(uint4 x, typename OperandOf<TYPE>::type w, f32x4 acc) {
    if constexpr (TYPE == kTypeF16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, x), w, acc, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), w, acc, 0, 0, 0);
}

// Eight inputs of a row as operands.
template <int TYPE> __device__ __forceinline__ void row_operand(const float (&x)[8], uint4 (&op)[kRowPlanes<TYPE>]) {
    if constexpr (TYPE == kTypeF16) {
        uint32_t b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) b[i] = (uint32_t)__half_as_ushort(__float2half_rn(x[2 * i])) | (uint32_t)__half_as_ushort(__float2half_rn(x[2 * i + 1])) << 16;
        op[0] = make_uint4(b[0], b[1], b[2], b[3]);
    } else planes_of<kRowPlanes<TYPE>>(x, op);
}

__device__ __forceinline__ float activate(float z, int kind) {
    if (kind == 0) return z / (1.f + expf(-z));
    if (kind == 1) return z * (0.5f * erfcf(-0.70710678118654752f * z));
    // (1 + tanh t) / 2 = 1 / (1 + e^(-2 t))
    return z / (1.f + expf(-1.5957691216057308f * (z + 0.044715f * z * z * z)));
}

// A result to its place: bias, what is added, one rounding.
__device__ __forceinline__ void put_result(const PackedArgs& a, int64_t m, int64_t n, float y) {
    if (a.bias) y += a.bias[n];
    const int64_t at = m * a.ld_out + n, add = m * a.ld_add + n;
    if (a.out_type == kTypeF32) {
        if (a.add) y += value_at<kTypeF32>(a.add, add);
        put_value<kTypeF32>(a.out, at, y);
    } else if (a.out_type == kTypeBf16) {
        if (a.add) y += value_at<kTypeBf16>(a.add, add);
        put_value<kTypeBf16>(a.out, at, y);
    } else {
        if (a.add) y += value_at<kTypeF16>(a.add, add);
        put_value<kTypeF16>(a.out, at, y);
    }
}

// What a wave asks of a tile's part.
struct PackedPiece { uint4 codes; uint64_t scales; uint32_t zeros; };
__device__ __forceinline__ PackedPiece load_piece(const PackedArgs& a, const PackedRef& w, int tile, int part) {
    const int64_t unit = (int64_t)tile * a.parts + part;
    const int ln = lane_id(), n = ln & 15, each = kPackInputs >> a.shift;
    PackedPiece p;
    p.codes = *reinterpret_cast<const uint4*>(w.codes + unit * kPackBytes + 16 * ln);
    // 8 bytes of scales and 4 of zeros, of which the lane's may be the last ones: they stay inside the tile's part
    const int at = min(n * each, 16 * each - 4);
    const uint16_t* s = w.scales + unit * (16 * each) + at;
    struct __attribute__((packed, aligned(2))) Eight { uint64_t v; };
    p.scales = reinterpret_cast<const Eight*>(s)->v >> (16 * (n * each - at));
    p.zeros = 0x08080808u;
    if (w.zeros) {
        struct __attribute__((packed, aligned(1))) Four { uint32_t v; };
        p.zeros = reinterpret_cast<const Four*>(w.zeros + unit * (16 * each) + at)->v >> (8 * (n * each - at));
    }
    return p;
}

// MT: 16 rows each; NS: tiles of a wave (gated: half of them of each matrix, gate and up in turn).
template <int TYPE, int MT, int NS, bool GATED>
__global__ void __launch_bounds__(64 * kPackedWaves) k_packed_rows(PackedArgs a) {
    extern __shared__ __align__(16) char lds[];
    constexpr int NP = kRowPlanes<TYPE>, ROWS = 16 * MT, CS = kRowsOfC<MT>, NT = GATED ? NS / 2 : NS;
    const int plane = packed_plane<MT>(a.chunk);
    float* sums = reinterpret_cast<float*>(lds + NP * plane);
    f32x4* join = reinterpret_cast<f32x4*>(lds + a.join_at);
    const int wave = __builtin_amdgcn_readfirstlane(wave_id()), ln = lane_id();
    const int across = a.across, deep = kPackedWaves / across, wn = wave % across, wk = wave / across;
    const int m0 = blockIdx.y * a.rows, rows = min(a.rows, a.M - m0);
    const int per = 1 << (a.shift - 5);                     // operands of a group
    const int chunks = (a.parts + a.chunk - 1) / a.chunk;

    PackedPiece next[NS];
    auto ask = [&](int set, int part) {
        part = min(part, a.parts - 1);
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            const int tile = min((set * across + wn) * NT + (GATED ? s >> 1 : s), a.tiles - 1);
            next[s] = load_piece(a, a.w[GATED ? s & 1 : 0], tile, part);
        }
    };
    ask(blockIdx.x, wk);
    for (int set = blockIdx.x; set < a.sets; set += gridDim.x) {
        f32x4 y[MT][NS], acc[MT][NS];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int s = 0; s < NS; ++s) { y[mt][s] = f32x4{0.f, 0.f, 0.f, 0.f}; acc[mt][s] = f32x4{0.f, 0.f, 0.f, 0.f}; }
        for (int chunk = 0; chunk < chunks; ++chunk) {
            const int part0 = chunk * a.chunk, here = min(a.chunk, a.parts - part0);
            if (chunks > 1 || set == (int)blockIdx.x) {
                __syncthreads();
                for (int u = threadIdx.x; u < here * ROWS * 4; u += 64 * kPackedWaves) {
                    const int c = u & 3, m = (u >> 2) % ROWS, p = (u >> 2) / ROWS;
                    if (m >= rows) continue;
                    float group = 0.f;
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const int k = (part0 + p) * kPackInputs + 32 * w + 8 * c;
                        const int64_t from = (int64_t)(m0 + m) * a.ldx + k;
                        float x[8];
                        if (k + 8 <= a.K) load_values<TYPE>(a.x, from, x);
                        else {
#pragma unroll
                            for (int i = 0; i < 8; ++i) x[i] = k + i < a.K ? value_at<TYPE>(a.x, from + i) : 0.f;
                        }
                        uint4 op[NP];
                        row_operand<TYPE>(x, op);
                        char* to = lds + ((p * 4 + w) * 4 + c) * CS + m * 16;
#pragma unroll
                        for (int i = 0; i < NP; ++i) *reinterpret_cast<uint4*>(to + i * plane) = op[i];
                        // the sum of a row's group: eight inputs of this lane, the other three lanes' of the 32, earlier operands'
                        float of = ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
                        of += dpp_f32<0xB1>(of);
                        of += dpp_f32<0x4E>(of);
                        group += of;
                        if ((w + 1) % per == 0) {
                            if (c == 0) sums[((p * 4 + w) / per) * ROWS + m] = group;
                            group = 0.f;
                        }
                    }
                }
                __syncthreads();
            }
            const int turns = (here + deep - 1) / deep;
            for (int turn = 0; turn < turns; ++turn) {
                const int p = turn * deep + wk;
                PackedPiece now[NS];
#pragma unroll
                for (int s = 0; s < NS; ++s) now[s] = next[s];
                if (turn + 1 < turns) ask(set, part0 + p + deep);
                else if (chunk + 1 < chunks) ask(set, part0 + a.chunk + wk);
                else if (set + (int)gridDim.x < a.sets) ask(set + gridDim.x, wk);
                if (p >= here) continue;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    uint4 x[MT][NP];
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                        for (int i = 0; i < NP; ++i)
                            x[mt][i] = *reinterpret_cast<const uint4*>(lds + i * plane + ((p * 4 + w) * 4 + (ln >> 4)) * CS + (16 * mt + (ln & 15)) * 16);
#pragma unroll
                    for (int s = 0; s < NS; ++s) {
                        const uint32_t word = w == 0 ? now[s].codes.x : w == 1 ? now[s].codes.y : w == 2 ? now[s].codes.z : now[s].codes.w;
                        const auto op = codes_operand<TYPE>(word);
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                            for (int i = NP - 1; i >= 0; --i) acc[mt][s] = product<TYPE>(x[mt][i], op, acc[mt][s]);
                    }
                    if ((w + 1) % per != 0) continue;
                    const int g = w / per;
                    if ((part0 + p) * kPackInputs + (g << a.shift) >= a.K) continue;     // (scales behind the last group are not used)
                    f32x4 X[MT];
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) X[mt] = *reinterpret_cast<const f32x4*>(sums + ((p * 4 + w) / per) * ROWS + 16 * mt + 4 * (ln >> 4));
#pragma unroll
                    for (int s = 0; s < NS; ++s) {
                        const uint32_t bits = (uint32_t)(now[s].scales >> (16 * g)) & 0xffffu;
                        const float sc = a.scale_f16 ? scale_f32<true>(bits) : scale_f32<false>(bits);
                        const float zero = (float)(now[s].zeros >> (8 * g) & 0xffu);
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
                            for (int i = 0; i < 4; ++i) y[mt][s][i] = fmaf(sc, fmaf(-zero, X[mt][i], acc[mt][s][i]), y[mt][s][i]);
                            acc[mt][s] = f32x4{0.f, 0.f, 0.f, 0.f};
                        }
                    }
                }
            }
        }
        auto finish = [&](int of, int mt, int nt, f32x4 g, f32x4 u) {
            const int64_t n = ((int64_t)(set * across + of) * NT + nt) * kPackOutputs + (ln & 15);
            if (n >= a.N) return;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int m = 16 * mt + 4 * (ln >> 4) + i;
                if (m < rows) put_result(a, m0 + m, n, GATED ? activate(g[i], a.activation) * u[i] : g[i]);
            }
        };
        if (deep == 1) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) finish(wn, mt, nt, y[mt][GATED ? 2 * nt : nt], y[mt][GATED ? 2 * nt + 1 : nt]);
            continue;
        }
        // waves that share inputs: their sums through LDS, each wave adds up some of the tiles, in order
        if (a.join_at == 0) __syncthreads();
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int s = 0; s < NS; ++s) join[(((wk * across + wn) * MT + mt) * NS + s) * 64 + ln] = y[mt][s];
        __syncthreads();
        for (int i = wave; i < across * MT * NT; i += kPackedWaves) {
            const int nt = i % NT, mt = i / NT % MT, of = i / (NT * MT);
            f32x4 sum[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
            for (int d = 0; d < deep; ++d)
#pragma unroll
                for (int h = 0; h < (GATED ? 2 : 1); ++h) sum[h] += join[(((d * across + of) * MT + mt) * NS + (GATED ? 2 * nt + h : nt)) * 64 + ln];
            finish(of, mt, nt, sum[0], sum[1]);
        }
        __syncthreads();
    }
}

}  // namespace lshbeam
