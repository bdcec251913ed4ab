// Rows times weights of 4 bits (lsh_packed_linear, lsh_packed_gated):
//   y[m, n] = sum_k x[m, k] (code[n, k] - zero[n, g]) scale[n, g] = sum_g scale[n, g] sum_{k in g} x[m, k] (code[n, k] - zero[n, g])
// code - zero is exact in bf16 and fp16, rows of fp32 are taken apart into three planes of bf16 that add up to them, so every product is exact and
// nothing but the fp32 sums rounds.  A conversion of eight codes is 11 instructions in fp16, else 19, and 13 where no matrix has zeros.  (The codes as they are,
// and the zero times the sum of a group's inputs taken off afterwards, is one of 7, but of two terms that are many times their difference where a row's inputs
// have one sign.)
//
// Few rows: two operations a weight and row, so the weights' bytes bound it.  The rows' operands are in LDS, made once where all of them fit; the weights come
// straight to registers, the next part of a wave while the others work.  The waves of a workgroup are side by side along the outputs or share the inputs of
// the same outputs among them, and workgroups go on to further outputs.  16 waves of up to 16 rows hide what each waits for (12 rows x 40000 x 1000,
// fp32: 14.9 us a launch, eight waves 17.3; 4096 x 4096 in bf16 7.7 and 8.4); eight for more rows, which have no registers for that, and for small matrices.
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
    // few outputs of many inputs: these are split among workgroups, whose sums k_packed_join adds up
    int splits, split_parts;
    float* partial;            // [splits][matrix][M, N]
    // of k_packed_rows
    int rows;                  // of a workgroup
    int log_across;            // log2 of the waves side by side along the outputs; the others share their inputs
    int chunk, turns;          // parts whose rows are in LDS at a time, the most that a wave has of them
    int sets;                  // groups of tiles
    int join_at;               // where in LDS waves that share inputs add up
};

constexpr int kRowsPlanesF32 = 3;
template <int TYPE> constexpr int kRowPlanes = TYPE == kTypeF32 ? kRowsPlanesF32 : 1;
// LDS: operands of 32 inputs: [plane][of the chunk][c][row] 16 bytes, the c's 32 bytes apart so that four neighbouring lanes write to banks
// of their own; twice (for one group of tiles and the next) what the waves that share inputs add up.
constexpr int rows_of_c(int rows) { return rows * 16 + 32; }
constexpr int packed_plane(int rows, int chunk) { return chunk * 4 * 4 * rows_of_c(rows); }
constexpr int packed_join(int waves, int row_tiles, int streams) { return waves * row_tiles * streams * 1024; }

template <int TYPE> struct OperandOf { using type = bf16x8; };
template <> struct OperandOf<kTypeF16> { using type = f16x8; };

// Is there a conversion of its own for zeros of 8?
template <int TYPE> constexpr bool kEights = TYPE != kTypeF16;
// Eight codes less their zero, exactly, as an operand.
template <int TYPE, bool EIGHT> __device__ __forceinline__ typename OperandOf<TYPE>::type weights_operand(uint32_t word, float zero) {
    if constexpr (EIGHT) {
        // code - 8 of all eight at once: its sign, and its size, 0 .. 8; a byte of both is an e4m3 number
        uint32_t negative = ~word & 0x88888888u;
        asm("" : "+v"(negative));                // (not taken for what it is: three instructions more)
        const uint32_t one = negative >> 3, size = ((word & 0x77777777u) ^ (negative - one)) + one;
        const uint32_t lo = (size & 0x0f0f0f0fu) | (negative << 4 & 0xf0f0f0f0u), hi = (size >> 4 & 0x0f0f0f0fu) | (negative & 0xf0f0f0f0u);
        const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 512.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 512.f, true);
        const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 512.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 512.f, true);
        return bf16x8{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
    }
    const uint32_t lo = word & 0x0f0f0f0fu, hi = word >> 4 & 0x0f0f0f0fu;
    if constexpr (TYPE == kTypeF16) {
        const _Float16 z = (_Float16)zero;
        const f16x2 zz = {z, z};
        const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 512.f, false) - zz, b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 512.f, true) - zz;
        const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 512.f, false) - zz, d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 512.f, true) - zz;
        return f16x8{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
    } else {
        bf16x8 op;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f32x2 v = i & 1 ? __builtin_amdgcn_cvt_pk_f32_fp8((int)(i & 2 ? hi : lo), true) : __builtin_amdgcn_cvt_pk_f32_fp8((int)(i & 2 ? hi : lo), false);
            const f32x2 w = {fmaf(v.x, 512.f, -zero), fmaf(v.y, 512.f, -zero)};
            const bf16x2 b = __builtin_convertvector(w, bf16x2);
            op[2 * i] = b.x;
            op[2 * i + 1] = b.y;
        }
        return op;
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

// A result to its place, with what is added to it; one rounding.
__device__ __forceinline__ float added(const PackedArgs& a, int64_t m, int64_t n) {
    const int64_t at = m * a.ld_add + n;
    return a.out_type == kTypeF32 ? value_at<kTypeF32>(a.add, at) : a.out_type == kTypeBf16 ? value_at<kTypeBf16>(a.add, at) : value_at<kTypeF16>(a.add, at);
}
__device__ __forceinline__ void put_result(const PackedArgs& a, int64_t m, int64_t n, float y) {
    const int64_t at = m * a.ld_out + n;
    if (a.out_type == kTypeF32) put_value<kTypeF32>(a.out, at, y);
    else if (a.out_type == kTypeBf16) put_value<kTypeBf16>(a.out, at, y);
    else put_value<kTypeF16>(a.out, at, y);
}

// A part of a result's sum.
template <bool GATED> __device__ __forceinline__ void put_partial(const PackedArgs& a, int split, int64_t m, int64_t n, float g, float u) {
    float* to = a.partial + ((int64_t)split * (GATED ? 2 : 1) * a.M + m) * a.N + n;
    to[0] = g;
    if (GATED) to[(int64_t)a.M * a.N] = u;
}
// The parts' sums, added up in order, to results.  A thread for each.
template <bool GATED> __global__ void __launch_bounds__(256) k_packed_join(PackedArgs a) {
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x, size = (int64_t)a.M * a.N;
    if (at >= size) return;
    const int64_t m = at / a.N, n = at - m * a.N;
    float g = 0.f, u = 0.f;
    for (int i = 0; i < a.splits; ++i) {
        const float* from = a.partial + (int64_t)i * (GATED ? 2 : 1) * size + at;
        g += from[0];
        if (GATED) u += from[size];
    }
    if constexpr (GATED) put_result(a, m, n, activate(g, a.activation) * u);
    else put_result(a, m, n, g + ((a.add ? added(a, m, n) : 0.f) + (a.bias ? a.bias[n] : 0.f)));
}

// What a wave asks of a tile's part: codes, its output's scales and zeros.
template <int PER> struct PackedPiece {
    uint4 codes;
    uint32_t scales[PER == 1 ? 2 : 1], zeros;
};

// MT: 16 rows each; NS: tiles of a wave (gated: half of them of each matrix, gate and up in turn); PER: times 32 inputs of a group; EIGHT: no matrix has zeros.
template <int TYPE, int MT, int NS, int PER, bool GATED, int WAVES, bool EIGHT>
__global__ void __launch_bounds__(64 * WAVES) k_packed_rows(PackedArgs a) {
    extern __shared__ __align__(16) char lds[];
    constexpr int NP = kRowPlanes<TYPE>, NT = GATED ? NS / 2 : NS, EACH = 4 / PER;
    const int wave = __builtin_amdgcn_readfirstlane(wave_id()), ln = lane_id(), c = ln >> 4;
    const int wn = wave & ((1 << a.log_across) - 1), wk = wave >> a.log_across;
    const int log_deep = (WAVES == 16 ? 4 : 3) - a.log_across, deep = 1 << log_deep;
    const int m0 = blockIdx.y * a.rows, rows = min(a.rows, a.M - m0), of_c = rows_of_c(a.rows), plane = packed_plane(a.rows, a.chunk);
    const int from_part = blockIdx.z * a.split_parts, parts = min(a.split_parts, a.parts - from_part);
    const int chunks = (parts + a.chunk - 1) / a.chunk;

    // the next part of the wave: asked for as soon as the one before it has been worked on
    int ask_set = blockIdx.x, ask_chunk = 0, ask_turn = 0;
    auto ask = [&](PackedPiece<PER> (&to)[NS]) {
        const int part = from_part + min(ask_chunk * a.chunk + min((ask_turn << log_deep) + wk, a.chunk - 1), parts - 1);
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            const int tile = min(((ask_set << a.log_across) + wn) * NT + (GATED ? s >> 1 : s), a.tiles - 1);
            const PackedRef& w = a.w[GATED ? s & 1 : 0];
            const int64_t unit = (int64_t)tile * a.parts + part, group = unit * (16 * EACH) + (ln & 15) * EACH;
            to[s].codes = *reinterpret_cast<const uint4*>(w.codes + unit * kPackBytes + 16 * ln);
            const uint16_t* scales = w.scales + group;
            const uint8_t* zeros = w.zeros ? w.zeros + group : reinterpret_cast<const uint8_t*>(scales);
            if constexpr (PER == 4) { to[s].scales[0] = *scales; to[s].zeros = *zeros; }
            else if constexpr (PER == 2) { to[s].scales[0] = *reinterpret_cast<const uint32_t*>(scales); to[s].zeros = *reinterpret_cast<const uint16_t*>(zeros); }
            else {
                const uint2 two = *reinterpret_cast<const uint2*>(scales);
                to[s].scales[0] = two.x; to[s].scales[1] = two.y;
                to[s].zeros = *reinterpret_cast<const uint32_t*>(zeros);
            }
        }
        if (++ask_turn == a.turns) {
            ask_turn = 0;
            if (++ask_chunk == chunks) { ask_chunk = 0; ask_set = min(ask_set + (int)gridDim.x, a.sets - 1); }   // (behind the end the last one once more)
        }
    };
    PackedPiece<PER> piece[NS];
    ask(piece);

    f32x4 y[MT][NS];
    auto work = [&](const PackedPiece<PER> (&now)[NS], int part0, int p) {
        f32x4 acc[MT][NS];
        const char* at = lds + p * (16 * of_c) + c * of_c;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            uint4 x[MT][NP];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int i = 0; i < NP; ++i)
                    x[mt][i] = *reinterpret_cast<const uint4*>(at + i * plane + w * (4 * of_c) + 16 * min(16 * mt + (ln & 15), rows - 1));
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                const float zero = !EIGHT && a.w[GATED ? s & 1 : 0].zeros ? (float)(now[s].zeros >> (8 * (w / PER)) & 0xffu) : 8.f;
                const auto op = weights_operand<TYPE, EIGHT>(w == 0 ? now[s].codes.x : w == 1 ? now[s].codes.y : w == 2 ? now[s].codes.z : now[s].codes.w, zero);
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int i = NP - 1; i >= 0; --i)
                        acc[mt][s] = product<TYPE>(x[mt][i], op, w % PER == 0 && i == NP - 1 ? f32x4{0.f, 0.f, 0.f, 0.f} : acc[mt][s]);
            }
            if ((w + 1) % PER != 0) continue;
            const int g = w / PER;
            const bool counts = (part0 + p) * kPackInputs + g * (32 * PER) < a.K;     // (scales behind the last group are not used)
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                const uint32_t bits = PER == 1 ? now[s].scales[PER == 1 ? g >> 1 : 0] >> (16 * (g & 1)) & 0xffffu : now[s].scales[0] >> (16 * g) & 0xffffu;
                const float sc = !counts ? 0.f : a.scale_f16 ? scale_f32<true>(bits) : scale_f32<false>(bits);
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) y[mt][s][i] = fmaf(sc, acc[mt][s][i], y[mt][s][i]);
            }
            if constexpr (PER == 1 && MT * NS == 8) __builtin_amdgcn_sched_barrier(0);   // (several groups' sums at once have no registers)
        }
    };

    const int finishing = (MT * NT) << a.log_across;    // tiles of results, no more than waves
    bool second = false;
    for (int set = blockIdx.x; set < a.sets; set += gridDim.x) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int s = 0; s < NS; ++s) y[mt][s] = f32x4{0.f, 0.f, 0.f, 0.f};
        // the tile of results that the wave finishes, and what is added to it
        const int nt = wave % NT, mt_of = wave / NT % MT, of = wave / (NT * MT);
        const int64_t n = ((int64_t)((set << a.log_across) + of) * NT + nt) * kPackOutputs + (ln & 15);
        const bool mine = wave < finishing && n < a.N;
        f32x4 plus = {0.f, 0.f, 0.f, 0.f};
        if (!GATED && mine && a.splits == 1) {
            const float b = a.bias ? a.bias[n] : 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int m = 16 * mt_of + 4 * c + i;
                plus[i] = a.add && m < rows ? added(a, m0 + m, n) + b : b;
            }
        }
        for (int chunk = 0; chunk < chunks; ++chunk) {
            const int part0 = from_part + chunk * a.chunk, here = min(a.chunk, parts - chunk * a.chunk);
            if (chunks > 1 || set == (int)blockIdx.x) {
                __syncthreads();
                for (int u = threadIdx.x; u < here * rows * 4; u += 64 * WAVES) {
                    const int q = u >> 2, m = q % rows, p = q / rows, cc = u & 3;
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const int k = (part0 + p) * kPackInputs + 32 * w + 8 * cc;
                        const int64_t from = (int64_t)(m0 + m) * a.ldx + k;
                        float x[8];
                        if (k + 8 <= a.K) load_values<TYPE>(a.x, from, x);
                        else {
#pragma unroll
                            for (int i = 0; i < 8; ++i) x[i] = k + i < a.K ? value_at<TYPE>(a.x, from + i) : 0.f;
                        }
                        uint4 op[NP];
                        row_operand<TYPE>(x, op);
                        char* to = lds + ((p * 4 + w) * 4 + cc) * of_c + m * 16;
#pragma unroll
                        for (int i = 0; i < NP; ++i) *reinterpret_cast<uint4*>(to + i * plane) = op[i];
                    }
                }
                __syncthreads();
            }
            for (int turn = 0; turn < a.turns; ++turn) {
                const int p = turn * deep + wk;
                if (p < here) work(piece, part0, p);
                ask(piece);
            }
        }
        auto finish = [&](f32x4 g, f32x4 u, int mt) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int m = 16 * mt + 4 * c + i;
                if (m >= rows) continue;
                if (a.splits > 1) put_partial<GATED>(a, blockIdx.z, m0 + m, n, g[i], u[i]);
                else put_result(a, m0 + m, n, GATED ? activate(g[i], a.activation) * u[i] : g[i] + plus[i]);
            }
        };
        // waves that share inputs: their sums through LDS, each wave adds up a tile, in order
        f32x4* join = reinterpret_cast<f32x4*>(lds + a.join_at + (second ? packed_join(WAVES, MT, NS) : 0));
        second = !second;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int s = 0; s < NS; ++s) join[((wave * MT + mt) * NS + s) * 64 + ln] = y[mt][s];
        lds_barrier();
        if (mine) {
            f32x4 sum[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
            for (int d = 0; d < deep; ++d)
#pragma unroll
                for (int h = 0; h < (GATED ? 2 : 1); ++h)
                    sum[h] += join[((((d << a.log_across) + of) * MT + mt_of) * NS + (GATED ? 2 * nt + h : nt)) * 64 + ln];
            finish(sum[0], sum[1], mt_of);
        }
    }
}

}  // namespace lshbeam
