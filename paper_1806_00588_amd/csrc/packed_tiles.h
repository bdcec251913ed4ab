// Many rows times weights of 4 bits: y[m, n] = sum_g scale[n, g] sum_{k in g} x[m, k] (code[n, k] - zero[n, g]).
//
// k_packed_lay brings the rows into the order of the matrix operands (fp32: three planes of bf16), so that everything k_packed_tiles loads are
// blocks of 1 KB, straight to LDS.  Rows of 16 bits, of which nothing has to be made before, come from where they lie if
// 16 bytes of them are always neighbours and in place: 40 rows of fp16 x 1000 x 16384 20 -> 16 us, 40 of bf16 x 8192 x 8192 29 -> 26,
// 2048 x 8192 x 8192 291 -> 286 in a graph.  A workgroup of eight waves makes 128 rows, two waves side by side along them and four along the outputs.  Weights are
// converted in registers, once by each of the two.  A group's products are summed up by themselves, then scaled and added to what came before, so
// that nothing but fp32 sums rounds; that takes two accumulators, and 64 x 64 results of a wave are what has room for both in 256 registers.  Up to 64 rows: the two waves with the same
// outputs take turns with the parts instead of sharing the rows, so that no weight is converted twice, and add up at the end.
// (128 x 64 and four waves, with accumulators in the other 256, which only the matrix instructions reach: 2048 x 8192 x 8192 in fp16 541 us, moves being
// most of it.)
#pragma once
#include "packed_rows.h"

namespace lshbeam {

constexpr int kTileAcross = 4;      // waves along the outputs
constexpr int kTileWaves = 2 * kTileAcross;

// [16 rows][part][4][plane] blocks of 1 KB.  A wave for 16 rows and a part; four neighbouring lanes read 32 neighbouring inputs.
template <int TYPE>
__global__ void __launch_bounds__(256) k_packed_lay(PackedArgs a, char* to, int64_t units) {
    constexpr int P = kRowPlanes<TYPE>;
    const int64_t unit = (int64_t)blockIdx.x * 4 + wave_id();
    if (unit >= units) return;
    const int64_t mt = unit / a.parts, m = mt * 16 + (lane_id() >> 2);
    const int part = (int)(unit - mt * a.parts), c = lane_id() & 3;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const int k = part * kPackInputs + 32 * w + 8 * c;
        const int64_t from = m * a.ldx + k;
        float x[8];
        if (m < a.M && k + 8 <= a.K) load_values<TYPE>(a.x, from, x);
        else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = m < a.M && k + i < a.K ? value_at<TYPE>(a.x, from + i) : 0.f;
        }
        uint4 op[P];
        row_operand<TYPE>(x, op);
#pragma unroll
        for (int p = 0; p < P; ++p) *reinterpret_cast<uint4*>(to + ((unit * 4 + w) * P + p) * 1024 + (16 * c + (lane_id() >> 2)) * 16) = op[p];
    }
}

// MT: times 16 rows of a wave; NS: its tiles of outputs; DEEP: the two waves with the same outputs have the same rows and every second part, else other
// rows and the same parts.
template <int TYPE, int MT, int NS, bool DEEP> struct TilesPlan {
    static constexpr int P = kRowPlanes<TYPE>;
    static constexpr int kHalves = DEEP ? 2 : 1, kRows = DEEP ? MT : 2 * MT;             // parts at a time; times 16 rows of a workgroup
    static constexpr int KS = P == 1 ? 2 : 1;                        // times 32 inputs of a stage
    static constexpr int kOf = 4 / KS;                               // stages of a part
    static constexpr int kRing = P == 1 ? 5 : 4;                     // stages of rows in LDS, or on their way
    static constexpr int kParts = (kRing - 2) / kOf + 2;             // turns of codes
    static constexpr int kRowsSlot = kHalves * kRows * KS * P * 1024;
    static constexpr int kRowsEach = kRowsSlot / 1024 / kTileWaves;  // a wave's loads of rows
    static constexpr int kCodesOf = kTileAcross * NS * kHalves, kCodesEach = kCodesOf < kTileWaves ? 1 : kCodesOf / kTileWaves;   // blocks of codes; a wave's loads
    static constexpr int kScalesEach = DEEP ? 3 : 2;
    static constexpr int kCodes = kRing * kRowsSlot, kCodesSlot = kCodesOf * 1024;
    static constexpr int kScales = kCodes + kParts * kCodesSlot, kScalesSlot = kTileAcross * kHalves * 768;
    static constexpr int kLds = kScales + kParts * kScalesSlot;
    static_assert(kLds <= (int)kMaxDynLds && kRowsEach * kTileWaves * 1024 == kRowsSlot && kHalves * kRows == kTileWaves, "every wave asks for as much");
    static_assert(!DEEP || kTileAcross * MT * NS * 1024 <= kCodes, "the sums of one half have room");
    // loads of a wave for the j-th stage of a turn
    static constexpr int loads(int j) { return kRowsEach + (j % kOf == 0 ? kCodesEach + kScalesEach : 0); }
    // ... that may be under way when stage j begins: all but those for it and the next one
    static constexpr int later(int j) {
        int n = 0;
        for (int i = j + 2; i <= j + kRing - 2; ++i) n += loads(i);
        return n;
    }
};

struct TilesArgs {
    PackedArgs p;
    bool as_they_are;          // rows are loaded from where they lie, 16 bytes a lane
    const char* x;             // k_packed_lay's blocks
    int row_tiles;             // 16 rows each
    int row_groups, sets;      // workgroups along the rows, along the outputs
};

// NS: tiles of 16 outputs of a wave (gated: half of them of each matrix, gate and up in turn); PER: times 32 inputs of a group; EIGHT: no matrix has zeros.
template <int TYPE, int MT, int NS, int PER, bool GATED, bool DEEP, bool EIGHT>
__global__ void __launch_bounds__(64 * kTileWaves, 1) k_packed_tiles(TilesArgs t) {
    using Plan = TilesPlan<TYPE, MT, NS, DEEP>;
    constexpr int P = Plan::P, KS = Plan::KS, OF = Plan::kOf, NT = GATED ? NS / 2 : NS, EACH = 4 / PER, HALVES = Plan::kHalves;
    constexpr bool AS_THEY_ARE = P == 1;
    extern __shared__ __align__(16) char lds[];
    const PackedArgs& a = t.p;
    const int wave = __builtin_amdgcn_readfirstlane(wave_id()), ln = lane_id(), wn = wave % kTileAcross, wm = DEEP ? 0 : wave / kTileAcross, wk = DEEP ? wave / kTileAcross : 0;
    // workgroups go round the eight XCDs one by one; an XCD gets neighbouring ones: four along the outputs, then along the rows
    const int total = t.row_groups * t.sets, each_xcd = (total + 7) / 8;
    const int u = (int)(blockIdx.x & 7) * each_xcd + (int)(blockIdx.x >> 3);
    if (u >= total || (int)(blockIdx.x >> 3) >= each_xcd) return;
    const int band = u / (4 * t.row_groups), wide = min(4, t.sets - 4 * band), in_band = u - band * 4 * t.row_groups;
    const int group = in_band / wide, set = 4 * band + in_band % wide;
    const int tile0 = (set * kTileAcross + wn) * NT, mt0 = group * Plan::kRows;
    // stream s of the waves with outputs w: matrix, tile's first part
    auto unit_of = [&](int w, int s) { return (int64_t)min((set * kTileAcross + w) * NT + (GATED ? s >> 1 : s), a.tiles - 1) * a.parts; };

    // (what is asked for of a half's part: from the part's place on)
    const char* rows_from[Plan::kRowsEach];      // of 16 rows those of a stage lie side by side
    const char* codes_from[Plan::kCodesEach];
    int rows_half[Plan::kRowsEach], codes_half[Plan::kCodesEach];
#pragma unroll
    for (int i = 0; i < Plan::kRowsEach; ++i) {
        const int b = wave * Plan::kRowsEach + i, mt = b / (KS * P);
        rows_half[i] = mt / Plan::kRows;
        const int tile = mt0 + mt % Plan::kRows, in_stage = b % (KS * P);
        if (AS_THEY_ARE && t.as_they_are) rows_from[i] = static_cast<const char*>(a.x) + (int64_t)min(16 * tile + (ln & 15), a.M - 1) * a.ldx * 2 + in_stage * 64 + 16 * (ln >> 4);
        else rows_from[i] = t.x + (int64_t)min(tile, t.row_tiles - 1) * a.parts * (4 * P * 1024) + in_stage * 1024 + 16 * ln;
    }
    const int rows_step = AS_THEY_ARE && t.as_they_are ? 64 : P * 1024;               // from 32 inputs to the next
#pragma unroll
    for (int i = 0; i < Plan::kCodesEach; ++i) {
        const int s = (wave * Plan::kCodesEach + i) % Plan::kCodesOf, of = s % (kTileAcross * NS);
        codes_half[i] = s / (kTileAcross * NS);
        codes_from[i] = reinterpret_cast<const char*>(a.w[GATED ? of & 1 : 0].codes) + unit_of(of / NS, of % NS) * kPackBytes + 16 * ln;
    }
    // scales and zeros of the wave's streams, 4 bytes a lane: 16 lanes a stream, scales twice that.  Waves with the same part share the work: the first
    // four ask for the scales, the others for the zeros
    const int mine = min(ln >> 4, NS - 1);
    const PackedRef& my = a.w[GATED ? mine & 1 : 0];
    const char* scales_from[3];
    int scales_step[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        if (i < 2 || !my.zeros) {
            scales_step[i] = 32 * EACH;
            scales_from[i] = reinterpret_cast<const char*>(my.scales) + unit_of(wn, mine) * scales_step[i] + 4 * min((ln & 15) + 16 * (i & 1), 8 * EACH - 1);
        } else {
            scales_step[i] = 16 * EACH;
            scales_from[i] = reinterpret_cast<const char*>(my.zeros) + unit_of(wn, mine) * scales_step[i] + 4 * min(ln & 15, 4 * EACH - 1);
        }
    }

    const int first_turn = blockIdx.y * (a.split_parts / HALVES), turns = min((a.parts + HALVES - 1) / HALVES, first_turn + a.split_parts / HALVES);
    int ask_turn = first_turn, ask_in = 0, ask_slot = 0, ask_codes = 0;
    auto part_of = [&](int half) { return (int64_t)min(ask_turn * HALVES + half, a.parts - 1); };
    auto ask = [&]() {
#pragma unroll
        for (int i = 0; i < Plan::kRowsEach; ++i)
            load_to_lds16(rows_from[i] + (part_of(rows_half[i]) * 4 + ask_in * KS) * rows_step, lds + ask_slot * Plan::kRowsSlot + (wave * Plan::kRowsEach + i) * 1024);
        if (ask_in == 0) {
#pragma unroll
            for (int i = 0; i < Plan::kCodesEach; ++i)
                load_to_lds16(codes_from[i] + part_of(codes_half[i]) * kPackBytes,
                              lds + Plan::kCodes + ask_codes * Plan::kCodesSlot + (wave * Plan::kCodesEach + i) % Plan::kCodesOf * 1024);
            char* to = lds + Plan::kScales + ask_codes * Plan::kScalesSlot + (wk * kTileAcross + wn) * 768;
            if (DEEP || wm == 0) {
                load_to_lds4(scales_from[0] + part_of(wk) * scales_step[0], to);
                load_to_lds4(scales_from[1] + part_of(wk) * scales_step[1], to + 256);
            } else {
                load_to_lds4(scales_from[2] + part_of(wk) * scales_step[2], to + 512);
                load_to_lds4(scales_from[2] + part_of(wk) * scales_step[2], to + 512);   // (as many loads as the other waves')
            }
            if constexpr (DEEP) load_to_lds4(scales_from[2] + part_of(wk) * scales_step[2], to + 512);
        }
        ask_slot = ask_slot + 1 == Plan::kRing ? 0 : ask_slot + 1;
        if (++ask_in == OF) {                    // (behind the end the last part once more)
            ask_in = 0;
            ask_turn = min(ask_turn + 1, turns - 1);
            ask_codes = ask_codes + 1 == Plan::kParts ? 0 : ask_codes + 1;
        }
    };
    for (int i = 0; i < Plan::kRing - 1; ++i) ask();

    f32x4 y[MT][NS], acc[MT][NS];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int s = 0; s < NS; ++s) y[m][s] = f32x4{0.f, 0.f, 0.f, 0.f};
    int slot = 0, codes_slot = 0;
    constexpr int AHEAD = P == 1;    // rows are read 32 inputs ahead (three planes: there are no registers for that, and three times the time)
    uint4 x[AHEAD + 1][MT][P];
    auto read_rows = [&](uint4 (&to)[MT][P], int of, int ks) {
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int p = 0; p < P; ++p) to[m][p] = *reinterpret_cast<const uint4*>(lds + of * Plan::kRowsSlot + ((((wk * Plan::kRows + wm * MT + m) * KS + ks) * P + p) * 1024) + 16 * ln);
    };
    wait_vmem<Plan::later(-1)>();
    lds_barrier();
    if constexpr (AHEAD) read_rows(x[0], 0, 0);
    for (int turn = first_turn; turn < turns; ++turn) {
        const int part = turn * HALVES + wk;
        uint4 codes[NS];
        float scale[NS], zero[NS];
        const char* sc = lds + Plan::kScales + codes_slot * Plan::kScalesSlot + (wk * kTileAcross + wn) * 768;
#pragma unroll
        for (int ks4 = 0; ks4 < 4; ++ks4) {
            const int j = ks4 / KS, ks = ks4 % KS, g = ks4 / PER;
            if (ks == 0) {                       // a stage: it is here, and so is the next one when the barrier is behind us
                if (j == 0) wait_vmem<Plan::later(0)>();
                else if (j == 1) wait_vmem<Plan::later(1)>();
                else if (j == 2) wait_vmem<Plan::later(2)>();
                else wait_vmem<Plan::later(3)>();
                lds_barrier();
                ask();
            }
            if (ks4 == 0) {
#pragma unroll
                for (int s = 0; s < NS; ++s) codes[s] = *reinterpret_cast<const uint4*>(lds + Plan::kCodes + codes_slot * Plan::kCodesSlot + ((wk * kTileAcross + wn) * NS + s) * 1024 + 16 * ln);
            }
            if (ks4 % PER == 0) {
#pragma unroll
                for (int s = 0; s < NS; ++s) {
                    const int at = (ln & 15) * EACH + g;
                    const uint32_t bits = *reinterpret_cast<const uint16_t*>(sc + (at >> 5) * 256 + s * 64 + 2 * (at & 31));
                    scale[s] = a.scale_f16 ? scale_f32<true>(bits) : scale_f32<false>(bits);
                    zero[s] = !EIGHT && a.w[GATED ? s & 1 : 0].zeros ? (float)*reinterpret_cast<const uint8_t*>(sc + 512 + s * 64 + at) : 8.f;
                }
            }
            if constexpr (AHEAD) {
                const int after = ks + 1 == KS ? (slot + 1 == Plan::kRing ? 0 : slot + 1) : slot;
                read_rows(x[(ks4 + 1) & 1], after, (ks + 1) % KS);
            } else read_rows(x[0], slot, ks);
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                const uint32_t word = ks4 == 0 ? codes[s].x : ks4 == 1 ? codes[s].y : ks4 == 2 ? codes[s].z : codes[s].w;
                const auto op = weights_operand<TYPE, EIGHT>(word, zero[s]);
                __builtin_amdgcn_s_setprio(1);      // (the two waves of a SIMD one behind the other: 1 to 3 %)
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int p = P - 1; p >= 0; --p)
                        acc[m][s] = product<TYPE>(x[ks4 & AHEAD][m][p], op, ks4 % PER == 0 && p == P - 1 ? f32x4{0.f, 0.f, 0.f, 0.f} : acc[m][s]);
            }
            __builtin_amdgcn_s_setprio(0);
            if ((ks4 + 1) % PER == 0) {
                const bool counts = part * kPackInputs + g * (32 * PER) < a.K;    // (scales behind the last group are not used)
#pragma unroll
                for (int s = 0; s < NS; ++s) {
                    const float f = counts ? scale[s] : 0.f;
#pragma unroll
                    for (int m = 0; m < MT; ++m)
#pragma unroll
                        for (int i = 0; i < 4; ++i) y[m][s][i] = fmaf(f, acc[m][s][i], y[m][s][i]);
                }
            }
            if (ks + 1 == KS) slot = slot + 1 == Plan::kRing ? 0 : slot + 1;
            if constexpr (PER < 4) __builtin_amdgcn_sched_barrier(0);   // (several groups' sums at once have no registers)
        }
        codes_slot = codes_slot + 1 == Plan::kParts ? 0 : codes_slot + 1;
    }
    wait_vmem<0>();                              // (nothing may come into another workgroup's LDS)
    if constexpr (DEEP) {                        // the second half's sums to the first
        lds_barrier();
        f32x4* join = reinterpret_cast<f32x4*>(lds) + wn * MT * NS * 64 + ln;
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int s = 0; s < NS; ++s)
                if (wk == 1) join[(m * NS + s) * 64] = y[m][s];
        lds_barrier();
        if (wk == 1) return;
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int s = 0; s < NS; ++s) y[m][s] += join[(m * NS + s) * 64];
    }
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int64_t n = (int64_t)(tile0 + nt) * kPackOutputs + (ln & 15);
            if (n >= a.N) continue;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int64_t row = (int64_t)(mt0 + wm * MT + m) * 16 + 4 * (ln >> 4) + i;
                if (row >= a.M) continue;
                if (a.splits > 1) put_partial<GATED>(a, blockIdx.y, row, n, y[m][GATED ? 2 * nt : nt][i], y[m][GATED ? 2 * nt + 1 : nt][i]);
                else if constexpr (GATED) put_result(a, row, n, activate(y[m][2 * nt][i], a.activation) * y[m][2 * nt + 1][i]);
                else put_result(a, row, n, y[m][nt][i] + ((a.add ? added(a, row, n) : 0.f) + (a.bias ? a.bias[n] : 0.f)));
            }
        }
}

}  // namespace lshbeam
