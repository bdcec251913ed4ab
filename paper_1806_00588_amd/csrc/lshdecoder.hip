// C ABI of what stands around a decoder that makes its own logits and keeps a paged cache (see include/lshbeam.h): selection
// from dense logits, block tables, cache writes, attention.  Host side: argument validation, the choice of kernels, launches.
// A translation unit of its own: its kernels are a code object of their own, so the places of the decode step's kernels in
// theirs (short kernels' times go by them) stay as they are.
#ifdef LSHBEAM_TRACE   // (the phase timestamps belong to the decode step's kernels)
#undef LSHBEAM_TRACE
#endif
#include "../../include/lshbeam.h"

#include <hip/hip_runtime.h>

#include <algorithm>

#include "beam_select.h"
#include "cache_attention.h"
#include "cache_tables.h"
#include "cache_write.h"
#include "launch.h"

using namespace lshbeam;

namespace {

constexpr int kMaxWords = 1 << 24, kMaxBeams = 256;
constexpr int kMaxBlocks = 1 << 24, kMaxColumns = 1 << 20;
constexpr int kMaxNew = kMaxColumns * 128;    // tokens that the widest table holds; kernels count new ones in 32 bits, a workgroup's threads at a time

// ---- selection ----------------------------------------------------------------------------------

bool select_ok(const lsh_select_params* p) {
    return p && p->S >= 1 && p->B >= 1 && p->B <= kMaxBeams && p->N >= 1 && p->N <= kMaxBeams && p->V >= 1 && p->V <= kMaxWords &&
           (int64_t)p->S * p->B <= kMaxRows;
}
int64_t row_pieces(const lsh_select_params* p) { return ceil_div(p->V, kSelPiece); }
bool select_is_small(const lsh_select_params* p) { return p->B * row_pieces(p) <= kSelSmall; }

// Pieces of a wave of k_select_tiles: one as long as there are few waves, four (its loads are under way together) with many, more where
// there are far more waves than the chip holds.
int wave_pieces(const lsh_select_params* p) {
    const int64_t R = (int64_t)p->S * p->B, all = row_pieces(p);
    int n = 1;
    while (n < kSelBatch && R * ceil_div(all, n) > 2048) n *= 2;
    while (n >= kSelBatch && n < 2 * kSelBatch && R * ceil_div(all, 2 * n) >= 256 * 32) n *= 2;
    return n;
}
size_t select_bytes(const lsh_select_params* p, size_t* tiles_bytes) {
    const size_t R = (size_t)p->S * p->B;
    *tiles_bytes = round_up(R * (size_t)ceil_div(p->V, kSelTile) * sizeof(float));
    return *tiles_bytes + round_up(R * (size_t)ceil_div(row_pieces(p), wave_pieces(p)) * sizeof(SelPart));
}

// ---- cache --------------------------------------------------------------------------------------

bool cache_ok(const lsh_cache_params* c) {
    return c && c->S >= 1 && c->B >= 1 && c->B <= kMaxBeams && (int64_t)c->S * c->B <= kMaxRows && c->n_blocks >= 1 && c->n_blocks <= kMaxBlocks &&
           (c->block == 16 || c->block == 32 || c->block == 64 || c->block == 128) && (int64_t)c->n_blocks * c->block <= INT32_MAX &&
           c->max_blocks >= 1 && c->max_blocks <= kMaxColumns && c->n_heads >= 1 && c->n_heads <= 65535 && c->head_dim >= 16 &&
           c->head_dim <= 256 && c->head_dim % 16 == 0;
}
bool pool_ok(const lsh_cache_pool* p) {
    return p && p->k && p->v && p->k_scale && p->v_scale && aligned(p->k, 16) && aligned(p->v, 16);
}
struct TablesRoom { size_t plan, base, free_ids, used, bytes; };
TablesRoom tables_room(const lsh_cache_params* c) {
    const size_t R = (size_t)c->S * c->B;
    TablesRoom w{};
    w.base = round_up(R * sizeof(RowPlan));
    w.free_ids = w.base + round_up(R * sizeof(int32_t));
    w.used = w.free_ids + round_up((size_t)c->n_blocks * sizeof(int32_t));
    w.bytes = w.used + round_up((size_t)c->n_blocks);
    return w;
}

bool attention_ok(const lsh_cache_params* c, const lsh_attention_params* p) {
    return cache_ok(c) && p && p->T >= 1 && p->T <= kMaxRows && p->n_heads >= 1 && p->n_heads <= 65535 && p->n_heads % c->n_heads == 0;
}
// Rows of queries, of all heads: the join has a wave for each.  What is derived from them (groups, workgroups, bytes) is not looked at before
// that is known: it need not fit its type.
int64_t query_rows(const lsh_cache_params* c, const lsh_attention_params* p) { return (int64_t)c->S * c->B * p->T * p->n_heads; }
bool rows_fit(const lsh_cache_params* c, const lsh_attention_params* p) { return ceil_div(query_rows(c, p), 4) <= kMaxGrid; }

// How a call of the attention is divided: a launch for all beams together (if the blocks that they have in common are given) and one
// for each row by itself, which a third joins if there is more than one part of a row.
struct AttnLaunch {
    int row_tiles;      // 1: k_attention_few, else the waves of k_attention_rows
    int chunk;          // tiles of 64 tokens at least
    int groups, splits;
    int64_t units;      // workgroups; 0: no such launch
};
struct AttnPlan {
    AttnLaunch common, own;
    size_t acc, bytes;  // where the parts' products begin in the workspace; its size
    bool fits() const { return common.units + own.units <= kMaxGrid; }
};
// sets: pairs of a row set and a head; tiles: of a row at most -- what a row has is known on the device only, and a chunk behind its
// last tile costs little.  A chunk of few rows has four tiles at least, eight or 16 where that still makes workgroups for the chip (a
// workgroup's begin and end and its part of the join are worth some tiles: 128 rows of up to 1024 tokens, 8 heads of 64, chunks of
// 4, 8, 16 tiles 25.9, 25.2, 19.1 us; 2 rows of 8192 13.8, 12.6, 14.2), one of k_attention_rows eight; more where a row would have
// more chunks than workgroups.  Rows of at most eight tiles are not split: one tile more for each wave costs less than the join
// (ten tiles of fp32 queries, 18 rows of 3 heads: split 14.9 us a call, not split 16.8).
AttnLaunch attention_launch(int64_t rows, int64_t most_rows, int64_t sets, int64_t tiles, int64_t most_splits) {
    AttnLaunch w{};
    w.groups = (int)ceil_div(rows, most_rows);
    w.row_tiles = (int)ceil_div(ceil_div(rows, w.groups), 16);
    sets *= w.groups;
    w.chunk = w.row_tiles > 1 || tiles <= 8 ? 8 : sets * ceil_div(tiles, 4) <= 256 ? 4 : sets * ceil_div(tiles, 8) <= 512 ? 8 : 16;
    w.splits = (int)std::min({ceil_div(tiles, w.chunk), std::max<int64_t>(1, (w.row_tiles > 1 ? 1024 : 2048) / sets), most_splits});
    w.units = sets * w.splits;
    return w;
}
// Rows of queries that a workgroup takes at most, by what the kernel for heads of D values has LDS for.
int64_t most_rows(int32_t dtype, int32_t D) {
    static_assert(kRowsMost<kTypeF32, 64> == 4 && kRowsMost<kTypeF32, 128> == 4 && kRowsMost<kTypeF32, 192> == 4 && kRowsMost<kTypeF16, 256> == 4 &&
                  kRowsMost<kTypeBf16, 256> == 4, "only fp32 with heads of 256 (and those that run in their code) is asked for here");
    return dtype == LSH_F32 && D > 128 && D != 192 ? 16 * kRowsMost<kTypeF32, 256> : 64;
}
AttnPlan attention_plan(const lsh_cache_params* c, const lsh_attention_params* p, int32_t dtype, bool shared) {
    AttnPlan w{};
    const int64_t most = most_rows(dtype, c->head_dim);
    const int64_t R = (int64_t)c->S * c->B, per_row = (int64_t)p->T * (p->n_heads / c->n_heads);
    int64_t tiles = ceil_div((int64_t)c->max_blocks * c->block, kAttnTile);
    if (p->window > 0) tiles = std::min(tiles, ceil_div((int64_t)p->window + p->T, kAttnTile) + 1);
    // beams together where it saves reading more than two launches more cost: 32 MB
    const bool common = shared && c->B > 1 && R * c->n_heads * tiles * kAttnTile * 2 * c->head_dim > (int64_t)32 << 20;
    if (common) w.common = attention_launch(c->B * per_row, most, (int64_t)c->S * c->n_heads, tiles, INT32_MAX);
    // (beams' own tokens are few, and whatever there is of them goes round the workgroups)
    w.own = attention_launch(per_row, most, R * c->n_heads, tiles, common ? std::max<int64_t>(1, 512 / (R * c->n_heads)) : INT32_MAX);
    const size_t parts = (size_t)(w.common.splits + w.own.splits), at = (size_t)R * p->T * p->n_heads * (parts > 1 ? parts : 0);
    w.acc = round_up(at * sizeof(float2));
    w.bytes = std::max<size_t>(256, w.acc + round_up(at * c->head_dim * sizeof(float)));
    return w;
}

// The launches over the cache: the common blocks' and the rows' own, one where the latter have at most 16 rows of queries.  (Heads of
// more than 128 values need more registers for these than two waves per SIMD have.)
template <int TYPE, int DP, bool EXACT> bool attend_both(const BothArgs& b, int row_tiles, unsigned grid, hipStream_t st) {
    if (row_tiles == 1) return launch_lds<k_attention_both<TYPE, DP, 1, EXACT>, kBothLds<TYPE, DP, 1>>(grid, 256, st, b);
    if (row_tiles == 2) return launch_lds<k_attention_both<TYPE, DP, 2, EXACT>, kBothLds<TYPE, DP, 2>>(grid, 256, st, b);
    if (row_tiles == 3) return launch_lds<k_attention_both<TYPE, DP, 3, EXACT>, kBothLds<TYPE, DP, 3>>(grid, 256, st, b);
    return launch_lds<k_attention_both<TYPE, DP, 4, EXACT>, kBothLds<TYPE, DP, 4>>(grid, 256, st, b);
}
template <int TYPE, int DP, bool EXACT> bool attend(const AttnArgs& a, const AttnLaunch& w, hipStream_t st) {
    const unsigned grid = (unsigned)w.units;
    if (w.row_tiles == 1) return launch_lds<k_attention_few<TYPE, DP, EXACT>, kFewLds<TYPE, DP>>(grid, 256, st, a);
    if (w.row_tiles == 2) return launch_lds<k_attention_rows<TYPE, DP, 2, EXACT>, kRowsLds<TYPE, DP, 2>>(grid, 128, st, a);
    if constexpr (kRowsMost<TYPE, DP> == 4) {
        if (w.row_tiles == 4) return launch_lds<k_attention_rows<TYPE, DP, 4, EXACT>, kRowsLds<TYPE, DP, 4>>(grid, 256, st, a);
    }
    return launch_lds<k_attention_rows<TYPE, DP, 3, EXACT>, kRowsLds<TYPE, DP, 3>>(grid, 192, st, a);
}
template <int TYPE, int DP, bool EXACT> bool attend(const BothArgs& b, const AttnPlan& plan, hipStream_t st) {
    if (plan.common.units == 0) return attend<TYPE, DP, EXACT>(b.own, plan.own, st);
    if constexpr (DP <= 128) {
        if (plan.own.row_tiles == 1) return attend_both<TYPE, DP, EXACT>(b, plan.common.row_tiles, (unsigned)(plan.common.units + plan.own.units), st);
    }
    return attend<TYPE, DP, EXACT>(b.common, plan.common, st) && attend<TYPE, DP, EXACT>(b.own, plan.own, st);
}

}  // namespace

extern "C" {

size_t lsh_select_workspace_bytes(const lsh_select_params* p) {
    size_t tiles = 0;
    return select_ok(p) ? select_bytes(p, &tiles) : 0;
}

lsh_status lsh_beam_select(const lsh_select_params* p, const void* logits_dev, const float* beam_scores_dev,
                           const uint32_t* allowed_dev, void* workspace_dev, size_t workspace_bytes, int32_t* out_beam_dev,
                           int32_t* out_word_dev, float* out_score_dev, float* out_lse_dev, void* hip_stream) {
    if (!select_ok(p) || !type_ok(p->dtype) || p->ld < p->V || !logits_dev || !beam_scores_dev || !out_beam_dev || !out_word_dev ||
        !out_score_dev || !aligned(logits_dev, type_bytes(p->dtype)))
        return LSH_ERR_INVALID_ARG;
    if (allowed_dev && p->allowed_ld != 0 && p->allowed_ld < (p->V + 31) / 32) return LSH_ERR_INVALID_ARG;
    const bool small = select_is_small(p);
    size_t tiles_bytes = 0;
    if (!workspace_dev || !aligned(workspace_dev, 256)) return LSH_ERR_INVALID_ARG;
    if (workspace_bytes < select_bytes(p, &tiles_bytes)) return LSH_ERR_WORKSPACE_TOO_SMALL;
    const int64_t R = (int64_t)p->S * p->B, pieces = row_pieces(p);
    SelArgs a{};
    a.x = logits_dev; a.ld = p->ld;
    a.allowed = reinterpret_cast<const uint8_t*>(allowed_dev); a.allowed_pitch = 4 * p->allowed_ld;
    a.scores = beam_scores_dev;
    a.V = p->V; a.B = p->B; a.N = p->N;
    a.tiles = (int)ceil_div(p->V, kSelTile);
    a.tile_max = static_cast<float*>(workspace_dev);
    a.part = reinterpret_cast<SelPart*>(static_cast<char*>(workspace_dev) + tiles_bytes);
    a.out_beam = out_beam_dev; a.out_word = out_word_dev; a.out_score = out_score_dev; a.out_lse = out_lse_dev;
    const hipStream_t st = (hipStream_t)hip_stream;
    if (small) {
        for_type(p->dtype, [&](auto type) {
            hipLaunchKernelGGL(k_select_small<decltype(type)::value>, dim3((unsigned)p->S), dim3(kSelThreads), 0, st, a);
        });
        return launched();
    }
    a.pieces = wave_pieces(p);
    a.parts = (int)ceil_div(pieces, a.pieces);
    const int64_t grid = R * ceil_div(a.parts, 4);
    if (grid > kMaxGrid) return LSH_ERR_UNSUPPORTED;
    for_type(p->dtype, [&](auto type) {
        hipLaunchKernelGGL(k_select_tiles<decltype(type)::value>, dim3((unsigned)grid), dim3(256), 0, st, a);
        hipLaunchKernelGGL(k_select_words<decltype(type)::value>, dim3((unsigned)p->S), dim3(kSelThreads), 0, st, a);
    });
    return launched();
}

size_t lsh_cache_workspace_bytes(const lsh_cache_params* c) { return cache_ok(c) ? tables_room(c).bytes : 0; }

lsh_status lsh_cache_advance(const lsh_cache_params* c, int32_t T, const int32_t* parents_dev, const int32_t* n_new_dev,
                             const int32_t* tables_in_dev, const int32_t* lengths_in_dev, int32_t* tables_out_dev,
                             int32_t* lengths_out_dev, int32_t* slots_dev, int32_t* copy_from_dev, int32_t* shared_dev,
                             int32_t* status_dev, void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
    if (!cache_ok(c) || T < 1 || T > kMaxNew || !tables_in_dev || !lengths_in_dev || !tables_out_dev || !lengths_out_dev || !slots_dev || !copy_from_dev ||
        !status_dev || tables_in_dev == tables_out_dev || lengths_in_dev == lengths_out_dev || !workspace_dev || !aligned(workspace_dev, 256))
        return LSH_ERR_INVALID_ARG;
    const TablesRoom w = tables_room(c);
    if (workspace_bytes < w.bytes) return LSH_ERR_WORKSPACE_TOO_SMALL;
    TablesArgs a{};
    a.S = c->S; a.B = c->B; a.T = T; a.n_blocks = c->n_blocks; a.block = c->block; a.width = c->max_blocks;
    a.parents = parents_dev; a.n_new = n_new_dev; a.tables_in = tables_in_dev; a.lengths_in = lengths_in_dev;
    a.tables_out = tables_out_dev; a.lengths_out = lengths_out_dev; a.slots = slots_dev; a.copy_from = copy_from_dev;
    a.shared = shared_dev; a.status = status_dev;
    char* room = static_cast<char*>(workspace_dev);
    a.plan = reinterpret_cast<RowPlan*>(room);
    a.base = reinterpret_cast<int32_t*>(room + w.base);
    a.free_ids = reinterpret_cast<int32_t*>(room + w.free_ids);
    a.used = reinterpret_cast<uint8_t*>(room + w.used);
    const hipStream_t st = (hipStream_t)hip_stream;
    const unsigned R = (unsigned)c->S * (unsigned)c->B;
    if (tables_at_once(R, c->max_blocks, c->n_blocks, T)) {
        hipLaunchKernelGGL(k_tables_once, dim3(1), dim3(1024), once_lds(R, c->n_blocks), st, a);
        return launched();
    }
    hipLaunchKernelGGL(k_tables_clear, dim3((unsigned)ceil_div(c->n_blocks, 16 * 256)), dim3(256), 0, st, a);
    hipLaunchKernelGGL(k_tables_rows, dim3(R), dim3(256), 0, st, a);
    hipLaunchKernelGGL(k_tables_take, dim3(1), dim3(1024), 0, st, a);
    hipLaunchKernelGGL(k_tables_finish, dim3(R + (shared_dev ? (unsigned)c->S : 0u)), dim3(256), 0, st, a);
    return launched();
}

lsh_status lsh_cache_write(const lsh_cache_params* c, const lsh_cache_pool* pool, int32_t T, const void* k_dev, const lsh_rows* k_rows,
                           const void* v_dev, const lsh_rows* v_rows, const int32_t* slots_dev, const int32_t* copy_from_dev, void* hip_stream) {
    if (!cache_ok(c) || !pool_ok(pool) || T < 1 || T > kMaxNew || !k_dev || !v_dev || !slots_dev || !pitch_ok(k_rows, c->head_dim) ||
        !pitch_ok(v_rows, c->head_dim) || k_rows->dtype != v_rows->dtype || !aligned(k_dev, type_bytes(k_rows->dtype)) ||
        !aligned(v_dev, type_bytes(v_rows->dtype)))
        return LSH_ERR_INVALID_ARG;
    WriteArgs a{};
    a.T = T; a.n_blocks = c->n_blocks; a.block = c->block; a.heads = c->n_heads; a.D = c->head_dim;
    a.per_row = (int)(((int64_t)T + c->block - 2) / c->block + 1);
    a.k = k_dev; a.v = v_dev;
    a.kp = RowsPitch{k_rows->row, k_rows->token, k_rows->head};
    a.vp = RowsPitch{v_rows->row, v_rows->token, v_rows->head};
    a.slots = slots_dev; a.copy_from = copy_from_dev;
    a.codes_k = pool->k; a.codes_v = pool->v; a.scale_k = pool->k_scale; a.scale_v = pool->v_scale;
    const int64_t grid = (int64_t)c->S * c->B * a.per_row;
    if (grid > kMaxGrid) return LSH_ERR_UNSUPPORTED;
    for_type(k_rows->dtype, [&](auto type) {
        auto kernel = T == 1 ? k_cache_write_one<decltype(type)::value> : k_cache_write<decltype(type)::value>;
        hipLaunchKernelGGL(kernel, dim3((unsigned)grid, (unsigned)c->n_heads), dim3(256), 0, (hipStream_t)hip_stream, a);
    });
    return launched();
}

size_t lsh_attention_workspace_bytes(const lsh_cache_params* c, const lsh_attention_params* p) {
    if (!attention_ok(c, p) || !rows_fit(c, p)) return 0;
    size_t bytes = 0;            // of any type's queries; and who has a workspace may leave `shared` out
    for (int32_t dtype : {LSH_F32, LSH_BF16})
        for (bool shared : {false, true}) {
            const AttnPlan plan = attention_plan(c, p, dtype, shared);
            if (plan.fits()) bytes = std::max(bytes, plan.bytes);
        }
    return bytes;
}

lsh_status lsh_cache_attention(const lsh_cache_params* c, const lsh_cache_pool* pool, const lsh_attention_params* p, const void* q_dev,
                               const lsh_rows* q_rows, const int32_t* tables_dev, const int32_t* lengths_dev, const int32_t* n_new_dev,
                               const int32_t* shared_dev, void* workspace_dev, size_t workspace_bytes, void* out_dev,
                               const lsh_rows* out_rows, float* lse_dev, void* hip_stream) {
    if (!attention_ok(c, p) || !pool_ok(pool) || p->window < 0 || (p->window > 0 && !p->causal) ||
        !(p->scale > 0.f && p->scale < INFINITY) || !q_dev || !tables_dev || !lengths_dev || !out_dev || !pitch_ok(q_rows, c->head_dim) || !pitch_ok(out_rows, c->head_dim) || q_rows->dtype != out_rows->dtype ||
        !aligned(q_dev, type_bytes(q_rows->dtype)) || !aligned(out_dev, type_bytes(out_rows->dtype)) || !workspace_dev ||
        !aligned(workspace_dev, 256))
        return LSH_ERR_INVALID_ARG;
    if (!rows_fit(c, p)) return LSH_ERR_UNSUPPORTED;
    if (heads_overlap(out_rows, (int64_t)c->S * c->B, p->T, p->n_heads, c->head_dim)) return LSH_ERR_INVALID_ARG;
    const AttnPlan plan = attention_plan(c, p, q_rows->dtype, shared_dev != nullptr);
    if (!plan.fits()) return LSH_ERR_UNSUPPORTED;
    const int64_t rows = query_rows(c, p);
    if (workspace_bytes < lsh_attention_workspace_bytes(c, p)) return LSH_ERR_WORKSPACE_TOO_SMALL;
    AttnArgs a{};
    a.S = c->S; a.B = c->B; a.T = p->T; a.q_heads = p->n_heads; a.heads = c->n_heads; a.D = c->head_dim;
    a.n_blocks = c->n_blocks; a.block = c->block; a.width = c->max_blocks;
    a.causal = p->causal != 0; a.window = p->window; a.scale = p->scale;
    a.q = q_dev; a.qp = RowsPitch{q_rows->row, q_rows->token, q_rows->head};
    a.codes_k = pool->k; a.codes_v = pool->v; a.scale_k = pool->k_scale; a.scale_v = pool->v_scale;
    a.tables = tables_dev; a.lengths = lengths_dev; a.n_new = n_new_dev; a.shared = shared_dev;
    a.out = out_dev; a.op = RowsPitch{out_rows->row, out_rows->token, out_rows->head};
    a.lse = lse_dev;
    a.has_common = plan.common.units > 0;
    a.parts = plan.common.splits + plan.own.splits;
    a.ml = static_cast<float2*>(workspace_dev);
    a.acc = reinterpret_cast<float*>(static_cast<char*>(workspace_dev) + plan.acc);
    BothArgs both{a, a, (unsigned)plan.common.units};
    for (int own = 0; own < 2; ++own) {
        AttnArgs& to = own ? both.own : both.common;
        const AttnLaunch& w = own ? plan.own : plan.common;
        to.common = !own;
        to.sets = own ? c->S * c->B : c->S;
        to.chunk = w.chunk; to.groups = w.groups; to.splits = w.splits;
        to.part0 = own ? plan.common.splits : 0;
    }
    const hipStream_t st = (hipStream_t)hip_stream;
    bool ok = true;
    for_type(q_rows->dtype, [&](auto type) {
        constexpr int kType = decltype(type)::value;
        const int D = c->head_dim;
        ok = D == 64    ? attend<kType, 64, true>(both, plan, st)
             : D < 64   ? attend<kType, 64, false>(both, plan, st)
             : D == 128 ? attend<kType, 128, true>(both, plan, st)
             : D < 128  ? attend<kType, 128, false>(both, plan, st)
             : D == 192 ? attend<kType, 192, true>(both, plan, st)
             : D == 256 ? attend<kType, 256, true>(both, plan, st)
                        : attend<kType, 256, false>(both, plan, st);
        if (ok && a.parts > 1) hipLaunchKernelGGL(k_attention_join<kType>, dim3((unsigned)ceil_div(rows, 4)), dim3(256), 0, st, a);
    });
    if (!ok) (void)hipGetLastError();   // (reported here, not by the caller's next call)
    return ok ? launched() : LSH_ERR_HIP;
}

}  // extern "C"
