// C ABI of a decoder's layers (see include/lshbeam.h): weights of 4 bits and rows times them, the gated delta rule.  Host side: argument
// validation, the choice of kernels, launches.  A translation unit, and so a code object, of its own, like the others.
#ifdef LSHBEAM_TRACE   // (the phase timestamps belong to the decode step's kernels)
#undef LSHBEAM_TRACE
#endif
#include "delta_chunks.h"
#include "launch.h"
#include "packed_launch.h"
#include "packed_tiles.h"

using namespace lshbeam;

namespace {

// ---- weights of 4 bits --------------------------------------------------------------------------

constexpr int kMaxOutputs = 1 << 24, kMaxInputs = 1 << 20;

bool packed_ok(const lsh_packed_params* p) {
    return p && p->N >= 1 && p->N <= kMaxOutputs && p->K >= 1 && p->K <= kMaxInputs && (p->group == 32 || p->group == 64 || p->group == 128);
}
bool weights_ok(const lsh_packed_weights* w) {
    return w && w->codes && w->scales && aligned(w->codes, 16) && aligned(w->scales, 16) && aligned(w->zeros, 16) &&
           (w->scale_dtype == LSH_BF16 || w->scale_dtype == LSH_F16);
}
bool matrix_ok(const void* at, const lsh_matrix* m, int32_t columns) {
    return at && m && type_ok(m->dtype) && m->ld >= columns && aligned(at, type_bytes(m->dtype));
}
int log2_of(int32_t group) { return group == 32 ? 5 : group == 64 ? 6 : 7; }
int64_t tiles_of(const lsh_packed_params* p) { return ceil_div(p->N, kPackOutputs); }
int64_t parts_of(const lsh_packed_params* p) { return ceil_div(p->K, kPackInputs); }
PackedRef ref(const lsh_packed_weights* w) { return PackedRef{w->codes, static_cast<uint16_t*>(w->scales), w->zeros}; }

bool quantize_args(const lsh_packed_params* p, const lsh_packed_weights* w, const void* x, int64_t ld, QuantArgs* a) {
    a->N = p->N; a->K = p->K; a->parts = (int)parts_of(p); a->shift = log2_of(p->group);
    a->units = tiles_of(p) * parts_of(p);
    a->w = x; a->ld = ld; a->to = ref(w);
    return ceil_div(a->units, 4) <= kMaxGrid;
}

// How few rows' products are divided among workgroups.
struct RowsPlan {
    int groups, rows, row_tiles;   // of rows
    int waves, streams;            // tiles of a wave (gated: of both matrices)
    int log_across, chunk, turns;
    int64_t sets;
    unsigned grid;                 // workgroups of a group of rows
    size_t lds;
    int join_at;
    int splits, split_parts;       // of the inputs
};
constexpr int kFewRows = 32;
RowsPlan rows_plan(const lsh_packed_params* p, int32_t M, int32_t dtype, bool gated) {
    RowsPlan w{};
    w.groups = (int)ceil_div(M, kFewRows);
    w.rows = (int)ceil_div(M, w.groups);
    w.row_tiles = (int)ceil_div(w.rows, 16);
    const int64_t tiles = tiles_of(p), parts = parts_of(p), planes = dtype == LSH_F32 ? 3 : 1;
    w.waves = w.row_tiles == 1 && tiles * parts > 8 * 256 ? 16 : 8;
    // waves side by side or on the same outputs, and how many tiles each: what the rounds of 256 workgroups come to, in units of 10 ns -- a wave's tile 40 a
    // part (fp32 57), its rows' operands 10 a part and plane, adding up and the results 65 a round, rows to LDS 1 for 400 bytes of operands, in every round
    // if they do not all stay there (fitted to 12 rows of fp32 x 40000 x 1000 and of bf16 x 4096 x 4096; of ten divisions each it
    // takes the quickest, 14.9 us of up to 26.0 and 7.7 of up to 12.1)
    const size_t of_part = planes * packed_plane(w.rows, 1);
    int64_t best = INT64_MAX;
    for (int each = 1; each <= (gated ? 1 : 2); each *= 2)
        for (int lg = 0; (w.row_tiles * each << lg) <= w.waves; ++lg) {
            const int64_t sets = ceil_div(tiles, (int64_t)each << lg), rounds = ceil_div(sets * w.groups, 256), streams = gated ? 2 * each : each;
            const bool stay = parts * of_part + 2 * packed_join(w.waves, w.row_tiles, (int)streams) <= kMaxDynLds;
            const int64_t cost = rounds * (ceil_div(parts, w.waves >> lg) * w.row_tiles * ((planes == 3 ? 57 : 40) * streams + 10 * planes) + 65) +
                                 (stay ? 1 : rounds) * w.rows * parts * planes * 256 / 400;
            if (cost < best) { best = cost; w.streams = (int)streams; w.log_across = lg; w.sets = sets; }
        }
    const int deep = w.waves >> w.log_across;
    // few workgroups that go through many parts: the parts are split (a launch more, some 3 us; 16 rows x 1000 x 16384 in fp16 24.5 -> 12.5 us)
    const int64_t turns = ceil_div(parts, deep), wide = w.sets * w.groups;
    w.split_parts = (int)parts;
    if (turns >= 6 && wide <= 128) w.split_parts = (int)(ceil_div(turns, std::min(turns / 2, 256 / wide)) * deep);
    w.splits = (int)ceil_div(parts, w.split_parts);
    const int64_t of_split = w.split_parts;
    // all rows in LDS, or as many of their parts as there is room for
    const size_t join = 2 * packed_join(w.waves, w.row_tiles, w.streams);
    const int64_t chunks = ceil_div(of_split, (int64_t)((kMaxDynLds - join) / of_part));
    int64_t chunk = ceil_div(of_split, chunks);
    if (chunks > 1 && chunk > deep) chunk = chunk / deep * deep;
    w.chunk = (int)chunk;
    w.turns = (int)ceil_div(chunk, deep);
    // (who has all rows goes on to further outputs)
    w.grid = (unsigned)(chunks > 1 ? w.sets : std::min<int64_t>(w.sets, std::max(1, 256 / w.groups)));
    w.join_at = (int)(chunk * of_part);
    w.lds = w.join_at + join;
    return w;
}

// More rows: 64 or 128 of them and 64, 128 or 256 outputs a workgroup, whatever makes the least work of the rounds of 256 workgroups.
struct TilesLaunch {
    bool deep;                 // 64 rows
    int streams, row_tiles, row_groups;
    int64_t sets;
    int splits, split_parts;   // of the inputs
    size_t room;               // the rows as operands
};
// From how many rows on k_packed_tiles is quicker than k_packed_rows goes by the matrix (us of the one and the other, in a graph).  Large ones: 16384 x 4096 gated,
// bf16, 24, 32 and 40 rows 28.5 and 29.0 and 30.1 against 28.4 and 31.6 and 49.8; fp32, 17, 32 and 33 rows 51 and 54 and 52 against 39 and 58 and 74; 40000 x 1000 in fp32, 17, 32, 33 and 40 rows
// 42 and 44 and 45 and 47 against 22 and 38 and 33 and 48.  With few parts, where there is little to go through between the first load and the results, 16-bit rows never: 40000 x 1000 in
// bf16, 40 and 128 rows 33 and 50 against 24 and 44 (40000 x 2048, 40 and 64 rows: 38 and 42 against 31 and 54).  Small ones do not pay for the rounds: 2048 x 2048 in bf16, 64 rows, 14.9 against 8.0.
// But rows of many parts do not stay in LDS: 1000 x 16384 in fp16, 24, 32 and 96 rows 15.3 and 15.6 and 19.2 against 16.9 and 19.1 and 53; fp32, 20 and 40 rows 24 and 24 against 26 and 47.
bool takes_tiles(const lsh_packed_params* p, int32_t M, int32_t dtype, bool gated) {
    const int64_t parts = parts_of(p), work = tiles_of(p) * parts * (gated ? 2 : 1);
    return M > 128 || (M > kFewRows && work >= 16384 && (dtype == LSH_F32 || parts >= 16)) || (M > (dtype == LSH_F32 ? kFewRows : 24) && parts > 48);
}
size_t tiles_room(const lsh_packed_params* p, int32_t M, int32_t dtype) {
    return round_up((size_t)ceil_div(M, 16) * parts_of(p) * 4 * 1024 * (dtype == LSH_F32 ? 3 : 1));
}
TilesLaunch tiles_plan(const lsh_packed_params* p, int32_t M, int32_t dtype, bool gated) {
    TilesLaunch w{};
    w.row_tiles = (int)ceil_div(M, 16);
    // (a part of 16 x 16 results of a wave some 16 ns on the matrix cores and beside them, of three planes 48; 250 for the rest of it)
    int64_t best = INT64_MAX;
    for (int deep = 0; deep < 2; ++deep)
        for (int streams = 4; streams >= (gated || !deep ? 2 : 1); streams /= 2) {
            if (streams == 4 && (deep || p->group == 32)) continue;     // (no LDS for twice as many codes; no registers for four groups of a part)
            const int64_t groups = ceil_div(w.row_tiles, deep ? 4 : 8), sets = ceil_div(tiles_of(p), kTileAcross * (gated ? streams / 2 : streams));
            const int64_t cost = ceil_div(groups * sets, 256) * (4 * streams * (dtype == LSH_F32 ? 48 : 16) + 250) / (deep ? 2 : 1);
            if (cost < best) { best = cost; w.deep = deep != 0; w.streams = streams; w.row_groups = (int)groups; w.sets = sets; }
        }
    const int64_t halves = w.deep ? 2 : 1, turns = ceil_div(parts_of(p), halves), wide = w.sets * w.row_groups;
    w.split_parts = (int)(turns * halves);
    if (w.deep && turns >= 12 && wide <= 128) w.split_parts = (int)(ceil_div(turns, std::min(turns / 4, 256 / wide)) * halves);
    w.splits = (int)ceil_div(parts_of(p), w.split_parts);
    w.room = tiles_room(p, M, dtype);
    return w;
}

// Are there workgroups enough to lay out the rows?
bool packed_fits(const lsh_packed_params* p, int32_t M) { return ceil_div(ceil_div(M, 16) * parts_of(p), 4) <= kMaxGrid; }
// What a call needs of the workspace: the rows as operands, and the sums of parts.
size_t packed_need(const lsh_packed_params* p, int32_t M, bool many, bool gated, const RowsPlan& w, const TilesLaunch& tiles) {
    const int splits = many ? tiles.splits : w.splits;
    return (many ? tiles.room : 0) + (splits > 1 ? (size_t)splits * (gated ? 2 : 1) * M * p->N * sizeof(float) : 0);
}
// At most that, for these rows or fewer, of any type, of one matrix or two.  Six parts and more are split where `wide` workgroups are 128 at most, into no more than parts / 2
// and 256 / wide pieces, and a workgroup has 8192 sums at most: 16 tiles of 16 x 16 of each matrix in k_packed_rows, 64 x 128 altogether in k_packed_tiles.
size_t packed_most(const lsh_packed_params* p, int32_t M) {
    size_t room = 0;
    for (int32_t dtype : {LSH_F32, LSH_BF16, LSH_F16})
        for (bool gated : {false, true})
            if (takes_tiles(p, M, dtype, gated)) room = std::max(room, tiles_room(p, M, dtype));
    const size_t sums = parts_of(p) < 6 ? 0 : std::min((size_t)(parts_of(p) / 2) * 2 * M * p->N, (size_t)1 << 21);
    return std::max<size_t>(256, room + sums * sizeof(float));
}

lsh_status packed_product(const lsh_packed_params* p, const lsh_packed_weights* const (&weights)[2], int32_t M, const void* x_dev, const lsh_matrix* x,
                          const float* bias_dev, const void* add_dev, int64_t add_ld, int32_t activation, void* workspace_dev, size_t workspace_bytes,
                          void* out_dev, const lsh_matrix* out, void* hip_stream) {
    const bool gated = weights[1] != nullptr;
    if (!packed_ok(p) || !weights_ok(weights[0]) || M < 1 || M > kMaxRows || !matrix_ok(x_dev, x, p->K) || !matrix_ok(out_dev, out, p->N) ||
        !aligned(bias_dev, 4) || (add_dev && (add_ld < p->N || !aligned(add_dev, type_bytes(out->dtype)))) || !workspace_dev || !aligned(workspace_dev, 256))
        return LSH_ERR_INVALID_ARG;
    const bool many = takes_tiles(p, M, x->dtype, gated);
    const RowsPlan w = rows_plan(p, M, x->dtype, gated);
    const TilesLaunch tiles = tiles_plan(p, M, x->dtype, gated);
    if (!packed_fits(p, M) || (many ? tiles.sets * tiles.row_groups > kMaxGrid / 2 : w.grid > kMaxGrid / 4)) return LSH_ERR_UNSUPPORTED;
    if (workspace_bytes < std::max(packed_most(p, M), packed_need(p, M, many, gated, w, tiles))) return LSH_ERR_WORKSPACE_TOO_SMALL;
    PackedArgs a{};
    a.M = M; a.N = p->N; a.K = p->K; a.tiles = (int)tiles_of(p); a.parts = (int)parts_of(p);
    a.shift = log2_of(p->group);
    a.scale_f16 = weights[0]->scale_dtype == LSH_F16;
    a.x = x_dev; a.ldx = x->ld;
    a.w[0] = ref(weights[0]);
    if (gated) a.w[1] = ref(weights[1]);
    a.bias = bias_dev; a.add = add_dev; a.ld_add = add_ld;
    a.out = out_dev; a.ld_out = out->ld; a.out_type = out->dtype == LSH_F32 ? kTypeF32 : out->dtype == LSH_BF16 ? kTypeBf16 : kTypeF16;
    a.activation = activation;
    a.rows = w.rows; a.log_across = w.log_across; a.chunk = w.chunk; a.turns = w.turns; a.sets = (int)w.sets; a.join_at = w.join_at;
    a.splits = many ? tiles.splits : w.splits; a.split_parts = many ? tiles.split_parts : w.split_parts;
    char* room = static_cast<char*>(workspace_dev);
    a.partial = reinterpret_cast<float*>(room + (many ? tiles.room : 0));
    const hipStream_t st = (hipStream_t)hip_stream;
    bool ok = false;
    if (many) {
        const bool as_they_are = x->dtype != LSH_F32 && p->K % kPackInputs == 0 && x->ld % 8 == 0 && aligned(x_dev, 16);   // (16 bytes at a time)
        const TilesArgs t{a, as_they_are, room, tiles.row_tiles, tiles.row_groups, (int)tiles.sets};
        ok = launch_packed_tiles(x->dtype, tiles.deep, tiles.streams, gated, t, st);
    } else ok = launch_packed_rows(x->dtype, w.row_tiles, w.waves, w.streams, gated, a, dim3(w.grid, (unsigned)w.groups, (unsigned)w.splits), w.lds, st);
    if (ok && a.splits > 1) {
        const unsigned grid = (unsigned)ceil_div((int64_t)M * p->N, 256);
        if (gated) hipLaunchKernelGGL(k_packed_join<true>, dim3(grid), dim3(256), 0, st, a);
        else hipLaunchKernelGGL(k_packed_join<false>, dim3(grid), dim3(256), 0, st, a);
    }
    if (!ok) (void)hipGetLastError();   // (reported here, not by the caller's next call)
    return ok ? launched() : LSH_ERR_HIP;
}

// ---- gated delta rule ---------------------------------------------------------------------------

bool delta_ok(const lsh_delta_params* p) {
    return p && p->S >= 1 && p->B >= 1 && p->B <= 256 && (int64_t)p->S * p->B <= kMaxRows && p->T >= 1 && p->T <= kMaxRows && p->n_k_heads >= 1 &&
           p->n_heads >= 1 && p->n_heads <= 65535 && p->n_heads % p->n_k_heads == 0 && p->k_dim >= 16 && p->k_dim <= 256 && p->k_dim % 16 == 0 &&
           p->v_dim >= 16 && p->v_dim <= 256 && p->v_dim % 16 == 0;
}
int64_t delta_slices(const lsh_delta_params* p) { return ceil_div(p->v_dim, kDeltaColumns); }
int64_t delta_pairs(const lsh_delta_params* p) { return (int64_t)p->S * p->B * p->n_heads; }
bool delta_fits(const lsh_delta_params* p) {
    return delta_pairs(p) <= kMaxGrid && delta_pairs(p) * p->T <= (int64_t)1 << 26 && ceil_div(delta_pairs(p), 8) * 8 * (p->v_dim / 16) <= kMaxGrid;
}
// Rows of more tokens than this go in chunks of 64 (16 pairs of 128 x 128, bf16, 8 and 16 tokens: token after token 12.6 and 21.4 us, a chunk 17.4; 512 pairs,
// 16 and 24 tokens: 44 and 59 against 55 and 57).
constexpr int kLeastChunked = 12;
int most_tokens(const lsh_delta_params* p) { return delta_pairs(p) * delta_slices(p) <= 256 ? kLeastChunked : 20; }

// The chunks' operands take turns in the workspace: as many pairs of a row and a head and as many of their chunks at a time as have room.
struct ChunksPlan {
    size_t of_chunk, bytes;
    int64_t pairs;             // of a launch
    int chunks;                // of a segment
};
constexpr size_t kChunksRoom = (size_t)256 << 20;
template <typename F> void for_dims(int32_t dim, F f) {   // f(std::integral_constant<int, ceil(k_dim / 32)>), some of them rounded up
    const int nk = (dim + 31) / 32;
    if (nk == 1) f(std::integral_constant<int, 1>());
    else if (nk == 2) f(std::integral_constant<int, 2>());
    else if (nk == 3) f(std::integral_constant<int, 3>());
    else if (nk == 4) f(std::integral_constant<int, 4>());
    else if (nk <= 6) f(std::integral_constant<int, 6>());
    else f(std::integral_constant<int, 8>());
}
size_t bytes_of_chunk(const lsh_delta_params* p, int32_t dtype) {
    size_t bytes = 0;
    for_type(dtype, [&](auto type) {
        for_dims(p->k_dim, [&](auto nk) { bytes = ChunkPlan<decltype(type)::value, decltype(nk)::value>::kBlocks * 1024; });
    });
    return bytes;
}
ChunksPlan chunks_plan(const lsh_delta_params* p, int32_t dtype) {
    ChunksPlan w{};
    w.of_chunk = bytes_of_chunk(p, dtype);
    const int64_t most = std::max<int64_t>(1, kChunksRoom / w.of_chunk), all = ceil_div(p->T, kChunk);
    w.pairs = std::min(most, delta_pairs(p));
    w.chunks = (int)std::min(std::max<int64_t>(1, most / w.pairs), all);
    w.bytes = w.of_chunk * (size_t)w.pairs * w.chunks;
    return w;
}
// At most that, for these rows and tokens or fewer, of any type.
size_t chunks_most(const lsh_delta_params* p) {
    size_t bytes = 256;
    if (p->T > kLeastChunked)
        for (int32_t dtype : {LSH_F32, LSH_BF16, LSH_F16}) {
            const size_t of_chunk = bytes_of_chunk(p, dtype), most = std::max<size_t>(1, kChunksRoom / of_chunk);
            bytes = std::max(bytes, of_chunk * std::min<size_t>(most, delta_pairs(p) * ceil_div(p->T, kChunk)));
        }
    return bytes;
}
template <int TYPE, int NK> bool chunks_launch(const lsh_delta_params* p, const DeltaArgs& d, const ChunksPlan& w, char* room, hipStream_t st) {
    ChunkArgs a{};
    a.d = d; a.room = room; a.bytes = w.of_chunk;
    const int all = (int)ceil_div(p->T, kChunk);
    for (int64_t pair = 0; pair < delta_pairs(p); pair += w.pairs) {
        const int64_t pairs = std::min(w.pairs, delta_pairs(p) - pair);
        a.pair0 = pair; a.pairs = pairs;
        for (int chunk = 0; chunk < all; chunk += w.chunks) {
            a.chunk0 = chunk;
            a.chunks = std::min(w.chunks, all - chunk);
            a.first = chunk == 0;
            if (!launch_room<k_delta_prepare<TYPE, NK>>(dim3((unsigned)(pairs * a.chunks)), 256, kPrepareLds<TYPE, NK>, st, a)) return false;
            const auto grid = [&](int tiles) { return dim3((unsigned)(ceil_div(pairs, 8) * 8 * ceil_div(p->v_dim / 16, tiles))); };
            constexpr int kMine = (NK + 3) / 4 * ChunkPlan<TYPE, NK>::P;      // (what there are registers for)
            if (grid(1).x <= 512) {
                if constexpr (kMine <= 3) hipLaunchKernelGGL((k_delta_apart<TYPE, NK, kMine == 1 ? 2 : 1>), grid(1), dim3(512), 0, st, a);
                else hipLaunchKernelGGL((k_delta_chain<TYPE, NK, true, 1>), grid(1), dim3(256), 0, st, a);
            } else hipLaunchKernelGGL((k_delta_chain<TYPE, NK, false, 2>), grid(2), dim3(256), 0, st, a);
        }
    }
    return true;
}
bool rows_aligned(const void* at, const lsh_rows* x, int32_t dim) { return at && pitch_ok(x, dim) && aligned(at, type_bytes(x->dtype)); }

}  // namespace

extern "C" {

lsh_status lsh_packed_quantize(const lsh_packed_params* p, const void* w_dev, const lsh_matrix* w, const lsh_packed_weights* to, void* hip_stream) {
    if (!packed_ok(p) || !weights_ok(to) || !matrix_ok(w_dev, w, p->K)) return LSH_ERR_INVALID_ARG;
    QuantArgs a{};
    if (!quantize_args(p, to, w_dev, w->ld, &a)) return LSH_ERR_UNSUPPORTED;
    const hipStream_t st = (hipStream_t)hip_stream;
    for_type(w->dtype, [&](auto type) {
        constexpr int kType = decltype(type)::value;
        const bool f16 = to->scale_dtype == LSH_F16;
        auto kernel = f16 ? (to->zeros ? k_packed_quantize<kType, true, true> : k_packed_quantize<kType, true, false>)
                          : (to->zeros ? k_packed_quantize<kType, false, true> : k_packed_quantize<kType, false, false>);
        hipLaunchKernelGGL(kernel, dim3((unsigned)ceil_div(a.units, 4)), dim3(256), 0, st, a);
    });
    return launched();
}

lsh_status lsh_packed_values(const lsh_packed_params* p, const lsh_packed_weights* from, void* out_dev, const lsh_matrix* out, void* hip_stream) {
    if (!packed_ok(p) || !weights_ok(from) || !matrix_ok(out_dev, out, p->K)) return LSH_ERR_INVALID_ARG;
    QuantArgs a{};
    if (!quantize_args(p, from, out_dev, out->ld, &a)) return LSH_ERR_UNSUPPORTED;
    for_type(out->dtype, [&](auto type) {
        constexpr int kType = decltype(type)::value;
        auto kernel = from->scale_dtype == LSH_F16 ? k_packed_values<kType, true> : k_packed_values<kType, false>;
        hipLaunchKernelGGL(kernel, dim3((unsigned)ceil_div(a.units, 4)), dim3(256), 0, (hipStream_t)hip_stream, a);
    });
    return launched();
}

size_t lsh_packed_workspace_bytes(const lsh_packed_params* p, int32_t M) {
    return packed_ok(p) && M >= 1 && M <= kMaxRows && packed_fits(p, M) ? packed_most(p, M) : 0;
}

lsh_status lsh_packed_linear(const lsh_packed_params* p, const lsh_packed_weights* w, int32_t M, const void* x_dev, const lsh_matrix* x,
                             const float* bias_dev, const void* add_dev, int64_t add_ld, void* workspace_dev, size_t workspace_bytes,
                             void* out_dev, const lsh_matrix* out, void* hip_stream) {
    return packed_product(p, {w, nullptr}, M, x_dev, x, bias_dev, add_dev, add_ld, 0, workspace_dev, workspace_bytes, out_dev, out, hip_stream);
}

lsh_status lsh_packed_gated(const lsh_packed_params* p, const lsh_packed_weights* gate, const lsh_packed_weights* up, int32_t M,
                            const void* x_dev, const lsh_matrix* x, int32_t activation, void* workspace_dev, size_t workspace_bytes,
                            void* out_dev, const lsh_matrix* out, void* hip_stream) {
    if (!weights_ok(gate) || !weights_ok(up) || gate->scale_dtype != up->scale_dtype || activation < LSH_SILU || activation > LSH_GELU_TANH)
        return LSH_ERR_INVALID_ARG;
    return packed_product(p, {gate, up}, M, x_dev, x, nullptr, nullptr, 0, activation, workspace_dev, workspace_bytes, out_dev, out, hip_stream);
}

size_t lsh_delta_workspace_bytes(const lsh_delta_params* p) {
    return delta_ok(p) && delta_fits(p) ? chunks_most(p) : 0;
}

lsh_status lsh_delta_rule(const lsh_delta_params* p, const void* q_dev, const lsh_rows* q_rows, const void* k_dev, const lsh_rows* k_rows,
                          const void* v_dev, const lsh_rows* v_rows, const float* decay_dev, const float* beta_dev,
                          const float* state_in_dev, const int32_t* parents_dev, const int32_t* n_new_dev, float* state_out_dev,
                          void* workspace_dev, size_t workspace_bytes, void* out_dev, const lsh_rows* out_rows, void* hip_stream) {
    if (!delta_ok(p) || !(p->scale > -INFINITY && p->scale < INFINITY) || !rows_aligned(q_dev, q_rows, p->k_dim) || !rows_aligned(k_dev, k_rows, p->k_dim) ||
        !rows_aligned(v_dev, v_rows, p->v_dim) || !rows_aligned(out_dev, out_rows, p->v_dim) || q_rows->dtype != k_rows->dtype ||
        q_rows->dtype != v_rows->dtype || q_rows->dtype != out_rows->dtype || !decay_dev || !beta_dev || !aligned(decay_dev, 4) || !aligned(beta_dev, 4) ||
        !state_out_dev || !aligned(state_out_dev, 16) || !aligned(state_in_dev, 16) || !aligned(parents_dev, 4) || !aligned(n_new_dev, 4) ||
        !workspace_dev || !aligned(workspace_dev, 256))
        return LSH_ERR_INVALID_ARG;
    if (!delta_fits(p)) return LSH_ERR_UNSUPPORTED;
    const int64_t R = (int64_t)p->S * p->B;
    if (state_in_dev) {   // a state is read by workgroups of other rows, unless each row continues its own
        const uintptr_t in = reinterpret_cast<uintptr_t>(state_in_dev), to = reinterpret_cast<uintptr_t>(state_out_dev);
        const uintptr_t size = (uintptr_t)(R * p->n_heads) * p->k_dim * p->v_dim * sizeof(float);
        if (in < to + size && to < in + size && (parents_dev || in != to)) return LSH_ERR_INVALID_ARG;
    }
    if (heads_overlap(out_rows, R, p->T, p->n_heads, p->v_dim)) return LSH_ERR_INVALID_ARG;
    const bool chunked = p->T > most_tokens(p);
    const ChunksPlan w = chunks_plan(p, q_rows->dtype);
    if (workspace_bytes < std::max(chunks_most(p), chunked ? w.bytes : 0)) return LSH_ERR_WORKSPACE_TOO_SMALL;
    DeltaArgs a{};
    a.S = p->S; a.B = p->B; a.T = p->T; a.heads = p->n_heads; a.k_heads = p->n_k_heads; a.Dk = p->k_dim; a.Dv = p->v_dim;
    a.scale = p->scale;
    a.q = q_dev; a.k = k_dev; a.v = v_dev;
    a.qp = RowsPitch{q_rows->row, q_rows->token, q_rows->head};
    a.kp = RowsPitch{k_rows->row, k_rows->token, k_rows->head};
    a.vp = RowsPitch{v_rows->row, v_rows->token, v_rows->head};
    a.decay = decay_dev; a.beta = beta_dev; a.state_in = state_in_dev; a.parents = parents_dev; a.n_new = n_new_dev;
    a.state_out = state_out_dev;
    a.out = out_dev; a.op = RowsPitch{out_rows->row, out_rows->token, out_rows->head};
    a.slices = (int)delta_slices(p);
    const hipStream_t st = (hipStream_t)hip_stream;
    bool ok = true;
    for_type(q_rows->dtype, [&](auto type) {
        constexpr int kType = decltype(type)::value;
        if (chunked) {
            for_dims(p->k_dim, [&](auto nk) { ok = chunks_launch<kType, decltype(nk)::value>(p, a, w, static_cast<char*>(workspace_dev), st); });
            return;
        }
        const auto pick = [&](auto one) {
            constexpr bool kOne = decltype(one)::value;
            const int rows = p->k_dim / 16;
            return rows <= 2   ? k_delta_tokens<kType, 2, kOne>
                   : rows <= 4 ? k_delta_tokens<kType, 4, kOne>
                   : rows <= 6 ? k_delta_tokens<kType, 6, kOne>
                   : rows <= 8 ? k_delta_tokens<kType, 8, kOne>
                   : rows <= 12 ? k_delta_tokens<kType, 12, kOne>
                                : k_delta_tokens<kType, 16, kOne>;
        };
        auto kernel = p->T == 1 ? pick(std::true_type()) : pick(std::false_type());
        hipLaunchKernelGGL(kernel, dim3((unsigned)(delta_pairs(p) * a.slices)), dim3(256), 0, st, a);
    });
    if (!ok) (void)hipGetLastError();   // (reported here, not by the caller's next call)
    return ok ? launched() : LSH_ERR_HIP;
}

}  // extern "C"
