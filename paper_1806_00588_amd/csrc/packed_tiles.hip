// Many rows times weights of 4 bits: the launches of k_packed_lay and k_packed_tiles.
#ifdef LSHBEAM_TRACE   // (the phase timestamps belong to the decode step's kernels)
#undef LSHBEAM_TRACE
#endif
#include "packed_launch.h"

namespace lshbeam {
namespace {

template <int TYPE, int MT, int NS, bool GATED> bool launch(const TilesArgs& a, hipStream_t st) {
    const dim3 grid((unsigned)((a.row_groups * (int64_t)a.sets + 7) / 8 * 8));
    constexpr size_t lds = TilesPlan<TYPE, MT, NS>::kLds;
    if constexpr (MT * NS < 16) {
        if (a.p.shift == 5) return launch_room<k_packed_tiles<TYPE, MT, NS, 1, GATED>>(grid, 64 * kTileWaves, lds, st, a);
    }
    if (a.p.shift == 6) return launch_room<k_packed_tiles<TYPE, MT, NS, 2, GATED>>(grid, 64 * kTileWaves, lds, st, a);
    return launch_room<k_packed_tiles<TYPE, MT, NS, 4, GATED>>(grid, 64 * kTileWaves, lds, st, a);
}
template <int TYPE, int MT> bool launch(int streams, bool gated, const TilesArgs& a, hipStream_t st) {
    if (gated) return streams == 2 ? launch<TYPE, MT, 2, true>(a, st) : launch<TYPE, MT, 4, true>(a, st);
    if constexpr (MT == 2) {
        if (streams == 1) return launch<TYPE, MT, 1, false>(a, st);
    }
    return streams == 2 ? launch<TYPE, MT, 2, false>(a, st) : launch<TYPE, MT, 4, false>(a, st);
}

}  // namespace

bool launch_packed_tiles(int32_t dtype, int wave_rows, int streams, bool gated, const TilesArgs& a, hipStream_t st) {
    bool ok = false;
    for_type(dtype, [&](auto type) {
        constexpr int kType = decltype(type)::value;
        const int64_t units = (int64_t)a.row_tiles * a.p.parts;
        hipLaunchKernelGGL(k_packed_lay<kType>, dim3((unsigned)ceil_div(units, 4)), dim3(256), 0, st, a.p, const_cast<char*>(a.x),
                           reinterpret_cast<float*>(const_cast<char*>(a.sums)), units);
        ok = wave_rows == 4 ? launch<kType, 4>(streams, gated, a, st) : launch<kType, 2>(streams, gated, a, st);
    });
    return ok;
}

}  // namespace lshbeam
