// Many rows times weights of 4 bits: the launches of k_packed_lay and k_packed_tiles.
#ifdef LSHBEAM_TRACE   // (the phase timestamps belong to the decode step's kernels)
#undef LSHBEAM_TRACE
#endif
#include "packed_launch.h"

namespace lshbeam {
namespace {

template <int TYPE, int NS, bool GATED, bool DEEP, bool EIGHT> bool launch(const TilesArgs& a, hipStream_t st) {
    const dim3 grid((unsigned)((a.row_groups * (int64_t)a.sets + 7) / 8 * 8), (unsigned)a.p.splits);
    constexpr size_t lds = TilesPlan<TYPE, 4, NS, DEEP>::kLds;
    if constexpr (NS < 4) {
        if (a.p.shift == 5) return launch_room<k_packed_tiles<TYPE, 4, NS, 1, GATED, DEEP, EIGHT>>(grid, 64 * kTileWaves, lds, st, a);
    }
    if (a.p.shift == 6) return launch_room<k_packed_tiles<TYPE, 4, NS, 2, GATED, DEEP, EIGHT>>(grid, 64 * kTileWaves, lds, st, a);
    return launch_room<k_packed_tiles<TYPE, 4, NS, 4, GATED, DEEP, EIGHT>>(grid, 64 * kTileWaves, lds, st, a);
}
template <int TYPE, int NS, bool GATED, bool DEEP> bool launch(const TilesArgs& a, hipStream_t st) {
    if constexpr (kEights<TYPE>) {
        if (!a.p.w[0].zeros && !a.p.w[1].zeros) return launch<TYPE, NS, GATED, DEEP, true>(a, st);
    }
    return launch<TYPE, NS, GATED, DEEP, false>(a, st);
}
template <int TYPE, bool DEEP> bool launch(int streams, bool gated, const TilesArgs& a, hipStream_t st) {
    if constexpr (DEEP) {
        if (gated) return launch<TYPE, 2, true, true>(a, st);
        return streams == 1 ? launch<TYPE, 1, false, true>(a, st) : launch<TYPE, 2, false, true>(a, st);
    } else {
        if (gated) return streams == 2 ? launch<TYPE, 2, true, false>(a, st) : launch<TYPE, 4, true, false>(a, st);
        return streams == 2 ? launch<TYPE, 2, false, false>(a, st) : launch<TYPE, 4, false, false>(a, st);
    }
}

}  // namespace

bool launch_packed_tiles(int32_t dtype, bool deep, int streams, bool gated, const TilesArgs& a, hipStream_t st) {
    bool ok = false;
    for_type(dtype, [&](auto type) {
        constexpr int kType = decltype(type)::value;
        const int64_t units = (int64_t)a.row_tiles * a.p.parts;
        if (!a.as_they_are) hipLaunchKernelGGL(k_packed_lay<kType>, dim3((unsigned)ceil_div(units, 4)), dim3(256), 0, st, a.p, const_cast<char*>(a.x),
                           units);
        ok = deep ? launch<kType, true>(streams, gated, a, st) : launch<kType, false>(streams, gated, a, st);
    });
    return ok;
}

}  // namespace lshbeam
