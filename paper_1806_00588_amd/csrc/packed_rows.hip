// Few rows times weights of 4 bits: the launches of k_packed_rows.
#ifdef LSHBEAM_TRACE   // (the phase timestamps belong to the decode step's kernels)
#undef LSHBEAM_TRACE
#endif
#include "packed_launch.h"

namespace lshbeam {
namespace {

template <int TYPE, int MT, int NS, bool GATED, int WAVES, bool EIGHT> bool launch(const PackedArgs& a, dim3 grid, size_t lds, hipStream_t st) {
    if (a.shift == 5) return launch_room<k_packed_rows<TYPE, MT, NS, 1, GATED, WAVES, EIGHT>>(grid, 64 * WAVES, lds, st, a);
    if (a.shift == 6) return launch_room<k_packed_rows<TYPE, MT, NS, 2, GATED, WAVES, EIGHT>>(grid, 64 * WAVES, lds, st, a);
    return launch_room<k_packed_rows<TYPE, MT, NS, 4, GATED, WAVES, EIGHT>>(grid, 64 * WAVES, lds, st, a);
}
template <int TYPE, int MT, int NS, bool GATED, int WAVES> bool launch(const PackedArgs& a, dim3 grid, size_t lds, hipStream_t st) {
    if constexpr (kEights<TYPE>) {
        if (!a.w[0].zeros && !a.w[1].zeros) return launch<TYPE, MT, NS, GATED, WAVES, true>(a, grid, lds, st);
    }
    return launch<TYPE, MT, NS, GATED, WAVES, false>(a, grid, lds, st);
}
template <int TYPE, int MT, int WAVES> bool launch(int streams, bool gated, const PackedArgs& a, dim3 grid, size_t lds, hipStream_t st) {
    if (gated) return launch<TYPE, MT, 2, true, WAVES>(a, grid, lds, st);
    return streams == 1 ? launch<TYPE, MT, 1, false, WAVES>(a, grid, lds, st) : launch<TYPE, MT, 2, false, WAVES>(a, grid, lds, st);
}

}  // namespace

bool launch_packed_rows(int32_t dtype, int row_tiles, int waves, int streams, bool gated, const PackedArgs& a, dim3 grid, size_t lds, hipStream_t st) {
    bool ok = false;
    for_type(dtype, [&](auto type) {
        constexpr int kType = decltype(type)::value;
        ok = row_tiles == 2 ? launch<kType, 2, 8>(streams, gated, a, grid, lds, st)
             : waves == 16  ? launch<kType, 1, 16>(streams, gated, a, grid, lds, st)
                            : launch<kType, 1, 8>(streams, gated, a, grid, lds, st);
    });
    return ok;
}

}  // namespace lshbeam
