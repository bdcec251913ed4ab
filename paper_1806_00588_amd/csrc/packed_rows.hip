// Few rows times weights of 4 bits: the launches of k_packed_rows.
#ifdef LSHBEAM_TRACE   // (the phase timestamps belong to the decode step's kernels)
#undef LSHBEAM_TRACE
#endif
#include "packed_launch.h"

namespace lshbeam {
namespace {

template <int TYPE, int MT, int NS, bool GATED> bool launch(const PackedArgs& a, dim3 grid, size_t lds, hipStream_t st) {
    if (a.shift == 5) return launch_room<k_packed_rows<TYPE, MT, NS, 1, GATED>>(grid, 64 * kPackedWaves, lds, st, a);
    if (a.shift == 6) return launch_room<k_packed_rows<TYPE, MT, NS, 2, GATED>>(grid, 64 * kPackedWaves, lds, st, a);
    return launch_room<k_packed_rows<TYPE, MT, NS, 4, GATED>>(grid, 64 * kPackedWaves, lds, st, a);
}
template <int TYPE, int MT> bool launch(int streams, bool gated, const PackedArgs& a, dim3 grid, size_t lds, hipStream_t st) {
    if (gated) return streams == 2 ? launch<TYPE, MT, 2, true>(a, grid, lds, st) : launch<TYPE, MT, 4, true>(a, grid, lds, st);
    return streams == 1   ? launch<TYPE, MT, 1, false>(a, grid, lds, st)
           : streams == 2 ? launch<TYPE, MT, 2, false>(a, grid, lds, st)
                          : launch<TYPE, MT, 4, false>(a, grid, lds, st);
}

}  // namespace

bool launch_packed_rows(int32_t dtype, int row_tiles, int streams, bool gated, const PackedArgs& a, dim3 grid, size_t lds, hipStream_t st) {
    bool ok = false;
    for_type(dtype, [&](auto type) {
        constexpr int kType = decltype(type)::value;
        ok = row_tiles == 1 ? launch<kType, 1>(streams, gated, a, grid, lds, st) : launch<kType, 2>(streams, gated, a, grid, lds, st);
    });
    return ok;
}

}  // namespace lshbeam
