// Launches of the kernels for weights of 4 bits, each in a translation unit of its own: there are many of them.
#pragma once
#include "launch.h"
#include "packed_tiles.h"

namespace lshbeam {

// Type of the rows; 16 rows each of a workgroup (tiles: 64 rows, not 128); its waves; tiles of outputs of a wave.  False: refused.
bool launch_packed_rows(int32_t dtype, int row_tiles, int waves, int streams, bool gated, const PackedArgs& a, dim3 grid, size_t lds, hipStream_t st);
bool launch_packed_tiles(int32_t dtype, bool deep, int streams, bool gated, const TilesArgs& a, hipStream_t st);

}  // namespace lshbeam
