// Where the rows of a packed cache lie inside a tile of 64 (include/mulo.h says the same in elements).
#pragma once
#include "mulo_internal.h"

namespace mulo {

constexpr int FP4 = 0, FP8 = 1;

// Places in bytes behind the start of the tile.
template <int FMT, int DH> struct Tile {
    static constexpr int ROW = FMT == FP4 ? DH / 2 : DH;                 // bytes of a row's codes
    static constexpr int G = DH / PACKED_GROUP, CODES = PACKED_TILE * ROW, BYTES = CODES + PACKED_TILE * G;
    static constexpr int UNIT = ROW / 16;                                // bytes of the values of one row that lie together
    static __host__ __device__ constexpr int k_scale(int r, int g) { return CODES + ((r & 15) * G + g) * 4 + (r >> 4); }
    static __host__ __device__ constexpr int v_code(int r, int unit) { return (r >> 2) * 4 * ROW + unit * 4 * UNIT + (r & 3) * UNIT; }
    static __host__ __device__ constexpr int v_scale(int r, int g) { return CODES + (((r >> 2 & 3) * G + g) * 4 + (r >> 4)) * 4 + (r & 3); }
};

}  // namespace mulo
