// Where the paged attention keeps a row's scores for the weights' kernel (no CUDA
// needed: host code can ask too).
#pragma once

#include <cstdint>

#ifdef __CUDACC__
#define PRISM_HD __host__ __device__ __forceinline__
#else
#define PRISM_HD inline
#endif

namespace prism {

// Scores [B, Hkv, G / tile, rows, heads of the tile] as fp32, rows = the block
// table's; the place of row 0 and head h0, the first of a tile, of KV head kvh.
PRISM_HD long long score_place(int b, int kvh, int h0, int Hkv, int G, long long rows) {
    return (((long long)b * Hkv + kvh) * G + h0) * rows;
}

// Whether the scores of heads h and h + 1, h even, of every row of a tile may be
// stored as eight bytes: `first` (of row 0 and the tile's first head) and the rows'
// distance are even.  G and the table's rows odd make every other `first` odd, also
// of a tile of 16 heads.
PRISM_HD bool score_pairs(const float *first, int heads) {
    return ((uintptr_t)first & 7u) == 0 && (heads & 1) == 0;
}

}  // namespace prism
