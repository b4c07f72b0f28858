// How the prefix's key tiles are dealt out to the CTAs of the tensor-core kernel; the same arithmetic on the host, in that
// kernel and where the parts are joined.
#pragma once

#include <cuda_runtime.h>

namespace rt {

constexpr int kTcTile = 128;       // keys per tile, and rows per stream
constexpr int kTcBlockRows = 256;  // rows per unit

struct PrefixSplit {
    int tiles;   // key tiles of the prefix
    int blocks;  // row blocks per key/value head; unit = key/value head * blocks + block
    int rows;    // rows per key/value head
    int run;     // consecutive tiles (numbered through over all units) per CTA; 0: the tensor-core kernel is not used
};

// Blocks of up to 128 rows are served by both streams of a CTA, which leave a part each.
__host__ __device__ __forceinline__ bool narrow_block(const PrefixSplit& s, int block) { return s.rows - block * kTcBlockRows <= kTcTile; }
__host__ __device__ __forceinline__ int parts_of_unit(const PrefixSplit& s, int unit, int block)
{
    const long long first = (long long)unit * s.tiles / s.run, last = ((long long)(unit + 1) * s.tiles - 1) / s.run;
    return (int)(last - first + 1) * (narrow_block(s, block) ? 2 : 1);
}
// No unit has more.
__host__ __device__ __forceinline__ int most_parts(const PrefixSplit& s)
{
    return ((s.tiles - 1) / s.run + 2) * (narrow_block(s, s.blocks - 1) ? 2 : 1);
}

}  // namespace rt
