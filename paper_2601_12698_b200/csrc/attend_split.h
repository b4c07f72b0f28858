// How the prefix is dealt out to the CTAs of the tensor-core kernel; the same arithmetic on the host, in that kernel and where
// the parts are joined.
#pragma once

#include <cuda_runtime.h>

namespace rt {

constexpr int kTcTile = 128;       // keys per tile, and rows per stream
constexpr int kTcBlockRows = 256;  // rows per CTA

// A CTA takes one key/value head, one block of its rows and one run of key tiles.  CTAs are numbered with the block fastest: those
// that read the same tiles run at the same time and share them in L2 (numbered the other way, a prefix of 32768 tokens for 1024
// rows per key/value head was read from memory almost four times, 504 MB instead of 137).
struct PrefixSplit {
    int tiles;   // key tiles of the prefix
    int blocks;  // row blocks per key/value head
    int rows;    // rows per key/value head
    int run;     // tiles per CTA; 0: the tensor-core kernel is not used
    int runs;    // CTAs per key/value head and block
};

// Blocks of up to 128 rows are served by both streams of a CTA, which leave a part each.
__host__ __device__ __forceinline__ bool narrow_block(const PrefixSplit& s, int block) { return s.rows - block * kTcBlockRows <= kTcTile; }
__host__ __device__ __forceinline__ int parts_of_block(const PrefixSplit& s, int block) { return s.runs * (narrow_block(s, block) ? 2 : 1); }

}  // namespace rt
