// What the attention kernels and their launch share.
#pragma once

#include "cache8.h"

namespace ds {

constexpr int kWaves = 4;
constexpr int kKeys = 32;                 // keys of a tile
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr int kMostSplits = 64;

struct AttnArgs {
    CacheView c;
    ChunkView n;
    const void *q;
    void *out;
    int64_t ldq, hldq, ldo, hldo;
    float *lse;
    float *part;                          // splits > 1: [split][token][head][dim] sums, then m and l
    float2 *ml;
    float scale;                          // times log2 e
    int heads, group;                     // query heads, and those of a cache head
    int causal, window, len;              // len: most keys of a sequence that are seen
    int splits, span;                     // keys of a split, a multiple of 32 (kWaves * 32 if waves share rows)
    int tiles;                            // of rows
    int vec_q, vec_o;
    FastDiv f_group;
};

// Blocks of 32 values that a row of dim is taken as: 2, 4 or 8.
constexpr int attn8_dim_blocks(int dim) { return dim <= 64 ? 2 : dim <= 128 ? 4 : 8; }
// Blocks of 32 rows of a wave that has rows of its own.
constexpr int attn8_blocks(bool f32, int dim_blocks) { return f32 || dim_blocks == 8 ? 1 : 1; }

// The kernel of a type (float, _Float16, __bf16).
template <typename T>
const void *attn8_kernel(int fmt, int dim, bool few);

}  // namespace ds
