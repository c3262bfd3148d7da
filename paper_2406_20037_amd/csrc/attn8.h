// What the attention kernels and their launch share.
#pragma once

#include "cache8.h"

namespace ds {

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
    int splits, span;                     // keys of a split
    int vec_q, vec_o;                     // rows of 16-byte groups
    FastDiv f_group, f_kv, f_splits, f_dim4;
};

// Four forms of the kernel (attn8_kernel.h): waves that share 16 or 32 rows and split the keys; waves of 32 rows
// each that read keys by themselves; waves of 32 rows each that share the keys through LDS.
enum { kAttnFew, kAttnShare, kAttnOwn, kAttnTiles };
constexpr int attn8_dim_blocks(int dim) { return dim <= 64 ? 2 : dim <= 128 ? 4 : 8; }
// (few rows of 65 to 128 values: eight waves of one workgroup in place of four of two; unequal sequences, whose
// longest one ends last, gain: 64 of up to 8192 keys 122 -> 117 us, 100 of up to 6000 136 -> 122; equal ones
// of 8192 lose, 167 -> 172)
constexpr int attn8_threads(int form, int dim_blocks) {
    return form == kAttnTiles || (form == kAttnFew && dim_blocks == 4) ? 512 : 256;
}
constexpr int attn8_rows(int form) { return form == kAttnFew ? 16 : form == kAttnShare ? 32 : form == kAttnTiles ? 256 : 128; }

// Whether the many rows of a type and width take kAttnOwn (else kAttnTiles): where the registers hold no more
// than one wave a SIMD unit.
template <typename T>
constexpr bool attn8_own_form(int dim_blocks) {
    return sizeof(T) == 4 || dim_blocks == 8;
}

// Workgroups that a compute unit holds: by their registers.
constexpr int attn8_groups(int form, bool f32, int dim_blocks) {
    if (form == kAttnFew) return dim_blocks >= 4 ? 1 : f32 ? 2 : 4;
    return form == kAttnTiles || dim_blocks == 8 || f32 ? 1 : 2;
}

struct AttnKernel {
    const void *func;
    int lds;                              // bytes of dynamic LDS
};
// The kernel of a type (float, _Float16, __bf16); exact: weights of 16 bits at least.
template <typename T>
AttnKernel attn8_kernel(int form, int fmt, int stype, int dim, bool exact);

}  // namespace ds
