// The paged 8-bit cache: host checks, what kernels take, and the arithmetic that leads from a token
// to its row.  That arithmetic reads numbers from device memory which the host has not seen, so it bounds
// each before it is used; it compiles for the host too, where tests run it on bad numbers.
#pragma once

#include <hip/hip_runtime.h>

#include "ds_internal.h"

namespace ds {

constexpr int kCacheDim = 256;            // most values of a head's row
constexpr int64_t kMaxPlaces = (int64_t(1) << 31) - (1 << 16);

// DS_OK, or DS_EINVAL with the error set.  heads_check of an output refuses rows that overlap.
int heads_check(const ds_heads *t, const char *what, bool output);
int cache8_check(const ds_cache8 *c);
int chunk_check(const ds_chunk *c, const ds_cache8 *cache);

template <typename T>
struct HeadsView {
    T *p;
    int64_t ld, hld;
};
template <typename T>
inline HeadsView<T> heads_view(const ds_heads *t) {
    return {static_cast<T *>(t->data), t->ld, t->head_ld};
}
// Rows of 16-byte groups.
inline int heads16(const ds_heads *t) {
    const int64_t per = 16 / (t->type == DS_TYPE_F32 ? 4 : 2);
    return reinterpret_cast<uintptr_t>(t->data) % 16 == 0 && t->dim % per == 0 &&
           (t->tokens <= 1 || t->ld % per == 0) && (t->heads <= 1 || t->head_ld % per == 0);
}

struct CacheView {
    uint8_t *k, *v;
    void *ks, *vs;
    int64_t stride, sstride;
    int pages, page, heads, dim, fmt, stype;
    FastDiv f_page;
};
inline CacheView cache_view(const ds_cache8 *c) {
    return {static_cast<uint8_t *>(c->k), static_cast<uint8_t *>(c->v), c->k_scale, c->v_scale, c->stride,
            c->scale_stride, int(c->pages), c->page, c->heads, c->dim, c->format, c->scale_type,
            make_fastdiv(c->page)};
}

struct ChunkView {
    const int32_t *starts, *lengths, *table;
    int64_t tld;
    int seqs, tokens, cap;                // cap: positions that the table holds
};
inline ChunkView chunk_view(const ds_chunk *c, const ds_cache8 *cache, int64_t tokens) {
    return {c->starts, c->lengths, c->table, c->table_ld, int(c->seqs), int(tokens),
            int(c->table_cols * cache->page)};
}

__host__ __device__ __forceinline__ int fdiv(int n, const FastDiv &d) {
#ifdef __HIP_DEVICE_COMPILE__
    return int((__umulhi(uint32_t(n), d.m) + uint32_t(n)) >> d.s);
#else
    return int((((uint64_t(uint32_t(n)) * d.m) >> 32) + uint32_t(n)) >> d.s);
#endif
}

// Last b of [0, seqs) with starts[b] <= t; 0 where there is none.  In range whatever starts holds.
template <typename Starts>
__host__ __device__ __forceinline__ int find_seq(const Starts &starts, int seqs, int t) {
    int lo = 0, n = seqs;
    while (n > 1) {
        const int half = n >> 1;
        if (starts[lo + half] <= t) {
            lo += half;
            n -= half;
        } else {
            n = half;
        }
    }
    return lo;
}

// Where a token's row lies: page and offset in it; page kNoPlace without a place, kNoSeq if the
// token is no sequence's.
constexpr int kNoPlace = -1, kNoSeq = -2;
struct Place {
    int page, off;
};
// The place of position pos of sequence b.
__host__ __device__ __forceinline__ Place place_at(const CacheView &c, const ChunkView &k, int b, int64_t pos) {
    if (pos < 0 || pos >= k.cap) return {kNoPlace, 0};
    const int col = fdiv(int(pos), c.f_page);
    const int id = k.table[int64_t(b) * k.tld + col];
    return {id >= 0 && id < c.pages ? id : kNoPlace, int(pos) - col * c.page};
}
template <typename Starts>
__host__ __device__ __forceinline__ Place place_of(const CacheView &c, const ChunkView &k, const Starts &starts, int t) {
    if (k.seqs == 0) return {kNoSeq, 0};
    const int b = find_seq(starts, k.seqs, t);
    const int end = starts[b + 1];
    if (starts[b] > t || t >= end) return {kNoSeq, 0};
    return place_at(c, k, b, int64_t(k.lengths[b]) - end + t);
}

}  // namespace ds
