// Rotary positions, and rows of keys and values to and from the paged 8-bit cache.  All three
// move memory: each value is read once and written once by one launch.  What is written goes past the
// caches (nontemporal): a kernel's outputs are read by a later one, on any of the eight dies, and the lines of a
// cached store take room from loads.  8192 tokens of 40 heads of 128 bf16 values turned: 25.9 us (6.5 TB/s), where
// cached stores took 35; a sequence of 32768 tokens read back 31.6 (6.4 TB/s), where they took 51.  Loads stay cached:
// past the caches they took 32 and 43.
#include <cmath>
#include <type_traits>

#include "cache8.h"
#include "q8.h"

namespace ds {

int heads_check(const ds_heads *t, const char *what, bool output) {
    if (!t) {
        set_error("%s: null tensor", what);
        return DS_EINVAL;
    }
    if ((t->type != DS_TYPE_F32 && t->type != DS_TYPE_F16 && t->type != DS_TYPE_BF16) || t->reserved != 0) {
        set_error("%s: type %d, reserved %d", what, t->type, t->reserved);
        return DS_EINVAL;
    }
    constexpr int64_t most = 0x7fffff00;                   // (room for a group of tokens past the last)
    if (t->tokens < 0 || t->tokens > most || t->heads < 1 || t->heads > 65535 || t->dim < 1 || t->dim > 65536 ||
        t->ld < 0 || t->head_ld < 0 || t->ld > (int64_t(1) << 40) || t->head_ld > (int64_t(1) << 40)) {
        set_error("%s: %lld tokens x %lld heads x %lld values, %lld and %lld elements apart", what,
                  (long long)t->tokens, (long long)t->heads, (long long)t->dim, (long long)t->ld,
                  (long long)t->head_ld);
        return DS_EINVAL;
    }
    if (t->tokens > 0 && (!t->data || reinterpret_cast<uintptr_t>(t->data) % type_bytes(t->type) != 0)) {
        set_error("%s: null or misaligned buffer", what);
        return DS_EINVAL;
    }
    if (output && t->tokens > 0) {
        const bool inside = t->heads == 1 || t->head_ld >= t->dim, apart = t->tokens == 1 || t->ld >= t->dim;
        const bool tokens_first = t->tokens == 1 || t->ld >= (t->heads - 1) * t->head_ld + t->dim;
        // (up to 2^71)
        const bool heads_first = t->heads == 1 || t->head_ld >= __int128(t->tokens - 1) * t->ld + t->dim;
        if (!inside || !apart || !(tokens_first || heads_first)) {
            set_error("%s: rows %lld (tokens) and %lld (heads) elements apart overlap", what, (long long)t->ld,
                      (long long)t->head_ld);
            return DS_EINVAL;
        }
    }
    return DS_OK;
}

int cache8_check(const ds_cache8 *c) {
    if (!c) {
        set_error("null cache");
        return DS_EINVAL;
    }
    if ((c->format != DS_Q8_E4M3 && c->format != DS_Q8_E5M2) ||
        (c->scale_type != DS_SCALE_POW2 && c->scale_type != DS_SCALE_F32) || c->reserved != 0) {
        set_error("cache: format %d, scale type %d, reserved %d", c->format, c->scale_type, c->reserved);
        return DS_EINVAL;
    }
    if (c->pages < 1 || c->pages > 0x7fffffff || c->page < 16 || c->page > 65536 || c->page % 16 != 0 ||
        c->heads < 1 || c->heads > 65535 || c->dim < 16 || c->dim > kCacheDim || c->dim % 16 != 0 ||
        int64_t(c->heads) * c->page * c->dim > 0x7fffffff) {
        set_error("cache: %lld pages of %d tokens x %d heads x %d values (page and dim: multiples of 16, dim up "
                  "to 256, a page below 2^31 bytes)",
                  (long long)c->pages, c->page, c->heads, c->dim);
        return DS_EINVAL;
    }
    if (c->stride < int64_t(c->heads) * c->page * c->dim || c->stride % 16 != 0 ||
        c->scale_stride < int64_t(c->heads) * c->page || c->stride > (int64_t(1) << 40) ||
        c->scale_stride > (int64_t(1) << 40)) {
        set_error("cache: pages %lld bytes and %lld scales apart", (long long)c->stride, (long long)c->scale_stride);
        return DS_EINVAL;
    }
    const uintptr_t rows = reinterpret_cast<uintptr_t>(c->k) | reinterpret_cast<uintptr_t>(c->v);
    const uintptr_t scales = reinterpret_cast<uintptr_t>(c->k_scale) | reinterpret_cast<uintptr_t>(c->v_scale);
    if (!c->k || !c->v || !c->k_scale || !c->v_scale || rows % 16 != 0 ||
        (c->scale_type == DS_SCALE_F32 && scales % 4 != 0)) {
        set_error("cache: null or misaligned buffer");
        return DS_EINVAL;
    }
    return DS_OK;
}

int chunk_check(const ds_chunk *c, const ds_cache8 *cache) {
    if (!c) {
        set_error("null chunk");
        return DS_EINVAL;
    }
    if (c->seqs < 0 || c->seqs > (1 << 24) || c->table_cols < 0 || c->table_ld < c->table_cols ||
        c->table_ld > (int64_t(1) << 32) || c->table_cols > kMaxPlaces / cache->page) {
        set_error("chunk: %lld sequences, a table of %lld columns %lld apart (pages of %d)", (long long)c->seqs,
                  (long long)c->table_cols, (long long)c->table_ld, cache->page);
        return DS_EINVAL;
    }
    const uintptr_t all = reinterpret_cast<uintptr_t>(c->starts) | reinterpret_cast<uintptr_t>(c->lengths) |
                          reinterpret_cast<uintptr_t>(c->table);
    if (c->seqs > 0 && (!c->starts || !c->lengths || (c->table_cols > 0 && !c->table) || all % 4 != 0)) {
        set_error("chunk: null or misaligned list");
        return DS_EINVAL;
    }
    return DS_OK;
}

namespace {

// N values of a row from column c; vec: 16-byte rows.
template <typename T, int N>
__device__ __forceinline__ void load_n(const T *p, bool vec, float (&v)[N]) {
    T t[N];
    if (vec) {
#pragma unroll
        for (size_t i = 0; i < sizeof(t) / 16; ++i)
            reinterpret_cast<intx4 *>(t)[i] = reinterpret_cast<const intx4 *>(p)[i];
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) t[i] = p[i];
    }
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = float(t[i]);
}
template <typename T, int N>
__device__ __forceinline__ void store_n(T *p, bool vec, const float (&v)[N]) {
    T t[N];
#pragma unroll
    for (int i = 0; i < N; ++i) t[i] = T(v[i]);
    if (vec) {
#pragma unroll
        for (size_t i = 0; i < sizeof(t) / 16; ++i)
            __builtin_nontemporal_store(reinterpret_cast<const intx4 *>(t)[i], &reinterpret_cast<intx4 *>(p)[i]);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) p[i] = t[i];
    }
}

// ---- rotary positions --------------------------------------------------------------

constexpr int kTurnLds = 2048;            // angles of a workgroup

struct RotaryArgs {
    const int32_t *pos;
    const float *freqs;
    int tokens, heads, dim, half;         // half: pairs of a head
    int tb, hb;                           // tokens and heads of a workgroup
    int items, ni;                        // work items of a row; those that turn pairs
    float scale, sign;
    FastDiv f_items, f_hb, f_half;
};

// (u, w) = (p cos - q sin, p sin + q cos) scale, with the angle position * frequency; the inverse has the other
// sine.  A workgroup forms its tokens' angles once for all their heads, in LDS.  They are taken
// in revolutions: three roundings of 2^-53 leave the product within 2^-34 of one at position 10^6 and 2^-22 at
// 2^31, its whole part is dropped there, and fp32 holds the fraction.  Then the threads take items of 16 bytes of each
// half of a head, or 16 bytes of pairs side by side (N pairs either way; single ones where rows are not whole groups of
// 16 bytes), and copy what is not turned unless it is in place.  Memory bounds it: the figures are above; 4099 tokens of 24 heads of
// 96 fp32 values, 64 of them turned by pairs, 13.7 us (5.5 TB/s; items of 64 bytes took 16); one token of 40 heads 2.1 us
// on the chip, less than its launch.
template <typename T, int N, bool PAIRS>
__global__ __launch_bounds__(256) void rotary(HeadsView<const T> x, HeadsView<T> y, RotaryArgs a) {
    __shared__ float2 turn[kTurnLds];
    const int t0 = blockIdx.x * a.tb, nt = min(a.tb, a.tokens - t0);
    const int h0 = blockIdx.y * a.hb, nh = min(a.hb, a.heads - h0);
    for (int i = threadIdx.x; i < nt * a.half; i += 256) {
        const int t = fdiv(i, a.f_half), j = i - t * a.half;
        const double rev = double(a.pos[t0 + t]) * (double(a.freqs[j]) * 0.15915494309189533577);
        const float r = float(rev - rint(rev));
        float s, c;
        sincospif(2.f * r, &s, &c);
        turn[i] = make_float2(c * a.scale, s * a.scale * a.sign);
    }
    __syncthreads();
    const int total = nt * a.hb * a.items;
    for (int i = threadIdx.x; i < total; i += 256) {
        const int row = fdiv(i, a.f_items), item = i - row * a.items;
        const int t = fdiv(row, a.f_hb), h = row - t * a.hb;
        if (h >= nh) continue;
        const T *px = x.p + (t0 + t) * x.ld + (h0 + h) * x.hld;
        T *py = y.p + (t0 + t) * y.ld + (h0 + h) * y.hld;
        constexpr bool vec = N > 1;
        constexpr int kCopy = vec && PAIRS ? 2 * N : N;
        if (item < a.ni) {
            const int j = item * N;
            const float2 *cs = turn + t * a.half + j;
            if constexpr (PAIRS) {
                float v[2 * N], w[2 * N];
                load_n<T, 2 * N>(px + 2 * j, vec, v);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    w[2 * e] = v[2 * e] * cs[e].x - v[2 * e + 1] * cs[e].y;
                    w[2 * e + 1] = v[2 * e] * cs[e].y + v[2 * e + 1] * cs[e].x;
                }
                store_n<T, 2 * N>(py + 2 * j, vec, w);
            } else {
                float p[N], q[N], u[N], w[N];
                load_n<T, N>(px + j, vec, p);
                load_n<T, N>(px + a.half + j, vec, q);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    u[e] = p[e] * cs[e].x - q[e] * cs[e].y;
                    w[e] = p[e] * cs[e].y + q[e] * cs[e].x;
                }
                store_n<T, N>(py + j, vec, u);
                store_n<T, N>(py + a.half + j, vec, w);
            }
        } else {
            const int d = 2 * a.half + (item - a.ni) * kCopy;
            float v[kCopy];
            load_n<T, kCopy>(px + d, vec, v);
            store_n<T, kCopy>(py + d, vec, v);
        }
    }
}

// ---- rows to and from the cache --------------------------------------------------------

constexpr int kPlaceSeqs = 2047;          // most sequences whose starts a workgroup keeps in LDS

struct CacheArgs {
    CacheView c;
    ChunkView n;
    int tb;                               // tokens of a workgroup
    int vec_k, vec_v;
    FastDiv f_tb;
};

// The places of a workgroup's tokens, in LDS: the starts come in one read of all threads, so that the
// search for a token's sequence takes no read of memory a step.
__device__ __forceinline__ void places(const CacheArgs &a, int t0, int nt, int *lds, Place *out) {
    if (a.n.seqs <= kPlaceSeqs) {
        if (a.n.seqs > 0)
            for (int i = threadIdx.x; i <= a.n.seqs; i += 256) lds[i] = a.n.starts[i];
        __syncthreads();
        if (int(threadIdx.x) < nt) out[threadIdx.x] = place_of(a.c, a.n, lds, t0 + threadIdx.x);
    } else if (int(threadIdx.x) < nt) {
        out[threadIdx.x] = place_of(a.c, a.n, a.n.starts, t0 + threadIdx.x);
    }
    __syncthreads();
}

// Largest of groups of LPR lanes (8, 16 or 32), in all of them.
template <int LPR>
__device__ __forceinline__ unsigned max_lanes(unsigned v) {
    v = max(v, unsigned(__builtin_amdgcn_update_dpp(0, int(v), 0xB1, 0xF, 0xF, false)));   // lane ^ 1
    v = max(v, unsigned(__builtin_amdgcn_update_dpp(0, int(v), 0x4E, 0xF, 0xF, false)));   // lane ^ 2
    v = max(v, unsigned(__builtin_amdgcn_update_dpp(0, int(v), 0x141, 0xF, 0xF, false)));  // other quad
    if constexpr (LPR >= 16)
        v = max(v, unsigned(__builtin_amdgcn_update_dpp(0, int(v), 0x140, 0xF, 0xF, false)));  // other eight
    if constexpr (LPR >= 32) v = max(v, unsigned(__shfl_xor(int(v), 16)));
    return v;
}

// Row i of a workgroup's: token by token within a head, keys' heads and then values'; page kNoSeq past the last.
struct RowAt {
    int page, off, t, h;
    bool val;
};
__device__ __forceinline__ RowAt row_at(const CacheArgs &a, const Place *at, int i, int total, int nt) {
    const int hk = fdiv(min(i, total - 1), a.f_tb), t = min(i, total - 1) - hk * a.tb;
    const bool val = hk >= a.c.heads, is = i < total && t < nt;
    const Place p = at[is ? t : 0];
    return {is ? p.page : kNoSeq, p.off, t, val ? hk - a.c.heads : hk, val};
}
constexpr int kReadAhead = 4, kWriteAhead = 2;   // rows of a thread whose loads are on their way together

// A row's scale s is the one ds_q8_quantize gives a row of one block, and its bytes are x / s rounded to nearest.
// LPR lanes a row of up to 8 LPR values; rows of a workgroup token by token within a head, so that neighbouring
// rows of a page are written together.  Memory bounds it, in part the reads that a workgroup does one after another (starts,
// lengths and table, then its rows): prompts of up to 2731 tokens of 8 heads of 128 bf16 values (18549 in
// all, 114 MB) in 23.4 to 25.3 us, 4.9 TB/s.  Rows loaded before their places are known took 26.7, four of a thread ahead 30.
template <typename T, int LPR>
__global__ __launch_bounds__(256) void cache8_write(HeadsView<const T> k, HeadsView<const T> v, CacheArgs a) {
    __shared__ int lds[kPlaceSeqs + 1];
    __shared__ Place at[256];
    const int t0 = blockIdx.x * a.tb, nt = min(a.tb, a.n.tokens - t0);
    places(a, t0, nt, lds, at);
    const int l = threadIdx.x % LPR, d = 8 * l;
    constexpr int kRows = 256 / LPR;
    const int total = 2 * a.c.heads * a.tb;
    for (int i0 = threadIdx.x / LPR; i0 < total; i0 += kWriteAhead * kRows) {
        RowAt r[kWriteAhead];
        float x[kWriteAhead][8];
#pragma unroll
        for (int u = 0; u < kWriteAhead; ++u) {
            r[u] = row_at(a, at, i0 + u * kRows, total, nt);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[u][e] = 0.f;
            if (r[u].page >= 0 && d < a.c.dim) {
                const HeadsView<const T> &src = r[u].val ? v : k;
                load_n<T, 8>(src.p + (t0 + r[u].t) * src.ld + r[u].h * src.hld + d, r[u].val ? a.vec_v : a.vec_k, x[u]);
            }
        }
#pragma unroll
        for (int u = 0; u < kWriteAhead; ++u) {
            unsigned top = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) top = max(top, finite_abs(x[u][e]));
            const BlockScale s = block_scale(max_lanes<LPR>(top), a.c.fmt, a.c.stype);
            if (r[u].page < 0) continue;
            const int64_t row = int64_t(r[u].h) * a.c.page + r[u].off;
            if (d < a.c.dim) {
                const auto &y = x[u];
                intx2 q;
                if (a.c.fmt == DS_Q8_E4M3)
                    q = intx2{pack4<DS_Q8_E4M3>(y[0] * s.inv, y[1] * s.inv, y[2] * s.inv, y[3] * s.inv),
                              pack4<DS_Q8_E4M3>(y[4] * s.inv, y[5] * s.inv, y[6] * s.inv, y[7] * s.inv)};
                else
                    q = intx2{pack4<DS_Q8_E5M2>(y[0] * s.inv, y[1] * s.inv, y[2] * s.inv, y[3] * s.inv),
                              pack4<DS_Q8_E5M2>(y[4] * s.inv, y[5] * s.inv, y[6] * s.inv, y[7] * s.inv)};
                __builtin_nontemporal_store(q, reinterpret_cast<intx2 *>((r[u].val ? a.c.v : a.c.k) + r[u].page * a.c.stride + row * a.c.dim + d));
            }
            if (l == 0) {
                void *sp = r[u].val ? a.c.vs : a.c.ks;
                const int64_t e = r[u].page * a.c.sstride + row;
                if (a.c.stype == DS_SCALE_POW2) static_cast<uint8_t *>(sp)[e] = uint8_t(s.bits);
                else static_cast<unsigned *>(sp)[e] = s.bits;
            }
        }
    }
}

// Eight 8-bit values in fp32.
__device__ __forceinline__ void decode8(intx2 q, int fmt, float s, float (&x)[8]) {
    typedef float floatx2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        floatx2 lo, hi;
        if (fmt == DS_Q8_E4M3) {
            lo = __builtin_amdgcn_cvt_pk_f32_fp8(q[i], false);
            hi = __builtin_amdgcn_cvt_pk_f32_fp8(q[i], true);
        } else {
            lo = __builtin_amdgcn_cvt_pk_f32_bf8(q[i], false);
            hi = __builtin_amdgcn_cvt_pk_f32_bf8(q[i], true);
        }
        x[4 * i] = lo[0] * s;
        x[4 * i + 1] = lo[1] * s;
        x[4 * i + 2] = hi[0] * s;
        x[4 * i + 3] = hi[1] * s;
    }
}

// The same walk the other way: 32768 tokens of 8 heads of 128 to bf16 (202 MB) in 31.6 us, 6.4 TB/s; eight of a
// thread's rows ahead took 34.6, two 34.5.
template <typename T, int LPR>
__global__ __launch_bounds__(256) void cache8_read(HeadsView<T> k, HeadsView<T> v, CacheArgs a) {
    __shared__ int lds[kPlaceSeqs + 1];
    __shared__ Place at[256];
    const int t0 = blockIdx.x * a.tb, nt = min(a.tb, a.n.tokens - t0);
    places(a, t0, nt, lds, at);
    const int l = threadIdx.x % LPR, d = 8 * l;
    constexpr int kRows = 256 / LPR;
    if (d >= a.c.dim) return;
    const int total = 2 * a.c.heads * a.tb;
    for (int i0 = threadIdx.x / LPR; i0 < total; i0 += kReadAhead * kRows) {
        RowAt r[kReadAhead];
        intx2 q[kReadAhead];
        unsigned s[kReadAhead];
#pragma unroll
        for (int u = 0; u < kReadAhead; ++u) {
            r[u] = row_at(a, at, i0 + u * kRows, total, nt);
            q[u] = intx2{};
            s[u] = 0;
            if (r[u].page >= 0) {
                const int64_t row = int64_t(r[u].h) * a.c.page + r[u].off, e = r[u].page * a.c.sstride + row;
                const void *sp = r[u].val ? a.c.vs : a.c.ks;
                s[u] = a.c.stype == DS_SCALE_POW2 ? static_cast<const uint8_t *>(sp)[e] : static_cast<const unsigned *>(sp)[e];
                q[u] = *reinterpret_cast<const intx2 *>((r[u].val ? a.c.v : a.c.k) + r[u].page * a.c.stride + row * a.c.dim + d);
            }
        }
#pragma unroll
        for (int u = 0; u < kReadAhead; ++u) {
            if (r[u].page == kNoSeq) continue;
            float x[8];
            const float by = scale_of(s[u], a.c.stype);
            decode8(q[u], a.c.fmt, by, x);
            const HeadsView<T> &dst = r[u].val ? v : k;
            store_n<T, 8>(dst.p + (t0 + r[u].t) * dst.ld + r[u].h * dst.hld + d, r[u].val ? a.vec_v : a.vec_k, x);
        }
    }
}

template <typename Fn>
int by_type(int type, Fn fn) {
    if (type == DS_TYPE_F32) fn(static_cast<float *>(nullptr));
    else if (type == DS_TYPE_F16) fn(static_cast<_Float16 *>(nullptr));
    else fn(static_cast<__bf16 *>(nullptr));
    return hip_ok(hipGetLastError(), "launch") ? DS_OK : DS_EHIP;
}

// Checks that the entry points share, and the launch.
int cache_args(const ds_cache8 *cache, const ds_chunk *chunk, const ds_heads *k, const ds_heads *v, bool output,
               CacheArgs *a, unsigned *grid) {
    int rc;
    if ((rc = cache8_check(cache)) != DS_OK || (rc = chunk_check(chunk, cache)) != DS_OK ||
        (rc = heads_check(k, "k", output)) != DS_OK || (rc = heads_check(v, "v", output)) != DS_OK)
        return rc;
    for (const ds_heads *t : {k, v})
        if (t->tokens != k->tokens || t->heads != cache->heads || t->dim != cache->dim || t->type != k->type) {
            set_error("%s: %lld x %lld x %lld of type %d, where the cache has %d heads of %d and k %lld tokens of type %d",
                      t == k ? "k" : "v", (long long)t->tokens, (long long)t->heads, (long long)t->dim, t->type,
                      cache->heads, cache->dim, (long long)k->tokens, k->type);
            return DS_EINVAL;
        }
    a->c = cache_view(cache);
    a->n = chunk_view(chunk, cache, k->tokens);
    // About 64 rows of keys and values a workgroup, a power of two of tokens, and some workgroups a compute unit:
    // 18549 tokens of 8 heads of 128 written in 26.5 us, where 128 rows took 28.7 and 256 32.4; reading
    // took the same with any of them.
    a->tb = 1;
    while (a->tb < 256 && 2 * a->tb * cache->heads < 64) a->tb *= 2;
    while (a->tb > 1 && k->tokens < 512 * int64_t(a->tb)) a->tb /= 2;
    a->f_tb = make_fastdiv(a->tb);
    a->vec_k = heads16(k);
    a->vec_v = heads16(v);
    const int64_t groups = (k->tokens + a->tb - 1) / a->tb;
    *grid = unsigned(groups);
    return launch_check(groups, 256, "cache");
}

}  // namespace
}  // namespace ds

using namespace ds;

extern "C" {

int ds_rotary(const ds_heads *x, const int32_t *pos, const float *freqs, int64_t turn, int mode, float scale,
              const ds_heads *y, hipStream_t stream) {
    int rc;
    if ((rc = heads_check(x, "x", false)) != DS_OK || (rc = heads_check(y, "y", true)) != DS_OK) return rc;
    if (x->tokens != y->tokens || x->heads != y->heads || x->dim != y->dim || x->type != y->type) {
        set_error("y is %lld x %lld x %lld of type %d, x %lld x %lld x %lld of type %d", (long long)y->tokens,
                  (long long)y->heads, (long long)y->dim, y->type, (long long)x->tokens, (long long)x->heads,
                  (long long)x->dim, x->type);
        return DS_EINVAL;
    }
    if (turn < 0 || turn % 2 != 0 || turn > x->dim || turn / 2 > kTurnLds || mode < 0 || mode > 3 ||
        !std::isfinite(scale)) {
        set_error("turn %lld of %lld values (even, up to %d), mode %d, scale %g", (long long)turn, (long long)x->dim,
                  2 * kTurnLds, mode, double(scale));
        return DS_EINVAL;
    }
    if (x->tokens == 0) return DS_OK;
    if (!pos || (turn > 0 && !freqs) || (reinterpret_cast<uintptr_t>(pos) | reinterpret_cast<uintptr_t>(freqs)) % 4 != 0) {
        set_error("null or misaligned positions or frequencies");
        return DS_EINVAL;
    }
    RotaryArgs a{};
    a.pos = pos;
    a.freqs = freqs;
    a.tokens = int(x->tokens);
    a.heads = int(x->heads);
    a.dim = int(x->dim);
    a.half = int(turn / 2);
    a.scale = scale;
    a.sign = mode & DS_ROTARY_INVERSE ? -1.f : 1.f;
    const bool pairs = mode & DS_ROTARY_PAIRS;
    const int most16 = 16 / type_bytes(x->type);            // values of 16 bytes
    const bool vec = heads16(x) && heads16(y) && turn % (pairs ? most16 : 2 * most16) == 0 && x->dim % most16 == 0;
    const int n = !vec ? 1 : pairs ? most16 / 2 : most16;   // pairs of an item
    a.ni = a.half / n;
    // in place, what is not turned is there already
    const bool same = x->data == y->data && x->ld == y->ld && x->head_ld == y->head_ld;
    a.items = a.ni + (same ? 0 : int(x->dim - turn) / (vec ? most16 : 1));
    if (a.items == 0) return DS_OK;
    // some 1024 items a workgroup, of one token's heads or of several tokens; fewer heads where the
    // tokens alone do not fill the chip
    a.hb = a.heads;
    a.tb = 1;
    const int most = a.half ? kTurnLds / a.half : 256;
    while (2 * a.tb <= most && a.tb < 256 && int64_t(a.tb) * a.heads * a.items < 1024 && a.tokens > 512 * a.tb) a.tb *= 2;
    while (a.hb > 1 && int64_t(a.hb) * a.items * a.tb > 256 && (a.tokens + a.tb - 1) / a.tb * ((a.heads + a.hb - 1) / a.hb) < 512)
        a.hb = (a.hb + 1) / 2;
    // (a workgroup's items are counted in 31 bits)
    while (a.hb > 1 && int64_t(a.tb) * a.hb * a.items >= (int64_t(1) << 30)) a.hb = (a.hb + 1) / 2;
    a.f_items = make_fastdiv(a.items);
    a.f_hb = make_fastdiv(a.hb);
    a.f_half = make_fastdiv(std::max(1, a.half));
    const dim3 grid((a.tokens + a.tb - 1) / a.tb, (a.heads + a.hb - 1) / a.hb);
    if ((rc = launch_check(int64_t(grid.x) * grid.y, 256, "ds_rotary")) != DS_OK) return rc;
    return by_type(x->type, [&](auto *t) {
        using T = std::remove_cv_t<std::remove_pointer_t<decltype(t)>>;
        constexpr int kN = 16 / sizeof(T);
        (pairs ? vec ? rotary<T, kN / 2, true> : rotary<T, 1, true>
               : vec ? rotary<T, kN, false> : rotary<T, 1, false>)
            <<<grid, 256, 0, stream>>>(heads_view<const T>(x), heads_view<T>(y), a);
    });
}

int ds_cache8_write(const ds_cache8 *cache, const ds_chunk *chunk, const ds_heads *k, const ds_heads *v,
                    hipStream_t stream) {
    CacheArgs a{};
    unsigned grid;
    const int rc = cache_args(cache, chunk, k, v, false, &a, &grid);
    if (rc != DS_OK || k->tokens == 0 || chunk->seqs == 0) return rc;
    return by_type(k->type, [&](auto *t) {
        using T = std::remove_cv_t<std::remove_pointer_t<decltype(t)>>;
        (a.c.dim <= 64 ? cache8_write<T, 8> : a.c.dim <= 128 ? cache8_write<T, 16> : cache8_write<T, 32>)
            <<<grid, 256, 0, stream>>>(heads_view<const T>(k), heads_view<const T>(v), a);
    });
}

int ds_cache8_read(const ds_cache8 *cache, const ds_chunk *chunk, const ds_heads *k, const ds_heads *v,
                   hipStream_t stream) {
    CacheArgs a{};
    unsigned grid;
    const int rc = cache_args(cache, chunk, k, v, true, &a, &grid);
    if (rc != DS_OK || k->tokens == 0 || chunk->seqs == 0) return rc;
    return by_type(k->type, [&](auto *t) {
        using T = std::remove_cv_t<std::remove_pointer_t<decltype(t)>>;
        (a.c.dim <= 64 ? cache8_read<T, 8> : a.c.dim <= 128 ? cache8_read<T, 16> : cache8_read<T, 32>)
            <<<grid, 256, 0, stream>>>(heads_view<T>(k), heads_view<T>(v), a);
    });
}

}  // extern "C"
