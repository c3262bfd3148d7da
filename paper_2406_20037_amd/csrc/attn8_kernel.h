// Attention of new tokens over the paged 8-bit cache.
//
// For one cache head a row is a pair of a new token and one of the query heads that share it.  A wave takes 16 or 32
// rows and walks over tiles of 32 or 64 keys with the running maximum m and sum l of each row's softmax.  It
// computes the products transposed, on 32x32x16 matrix instructions (16 rows: on 16x16x32, in the like way):
//     S^T = K Q^T:  lane (i, h), i = lane % 32, h = lane / 32, has S of row i and 16 of 32 keys,
//     O^T = V^T P^T: and the same lane needs P of row i and 8 keys an instruction as the second operand:
// those that it holds, if V's keys are taken in the same order.  So weights never leave their lane, and a
// row's maximum is one of its registers and one exchange of halves (of quarters).
//
// Few rows: memory bounds it.  Keys and values come from memory as they lie, without LDS and without a barrier: a lane's 16
// bytes of a key's row are the first operand of two instructions (Q in the same order of values), and its 4 or 8 bytes
// of eight keys' rows are those of four or eight, transposed by byte permutes, a value and its
// neighbour key's in one conversion.  64 tokens of 64 query heads over 8192 keys of 8 heads of 128 each: 170 us, 6.4
// TB/s; over up to 8192, 116 us, 4.7 TB/s; four tokens each, on 32 rows, 136.
//
// Many rows: the matrix and the vector unit bound it, and decoding is a third of the vector unit's work if each wave does it.
// So eight waves share decoded tiles of 64 keys in LDS, K by rows and V by columns.  A prompt of 8192 tokens of 32
// heads over 8 of 128: 590 to 602 us, 914 to 932 TFLOP/s.
#pragma once

#include <cmath>
#include <type_traits>

#include "attn8.h"
#include "kern_common.h"
#include "q8.h"

namespace ds {
namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float floatx2 __attribute__((ext_vector_type(2)));

constexpr int kKeys = 32;                 // keys of a matrix instruction's tile
constexpr float kLn2 = 0.69314718055994530942f;

// How the types compute: Q in QP parts of operand type, P in PP parts of bf16 or more (see attn8_kernel).
template <typename T>
struct Parts;
template <>
struct Parts<__bf16> {
    static constexpr int QP = 1, PP = 1;
    typedef bf16x8 Op;
};
template <>
struct Parts<_Float16> {
    static constexpr int QP = 1, PP = 2;
    typedef f16x8 Op;
};
template <>
struct Parts<float> {
    static constexpr int QP = 3, PP = 3;
    typedef bf16x8 Op;
};

__device__ __forceinline__ floatx16 mma(bf16x8 a, bf16x8 b, floatx16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ floatx16 mma(f16x8 a, f16x8 b, floatx16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

// Eight bytes of a key's row as an operand, times a power of two (1 for fp16): exact in both types.
template <int FMT, typename Op>
__device__ __forceinline__ Op decode_k(int lo, int hi, float by = 1.f) {
    if constexpr (std::is_same_v<Op, bf16x8>) {
        return to_bf16<FMT>(lo, hi, by);
    } else {
        const int w[2] = {lo, hi};
        f16x8 r;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f16x2 t;
            if constexpr (FMT == DS_Q8_E4M3)
                t = (i & 1) ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[i >> 1], 1.f, true)
                            : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[i >> 1], 1.f, false);
            else
                t = (i & 1) ? __builtin_amdgcn_cvt_scalef32_pk_f16_bf8(w[i >> 1], 1.f, true)
                            : __builtin_amdgcn_cvt_scalef32_pk_f16_bf8(w[i >> 1], 1.f, false);
            r[2 * i] = t[0];
            r[2 * i + 1] = t[1];
        }
        return r;
    }
}

// The other half's value (lane ^ 32).
__device__ __forceinline__ float other_half(float v) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(threadIdx.x & 32 ? a[0] : a[1]);
}

// Whether a number in parts, times one of the format, can come to none where the whole does not: in three parts, which are 0
// or of either sign, times an infinity, which only e5m2 has (of two parts see put_weight).  Sums that are no number are
// then taken by slow_sums; a number that is none among the values leads there too.
template <typename T, int FMT>
constexpr bool kPartsApart = FMT == DS_Q8_E5M2 && Parts<T>::PP == 3;

// Any byte of the word that stands for no finite number.
template <int FMT>
__device__ __forceinline__ unsigned not_finite(unsigned w) {
    if constexpr (FMT == DS_Q8_E4M3) return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
    else return ((w & 0x7c7c7c7cu) + 0x04040404u) & 0x80808080u;
}

// Two of a word's bytes as bf16, times a power of two.
template <int FMT, bool HIGH>
__device__ __forceinline__ bf16x2 decode2(unsigned w, float by) {
    if constexpr (FMT == DS_Q8_E4M3) return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(int(w), by, HIGH);
    else return __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(int(w), by, HIGH);
}

__device__ __forceinline__ unsigned load_scale(const void *p, int stype, int64_t at) {
    return stype == DS_SCALE_POW2 ? static_cast<const uint8_t *>(p)[at] : static_cast<const unsigned *>(p)[at];
}

// The kernel's argument once more, read again here: what a long loop does not use needs no scalar registers
// through it.
__device__ __forceinline__ AttnArgs late_args() {
    typedef const __attribute__((address_space(4))) AttnArgs *Ptr;
    uint64_t at = reinterpret_cast<uint64_t>(__builtin_amdgcn_kernarg_segment_ptr());
    __asm__ volatile("" : "+s"(at));
    AttnArgs a;
    typedef const __attribute__((address_space(4))) int *Word;
    const Word from = reinterpret_cast<Word>(at);
    int *to = reinterpret_cast<int *>(&a);
#pragma unroll
    for (size_t i = 0; i < sizeof(AttnArgs) / 4; ++i) to[i] = from[i];
    // (global memory, which a pointer read from memory does not say)
    const auto global = [](auto *&p) {
        using V = std::remove_reference_t<decltype(*p)>;
        p = (V *)(__attribute__((address_space(1))) V *)p;
    };
    global(a.lse);
    global(a.part);
    global(a.ml);
    global(a.c.k);
    global(a.c.v);
    global(a.n.table);
    a.q = (const void *)(const __attribute__((address_space(1))) void *)a.q;
    a.out = (void *)(__attribute__((address_space(1))) void *)a.out;
    a.c.ks = (void *)(__attribute__((address_space(1))) void *)a.c.ks;
    a.c.vs = (void *)(__attribute__((address_space(1))) void *)a.c.vs;
    return a;
}

// The page of 16 keys from `key` on (a multiple of 16) of a sequence of length len > 0: its number as its row of the
// table has it, and the offset; of the last key's page for keys past the end.  The number is read as vectors are, although
// it is the same for all lanes: reads of scalars are counted with LDS accesses, whose waits would wait for them.
struct PageRef {
    int raw, off;
};
__device__ __forceinline__ PageRef page_ref(const AttnArgs &a, const int32_t *table, int len, int key) {
    const int k = min(key, len - 1), col = fdiv(k, a.c.f_page);
    unsigned at = col;
    __asm__ volatile("" : "+v"(at));
    return {table[at], (k - col * a.c.page) & ~15};
}
// The number where it is used: kNoPlace unless it is one of the cache's.
__device__ __forceinline__ int page_of(const AttnArgs &a, const PageRef &r) {
    const int id = __builtin_amdgcn_readfirstlane(r.raw);
    return id >= 0 && id < a.c.pages ? id : kNoPlace;
}

// Key of register r among 32: the order in which both products take keys.
__device__ __forceinline__ int key_of(int r, int h) { return 8 * (r >> 2) + 4 * h + (r & 3); }

// ---- a workgroup's and a wave's rows ------------------------------------------------------

// Sequence of a tile of rows: the tiles of sequence b begin at starts[b] * group / rows + b, which leaves each at
// least as many as it needs, without a sum over the sequences before it.
template <int ROWS>
__device__ __forceinline__ int first_tile(const AttnArgs &a, int b) {
    return int(unsigned(min(max(a.n.starts[b], 0), a.n.tokens)) * unsigned(a.group) / ROWS) + b;
}

struct Work {
    int b, head, split;                   // sequence, cache head, split (all uniform)
    int len;                              // keys of the sequence that may be seen
    int s0, rows;                         // its first token, its rows
    int row0;                             // the workgroup's first row
    int64_t shift;                        // token s0 + t is at position shift + t

    __device__ __forceinline__ int token(const AttnArgs &a, int r) const { return fdiv(min(r, rows - 1), a.f_group); }
    // the rows of token t see keys low .. lim - 1
    __device__ __forceinline__ int lim(const AttnArgs &a, int t) const {
        return a.causal ? int(min(max(shift + t + 1, int64_t(0)), int64_t(len))) : len;
    }
    __device__ __forceinline__ int low(const AttnArgs &a, int t) const {
        return a.window > 0 ? int(max(min(shift + t + 1 - a.window, int64_t(len)), int64_t(0))) : 0;
    }
    // Keys of the split for the workgroup's rows, [from, until): its first key is the tile's, a multiple of 64.
    __device__ __forceinline__ void keys(const AttnArgs &a, int last_row, int &from, int &until) const {
        const int base = low(a, token(a, row0)) & ~63;
        from = int(min(int64_t(base) + int64_t(split) * a.span, kMaxPlaces)) & ~63;
        until = int(min(int64_t(lim(a, token(a, last_row))), int64_t(base) + int64_t(split + 1) * a.span));
    }
};

template <int ROWS>
__device__ __forceinline__ bool find_work(const AttnArgs &a, Work &w) {
    const int lane = threadIdx.x & 63;
    // Workgroups go to the chip's eight parts in turn.  Heads side by side: the workgroups of a head share the caches
    // of as few parts as the number of heads allows.  Of few rows none share keys, and a part takes four heads of the
    // same pages: that lets memory stream (four waves a workgroup, 64 sequences of 8192 keys each: 242 -> 166 us, 6.5
    // TB/s; two heads 244, eight 166, but 100 unequal sequences 145, where one to four take 135).
    int idx;
    const int whole = int(gridDim.x) / (8 * a.c.heads) * (8 * a.c.heads);
    if (ROWS == 16 && a.c.heads % 4 == 0 && int(blockIdx.x) < whole) {
        const int four = int(blockIdx.x >> 5) * 8 + int(blockIdx.x & 7);       // of the fours of heads
        idx = fdiv(4 * four, a.f_kv);
        w.head = 4 * four - idx * a.c.heads + int(blockIdx.x >> 3 & 3);
    } else {
        idx = fdiv(blockIdx.x, a.f_kv);
        w.head = int(blockIdx.x) - idx * a.c.heads;
    }
    const int tile = fdiv(idx, a.f_splits);
    w.split = idx - tile * a.splits;
    int b = 0;
    for (int n = a.n.seqs; n > 1;) {       // 64 sequences a step
        const int by = (n + 63) / 64;
        const bool ok = lane == 0 || (lane * by < n && first_tile<ROWS>(a, b + lane * by) <= tile);
        const int k = 63 - __clzll(__ballot(ok));
        b += k * by;
        n = min(by, n - k * by);
    }
    w.b = __builtin_amdgcn_readfirstlane(b);
    const int length = a.n.lengths[w.b], end = a.n.starts[w.b + 1];
    w.s0 = min(max(a.n.starts[w.b], 0), a.n.tokens);
    const int s1 = min(max(end, w.s0), a.n.tokens);
    w.rows = (s1 - w.s0) * a.group;
    const int mine = tile - (int(unsigned(w.s0) * unsigned(a.group) / ROWS) + w.b), all = (w.rows + ROWS - 1) / ROWS;
    if (mine < 0 || mine >= all) return false;
    // the last rows, which see most keys, first
    w.row0 = (a.causal ? all - 1 - mine : mine) * ROWS;
    w.len = min(max(length, 0), a.len);
    w.shift = int64_t(length) - end + w.s0;  // (of all its tokens, also of those that the call does not have)
    return true;
}

// A lane's row.
struct Row {
    int tok, head;
    bool is;
    int low, lim;
};
__device__ __forceinline__ Row find_row(const AttnArgs &a, const Work &w, int r) {
    const int t = w.token(a, r);
    return {w.s0 + t, w.head * a.group + min(r, w.rows - 1) - t * a.group, r < w.rows, w.low(a, t), w.lim(a, t)};
}

// Values d to d + 7 of the row of Q as an operand, in parts.
template <typename T>
__device__ __forceinline__ void load_q1(const AttnArgs &a, const Row &row, int d, float by,
                                        typename Parts<T>::Op (&q)[Parts<T>::QP]) {
    const T *qp = static_cast<const T *>(a.q) + row.tok * a.ldq + row.head * a.hldq;
    T x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = T(0.f);
    if (d < a.c.dim) {
        if (a.vec_q) {
#pragma unroll
            for (size_t e = 0; e < sizeof(x) / 16; ++e)
                reinterpret_cast<intx4 *>(x)[e] = reinterpret_cast<const intx4 *>(qp + d)[e];
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = qp[d + e];
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if constexpr (Parts<T>::QP == 1) {
            q[0][e] = T(float(x[e]) * by);
        } else {
            float rest = float(x[e]) * by;
#pragma unroll
            for (int p = 0; p < Parts<T>::QP; ++p) {
                q[p][e] = __bf16(rest);
                rest -= float(q[p][e]);
            }
        }
    }
}
// Operand c of a row: values q_at(c, h) and on.
__device__ __forceinline__ int q_at(int c, int h) { return 32 * (c >> 1) + 16 * h + 8 * (c & 1); }
template <typename T, int DB>
__device__ __forceinline__ void load_q(const AttnArgs &a, const Row &row, int h, float by,
                                       typename Parts<T>::Op (&q)[Parts<T>::QP][2 * DB]) {
#pragma unroll
    for (int c = 0; c < 2 * DB; ++c) {
        typename Parts<T>::Op x[Parts<T>::QP];
        load_q1<T>(a, row, q_at(c, h), by, x);
#pragma unroll
        for (int p = 0; p < Parts<T>::QP; ++p) q[p][c] = x[p];
    }
}

// Q where a wave keeps it: in registers, or in LDS, where waves of the same rows share it and leave registers
// for keys that are on their way.
template <typename T, int DB>
struct HeldQ {
    typename Parts<T>::Op q[Parts<T>::QP][2 * DB];
    __device__ __forceinline__ typename Parts<T>::Op get(int p, int c) const { return q[p][c]; }
};
template <typename T, int DB>
struct SharedQ {
    const intx4 *q;                       // [part][operand][lane]
    __device__ __forceinline__ typename Parts<T>::Op get(int p, int c) const {
        return __builtin_bit_cast(typename Parts<T>::Op, q[(p * 2 * DB + c) * 64]);
    }
};

// ---- a row's sums -----------------------------------------------------------------------------

constexpr float kLoose = 12.f;

// Register r of block blk is value DB * i + blk of the lane's row, i = key_of(r, h).
template <int DB>
struct Sums {
    floatx16 o[DB];
    float m, l;                           // l: of the lane's half of the keys until halves() joins them

    __device__ __forceinline__ void clear() {
        m = -INFINITY;
        l = 0.f;
#pragma unroll
        for (int blk = 0; blk < DB; ++blk) o[blk] = floatx16{};
    }
    // The running maximum follows `top`, if that is above it by kLoose or more: any number near it serves, as weights
    // of up to 2^kLoose lose nothing in fp32 or bf16.
    __device__ __forceinline__ void follow(float top) {
        if (__any(top > m + kLoose || (m == -INFINITY && top > -INFINITY))) {
            const float now = fmaxf(m, top);
            const float by = now == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - now);
            m = now;
            l *= by;
#pragma unroll
            for (int blk = 0; blk < DB; ++blk)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[blk][r] *= by;
        }
    }
    // What weights are taken from.
    __device__ __forceinline__ float base() const { return m == -INFINITY ? 0.f : m; }
    // Whether a sum of the wave's is no number.
    __device__ __forceinline__ bool none() const {
        bool is = l != l;
#pragma unroll
        for (int blk = 0; blk < DB; ++blk)
#pragma unroll
            for (int r = 0; r < 16; ++r) is |= o[blk][r] != o[blk][r];
        return __any(is);
    }
};

// w in parts of bf16, element e of an operand.  Two parts that may meet an infinity (of e5m2) are cut, not rounded, and the
// last of w's 24 bits is set: so neither is 0 or of the other sign, and their sum is the infinity.  The cut doubles the
// second part's rounding, to 2^-16 of w at most.
template <int PP, int FMT>
__device__ __forceinline__ void put_weight(bf16x8 (&to)[PP], int e, float w) {
    if constexpr (PP == 2 && FMT == DS_Q8_E5M2) {
        const unsigned all = __float_as_uint(w) | 1u;
        to[0][e] = __builtin_bit_cast(__bf16, uint16_t(all >> 16));
        to[1][e] = __bf16(__uint_as_float(all) - __uint_as_float(all & 0xffff0000u));
        return;
    }
#pragma unroll
    for (int part = 0; part < PP; ++part) {
        const __bf16 top8 = __bf16(w);
        to[part][e] = top8;
        w -= float(top8);
    }
}

// The rows' sums once more, key by key in plain fp32, [key, until): for tiles whose values (or their scales) hold infinities or NaNs
// where some row does not see all keys, as 0 times those is no 0, and for infinities that meet parts (kPartsApart).  Slow, small and
// met by broken numbers only: 3 us a key and wave, so that one infinity among 8192 keys takes a prompt of fp16
// queries from 824 us to 1035, for the rows at whose edge it is.
template <typename T, int FMT, int DB, typename Q>
__device__ __forceinline__ void slow_sums(const AttnArgs &a, const Work &w, const Row &row, const Q &q, int h, int key,
                                          int until, Sums<DB> &s) {
    const auto bytes = [](const uint8_t *p, int n) {
        unsigned x = 0;
        for (int e = 0; e < n; ++e) x |= unsigned(p[e]) << (8 * e);
        return x;
    };
    s.clear();
#pragma unroll 1
    for (; key < until; ++key) {
        const Place at = key < w.len ? place_at(a.c, a.n, w.b, key) : Place{kNoPlace, 0};
        if (at.page < 0) continue;
        const int64_t rows = int64_t(w.head) * a.c.page + at.off, scales = at.page * a.c.sstride + rows;
        const uint8_t *k = a.c.k + at.page * a.c.stride + rows * a.c.dim, *v = a.c.v + at.page * a.c.stride + rows * a.c.dim;
        const float sk = scale_of(load_scale(a.c.ks, a.c.stype, scales), a.c.stype) * a.scale;
        const float sv = scale_of(load_scale(a.c.vs, a.c.stype, scales), a.c.stype);
        float x = 0.f;
#pragma unroll
        for (int c = 0; c < 2 * DB; ++c) {
            const int d = 32 * (c >> 1) + 16 * h + 8 * (c & 1);
            if (d >= a.c.dim) continue;
            const bf16x8 kd = decode_k<FMT, bf16x8>(int(bytes(k + d, 4)), int(bytes(k + d + 4, 4)));
            float whole[8] = {};                           // (parts add up to the value without rounding)
#pragma unroll
            for (int p = Parts<T>::QP - 1; p >= 0; --p) {
                intx4 held = __builtin_bit_cast(intx4, q.get(p, c));
                __asm__ volatile("" : "+v"(held));         // (its fp32 values are no registers of the loop's)
                const auto qd = __builtin_bit_cast(typename Parts<T>::Op, held);
#pragma unroll
                for (int e = 0; e < 8; ++e) whole[e] += float(qd[e]);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) x += float(kd[e]) * whole[e];
        }
        x = (x + other_half(x)) * sk;
        if (key < row.low || key >= row.lim) continue;
        if (x > s.m) {
            const float by = __builtin_amdgcn_exp2f(s.m - x);
            s.m = x;
            s.l *= by;
#pragma unroll
            for (int blk = 0; blk < DB; ++blk)
#pragma unroll
                for (int r = 0; r < 16; ++r) s.o[blk][r] *= by;
        }
        const float p = __builtin_amdgcn_exp2f(x - (s.m == -INFINITY ? 0.f : s.m));
        s.l += h == 0 ? p : 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int d = DB * key_of(r, h);
            if (d >= a.c.dim) continue;
#pragma unroll
            for (int blk = 0; blk < DB; blk += 2) {
                const bf16x2 x2 = decode2<FMT, false>(bytes(v + d + blk, 2), 1.f);
                s.o[blk][r] += p * (float(x2[0]) * sv);
                s.o[blk + 1][r] += p * (float(x2[1]) * sv);
            }
        }
    }
}

// What a wave's rows come to: written, or left as a part of them.
template <typename T, int DB>
__device__ __forceinline__ void finish(const AttnArgs &a, const Work &w, const Row &row, const Sums<DB> &s, int h) {
    if (!row.is) return;
    const int64_t at = int64_t(row.tok) * a.heads + row.head;
    if (a.splits > 1) {
        const int64_t p = int64_t(w.split) * a.n.tokens * a.heads + at;
        if (h == 0) a.ml[p] = make_float2(s.m, s.l);
        if (s.l == 0.f) return;
        float *to = a.part + p * a.c.dim;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int d = DB * key_of(r, h);
            if (d < a.c.dim) {
#pragma unroll
                for (int blk = 0; blk < DB; blk += 2) {
                    *reinterpret_cast<floatx2 *>(to + d + blk) = floatx2{s.o[blk][r], s.o[blk + 1][r]};
                }
            }
        }
        return;
    }
    const float by = s.l == 0.f ? 0.f : 1.f / s.l;
    if (a.lse && h == 0) a.lse[at] = s.l == 0.f ? -INFINITY : (s.m + log2f(s.l)) * kLn2;
    T *to = static_cast<T *>(a.out) + row.tok * a.ldo + row.head * a.hldo;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int d = DB * key_of(r, h);
        if (d >= a.c.dim) continue;
        T x[DB];
#pragma unroll
        for (int blk = 0; blk < DB; ++blk) x[blk] = T(s.l == 0.f ? 0.f : s.o[blk][r] * by);
        if (a.vec_o) {
            // (DB values of a 16-byte row: 4 bytes at least, aligned to their size up to 16)
            constexpr int kBytes = sizeof(x) < 16 ? sizeof(x) : 16;
            typedef int intv __attribute__((ext_vector_type(kBytes / 4)));
#pragma unroll
            for (size_t e = 0; e < sizeof(x) / kBytes; ++e)
                reinterpret_cast<intv *>(to + d)[e] = reinterpret_cast<const intv *>(x)[e];
        } else {
#pragma unroll
            for (int blk = 0; blk < DB; ++blk) to[d + blk] = x[blk];
        }
    }
}

// ---- keys and values straight from memory -----------------------------------------------------------

// The tile's bytes of a lane.  DB: blocks of 32 values that a row is taken as (2, 4 or 8), also the
// bytes of a lane of each key of V.
template <int DB>
struct Tile {
    static constexpr int W = DB == 8 ? 2 : 1;
    intx4 k[DB];
    unsigned v[2][8][W];
    unsigned s;                           // the scale as stored of key i: K's in half 0, V's in half 1
    int valid;                            // keys of each 16 that exist: low and high half word
};

// Where the lane's DB bytes of a row of V begin; lanes past a row's end take its last ones, for sums that nobody
// stores.
template <int DB>
__device__ __forceinline__ int v_column(int i, int dim) {
    return min(DB * i, dim - DB);
}
// (once: past the caches; see Few::load)
template <int DB, bool ONCE>
__device__ __forceinline__ void load_v(const uint8_t *p, unsigned at, unsigned (&w)[DB == 8 ? 2 : 1]) {
    const auto get = [&](const auto *from) {
        if constexpr (ONCE) return __builtin_nontemporal_load(from);
        else return *from;
    };
    if constexpr (DB == 2) {
        w[0] = get(reinterpret_cast<const uint16_t *>(p + at));
    } else if constexpr (DB == 4) {
        w[0] = get(reinterpret_cast<const unsigned *>(p + at));
    } else {
        const intx2 x = get(reinterpret_cast<const intx2 *>(p + at));
        w[0] = x[0];
        w[1] = x[1];
    }
}

// TILES: of a lane's registers, one in use and the others on their way.
template <typename T, int FMT, int PP, int DB, typename Q, int TILES>
struct Direct {
    using P = Parts<T>;
    using Op = typename P::Op;

    const AttnArgs &a;
    const Work &w;
    const Row &row;
    const Q &q;
    Sums<DB> &s;
    const int lane, i, h;
    const unsigned koff, voff;            // of the lane in a 16-key part of a page

    __device__ __forceinline__ Direct(const AttnArgs &a_, const Work &w_, const Row &r_, const Q &q_, Sums<DB> &s_)
        : a(a_), w(w_), row(r_), q(q_), s(s_), lane(threadIdx.x & 63), i(lane & 31), h(lane >> 5),
          koff((i & 15) * a_.c.dim), voff(4 * h * a_.c.dim + v_column<DB>(i, a_.c.dim)) {}

    struct Pages {
        PageRef p[2];
    };
    __device__ __forceinline__ Pages pages(int key0) const {
        const int32_t *table = a.n.table + int64_t(w.b) * a.n.tld;
        return {page_ref(a, table, w.len, key0), page_ref(a, table, w.len, key0 + 16)};
    }

    // Loads of a tile.  A part without a page reads page 0 and counts as no key; past a row's dim its last
    // bytes are read again, and the rows of a part past the sequence's end are the page's own.
    __device__ __forceinline__ void load(Tile<DB> &t, const Pages &p, int key0) const {
        const int dim = a.c.dim;
        int valid[2];
        int64_t page[2];
#pragma unroll
        for (int st = 0; st < 2; ++st) {
            const int id = page_of(a, p.p[st]);
            valid[st] = id >= 0 ? min(16, max(w.len - key0 - 16 * st, 0)) : 0;
            page[st] = max(id, 0);
        }
        t.valid = valid[0] | valid[1] << 16;
        const int at[2] = {w.head * a.c.page + p.p[0].off, w.head * a.c.page + p.p[1].off};
        const int64_t byte[2] = {page[0] * a.c.stride + int64_t(at[0]) * dim, page[1] * a.c.stride + int64_t(at[1]) * dim};
        const bool up = i & 16;
        const uint8_t *kp = a.c.k + (up ? byte[1] : byte[0]) + koff;
#pragma unroll
        for (int c = 0; c < DB; ++c) t.k[c] = *reinterpret_cast<const intx4 *>(kp + min(32 * c + 16 * h, dim - 16));
#pragma unroll
        for (int st = 0; st < 2; ++st)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                load_v<DB, std::is_same_v<Q, SharedQ<T, DB>>>(a.c.v + byte[st] + (e < 4 ? e : e + 4) * dim, voff, t.v[st][e]);
        const int64_t se = (up ? page[1] : page[0]) * a.c.sstride + (up ? at[1] : at[0]) + (i & 15);
        t.s = load_scale(h ? a.c.vs : a.c.ks, a.c.stype, se);
    }

    // The operand of block blk and 16 keys: row i of it is value DB i + blk.
    __device__ __forceinline__ bf16x8 decode_v(const Tile<DB> &t, int st, int blk) const {
        const int word = blk >> 2, j = blk & 3;
        bf16x8 r;
        unsigned pair[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            pair[e] = __builtin_amdgcn_perm(t.v[st][2 * e + 1][word], t.v[st][2 * e][word], j & 2 ? 0x07030602u : 0x05010400u);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bf16x2 x = j & 1 ? decode2<FMT, true>(pair[e], 1.f) : decode2<FMT, false>(pair[e], 1.f);
            r[2 * e] = x[0];
            r[2 * e + 1] = x[1];
        }
        return r;
    }

    // One tile; edge: some row does not see some key of it, or some key does not exist.  False where that needs
    // slow_sums.
    __device__ __forceinline__ bool step(Tile<DB> &t, int key0, bool edge, float *lds) {
        // the scales of all 32 keys to every lane that needs them; 0 of keys that do not exist
        const int valid[2] = {t.valid & 0xffff, t.valid >> 16};
        float sc = scale_of(t.s, a.c.stype);
        if (edge) sc = (i & 15) < (i & 16 ? valid[1] : valid[0]) ? sc : 0.f;
        lds[lane] = h ? sc : sc * a.scale;
        __builtin_amdgcn_wave_barrier();
        if (a.c.dim < 32 * DB)                // (a number that is none times Q's 0 is no 0)
#pragma unroll
            for (int c = 0; c < DB; ++c)
                if (32 * c + 16 * h >= a.c.dim) t.k[c] = intx4{};
        floatx16 sum = {};
#pragma unroll
        for (int c = 0; c < DB; ++c)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const Op k = decode_k<FMT, Op>(t.k[c][2 * u], t.k[c][2 * u + 1]);
#pragma unroll
                for (int p = P::QP - 1; p >= 0; --p) sum = mma(k, q.get(p, 2 * c + u), sum);
            }
        __builtin_amdgcn_sched_barrier(0);
        bf16x8 pt[2][PP];
        if (edge) {
            unsigned bad = h && !(fabsf(sc) < INFINITY);   // (values' scales)
            int has[2] = {valid[0] - 4 * h, valid[1] - 4 * h};
            __asm__ volatile("" : "+v"(has[0]), "+v"(has[1]));
#pragma unroll
            for (int st = 0; st < 2; ++st)
#pragma unroll
                for (int e = 0; e < 8; ++e)
#pragma unroll
                    for (int word = 0; word < Tile<DB>::W; ++word) {
                        unsigned &x = t.v[st][e][word];
                        if ((e < 4 ? e : e + 4) >= has[st]) x = 0;
                        bad |= not_finite<FMT>(x);
                    }
            if (__any(bad != 0)) return false;
        }
        float x[16];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const floatx4 sk = *reinterpret_cast<const floatx4 *>(lds + 8 * j + 4 * h);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[4 * j + e] = sum[4 * j + e] * sk[e];
        }
        if (edge) {
            // (known here alone, so that this stays a branch: tiles that all rows see spend nothing on it)
            int low = row.low - key0 - 4 * h, lim = row.lim - key0 - 4 * h, has[2] = {valid[0] - 4 * h, valid[1] - 4 * h};
            __asm__ volatile("" : "+v"(low), "+v"(lim), "+v"(has[0]), "+v"(has[1]));
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int k = key_of(r, 0);
                const bool sees = k >= low && k < lim && (k & 15) < has[r >> 3];
                x[r] = sees ? x[r] : -INFINITY;
            }
        }
        float top = fmaxf(x[0], x[1]);
#pragma unroll
        for (int r = 2; r < 16; r += 2) top = fmaxf(fmaxf(top, x[r]), x[r + 1]);
        s.follow(fmaxf(top, other_half(top)));
        const float off = s.base();
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            x[r] = __builtin_amdgcn_exp2f(x[r] - off);
            s.l += x[r];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const floatx4 sv = *reinterpret_cast<const floatx4 *>(lds + 32 + 8 * j + 4 * h);
#pragma unroll
            for (int e = 0; e < 4; ++e) put_weight<PP, FMT>(pt[j >> 1], 4 * (j & 1) + e, x[4 * j + e] * sv[e]);
        }
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int blk = 0; blk < DB; ++blk) {
#pragma unroll
            for (int st = 0; st < 2; ++st) {
                const bf16x8 v = decode_v(t, st, blk);
#pragma unroll
                for (int part = PP - 1; part >= 0; --part) s.o[blk] = mma(v, pt[st][part], s.o[blk]);
            }
        }
        return true;
    }

    // The keys from `key` on in steps of STEP, until `until`; every, since: keys that all rows of the wave see.
    // False where a tile needs slow_sums.
    template <int STEP>
    __device__ __forceinline__ bool walk(int key, int until, int every, int since, float *lds) {
        bool fine = true;
        const auto edge = [&](const Tile<DB> &t) {
            return key + kKeys > every || key < since || t.valid != (16 | 16 << 16);
        };
        s.clear();
        if constexpr (TILES == 1) {
            for (; key < until && fine; key += STEP) {
                Tile<DB> t;
                load(t, pages(key), key);
                fine = step(t, key, edge(t), lds);
            }
        } else if (key < until) {
            Tile<DB> t[TILES];
            Pages next = pages(key);
#pragma unroll
            for (int x = 0; x + 1 < TILES; ++x) {
                const Pages after = pages(key + (x + 1) * STEP);
                if (x == 0 || key + x * STEP < until) load(t[x], next, key + x * STEP);
                next = after;
            }
            while (fine && key < until) {
#pragma unroll
                for (int x = 0; x < TILES; ++x) {
                    if (!fine || key >= until) break;
                    const Pages after = pages(key + TILES * STEP);
                    if (key + (TILES - 1) * STEP < until) load(t[(x + TILES - 1) % TILES], next, key + (TILES - 1) * STEP);
                    next = after;
                    fine = step(t[x], key, edge(t[x]), lds);
                    key += STEP;
                }
            }
        }
        return fine;
    }
};

// The sums of waves that share rows, JOIN rows at a time: put(r0) writes those from row r0 on, and all
// threads join four values each, a wave's after another's.
template <typename T, int JOIN, int LINE, int WAVES, int ROWS, typename Put>
__device__ __forceinline__ void join_waves(const AttnArgs &a, const Work &w, const float (&sums)[WAVES][JOIN][LINE],
                                           const float2 (&ml)[WAVES][ROWS], int rows, Put put) {
#pragma unroll 1
    for (int r0 = 0; r0 < rows; r0 += JOIN) {
        if (r0 > 0) __syncthreads();
        put(r0);
        __syncthreads();
        const int line = a.c.dim / 4, n = min(JOIN, rows - r0) * line;
        for (int x = threadIdx.x; x < n; x += 64 * WAVES) {
            const int r = fdiv(x, a.f_dim4), d = 4 * (x - r * line);
            const Row out = find_row(a, w, w.row0 + r0 + r);
            float m = -INFINITY, l = 0.f;
#pragma unroll
            for (int y = 0; y < WAVES; ++y) m = fmaxf(m, ml[y][r0 + r].x);
            floatx4 sum = {};
#pragma unroll
            for (int y = 0; y < WAVES; ++y) {
                const float2 of = ml[y][r0 + r];
                const float by = of.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(of.x - m);
                l += of.y * by;
                sum += by * *reinterpret_cast<const floatx4 *>(&sums[y][r][d]);
            }
            const int64_t at = int64_t(out.tok) * a.heads + out.head;
            if (a.splits > 1) {
                const int64_t p = int64_t(w.split) * a.n.tokens * a.heads + at;
                if (d == 0) a.ml[p] = make_float2(m, l);
                *reinterpret_cast<floatx4 *>(a.part + p * a.c.dim + d) = sum;
                continue;
            }
            const float by = l == 0.f ? 0.f : 1.f / l;
            if (a.lse && d == 0) a.lse[at] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
            T y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = T(l == 0.f ? 0.f : sum[e] * by);
            T *to = static_cast<T *>(a.out) + out.tok * a.ldo + out.head * a.hldo + d;
            if (a.vec_o) {
                typedef int intv __attribute__((ext_vector_type(sizeof(T))));
                *reinterpret_cast<intv *>(to) = *reinterpret_cast<const intv *>(y);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) to[e] = y[e];
            }
        }
    }
}

// Tiles of keys that a wave of attn8_share has in registers.
template <typename T, int DB>
constexpr int share_tiles = DB == 8 ? 2 : 3;

// Four waves share 32 rows and take tiles of keys in turn.  Their sums meet in LDS, some rows at a time, and
// all threads join four values each.  Memory's latency bounds it: three tiles of a wave in registers, one in use, which
// Q in LDS makes room for.  64 sequences of up to 8192 keys of 8 heads of 128, four tokens and 8 query heads each: 136 us, 4.0 TB/s.
template <typename T, int FMT, int PP, int DB>
__global__ __launch_bounds__(256, (attn8_groups(kAttnShare, sizeof(T) == 4, DB))) void attn8_share(AttnArgs a) {
    constexpr int kJoin = DB == 8 ? 8 : 16, kLine = 32 * DB + 4;      // rows at a time, floats between them
    __shared__ __attribute__((aligned(16))) float scales[4 * 64];
    __shared__ __attribute__((aligned(16))) float sums[4][kJoin][kLine];
    __shared__ float2 ml[4][32];
    __shared__ intx4 qs[Parts<T>::QP][2 * DB][64];
    Work w;
    if (!find_work<32>(a, w)) return;
    const int lane = threadIdx.x & 63, i = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Row row = find_row(a, w, w.row0 + i);
    int from, until;
    w.keys(a, w.row0 + 31, from, until);
    if (a.splits > 1 && from >= until) {   // a split past the sequence's end
        if (wave == 0 && h == 0 && row.is)
            a.ml[(int64_t(w.split) * a.n.tokens + row.tok) * a.heads + row.head] = make_float2(-INFINITY, 0.f);
        return;
    }
#pragma unroll
    for (int y = 0; y < DB / 2; ++y) {
        typename Parts<T>::Op x[Parts<T>::QP];
        const int c = wave * (DB / 2) + y;
        load_q1<T>(a, row, q_at(c, h), 1.f, x);
#pragma unroll
        for (int p = 0; p < Parts<T>::QP; ++p) qs[p][c][lane] = __builtin_bit_cast(intx4, x[p]);
    }
    __syncthreads();
    const SharedQ<T, DB> q{&qs[0][0][lane]};
    Sums<DB> s;
    bool fine = Direct<T, FMT, PP, DB, SharedQ<T, DB>, share_tiles<T, DB>>(a, w, row, q, s)
                          .template walk<4 * kKeys>(from + wave * kKeys, until, w.lim(a, w.token(a, w.row0)),
                                                    w.low(a, w.token(a, w.row0 + 31)), scales + wave * 64);
    if constexpr (kPartsApart<T, FMT>) fine = fine && !s.none();
    if (__syncthreads_or(!fine)) {        // then the first wave takes all keys
        s.clear();
        if (wave == 0) slow_sums<T, FMT, DB, SharedQ<T, DB>>(late_args(), w, row, q, h, from, until, s);
    }
    s.l += other_half(s.l);
    if (h == 0) ml[wave][i] = make_float2(s.m, s.l);
    join_waves<T, kJoin, kLine>(late_args(), w, sums, ml, min(32, w.rows - w.row0), [&](int r0) {
        if (i >= r0 && i < r0 + kJoin) {
            float *to = sums[wave][i - r0];
#pragma unroll
            for (int r = 0; r < 16; ++r)
#pragma unroll
                for (int blk = 0; blk < DB; blk += 2)
                    *reinterpret_cast<floatx2 *>(to + DB * key_of(r, h) + blk) = floatx2{s.o[blk][r], s.o[blk + 1][r]};
        }
    });
}

// Each wave has rows of its own and reads keys by itself: where its registers (sums of 256 values, or fp32 queries in
// three parts) leave one wave a SIMD unit, so that none would wait beside another at a tile's barrier.  The vector unit's
// decoding bounds it, once a wave: four prompts of 2048 tokens of 32 heads over 8 of 256 take 848 to 856 us, 325
// TFLOP/s; one in fp32, of 128, 173 us, 199.
template <typename T, int FMT, int PP, int DB>
__global__ __launch_bounds__(256, (attn8_groups(kAttnOwn, sizeof(T) == 4, DB))) void attn8_own(AttnArgs a) {
    __shared__ __attribute__((aligned(16))) float scales[4 * 64];
    Work w;
    if (!find_work<128>(a, w)) return;
    const int lane = threadIdx.x & 63, i = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row0 = w.row0 + 32 * wave;
    if (row0 >= w.rows) return;
    const Row row = find_row(a, w, row0 + i);
    HeldQ<T, DB> q;
    load_q<T, DB>(a, row, h, 1.f, q.q);
    int from, until;
    w.keys(a, row0 + 31, from, until);
    Sums<DB> s;
    from = max(from, w.low(a, w.token(a, row0)) & ~(kKeys - 1));
    bool fine = Direct<T, FMT, PP, DB, HeldQ<T, DB>, DB == 8 ? 1 : 2>(a, w, row, q, s)
                          .template walk<kKeys>(from, until, w.lim(a, w.token(a, row0)), w.low(a, w.token(a, row0 + 31)),
                                                scales + wave * 64);
    if constexpr (kPartsApart<T, FMT>) fine = fine && !s.none();
    if (!fine) slow_sums<T, FMT, DB, HeldQ<T, DB>>(late_args(), w, row, q, h, from, until, s);
    s.l += other_half(s.l);
    finish<T, DB>(late_args(), w, row, s, h);
}

// ---- up to 16 rows -------------------------------------------------------------------------------

// The same on 16x16x32 instructions: half of the weights, and of the sums' registers.  Lane (i, g), i = lane % 16,
// g = lane / 16, has S of row i and keys 4 g .. 4 g + 3 of each 16, and as the second operand of the second product
// P of row i and those eight keys.  Both operands of the first product take values 64 c + 16 g + 8 u and on.
__device__ __forceinline__ floatx4 mma16(bf16x8 a, bf16x8 b, floatx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ floatx4 mma16(f16x8 a, f16x8 b, floatx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
// Over the four lanes of a row.
template <typename Fn>
__device__ __forceinline__ float over_groups(float v, Fn fn) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fn(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fn(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

template <typename T, int FMT, bool POW2, int PP, int DB>
struct Few {
    using P = Parts<T>;
    using Op = typename P::Op;
    static constexpr bool kFoldK = POW2 && std::is_same_v<Op, bf16x8>;
    static constexpr int NB = 2 * DB;                              // blocks of 16 values, a lane's bytes of a key of V
    static constexpr int W = NB / 4;

    struct Tile {
        intx4 k[2][DB / 2];
        unsigned v[8][W];                 // keys 4 g + e of the first 16, then of the second
        unsigned s;                       // the scale as stored of key lane % 32: K's in lanes 0 to 31, V's in the others
        int valid[2];
    };
    struct Pages {
        PageRef p[2];
    };

    const AttnArgs &a;
    const Work &w;
    const Row &row;
    const float c;                        // what sums are multiplied with (powers of two in K's operands)
    const int lane, i, g;
    const unsigned koff, voff;
    const int32_t *table;
    Op q[P::QP][DB];
    floatx4 o[NB];
    float m, l;                           // l: of the lane's keys

    __device__ __forceinline__ Few(const AttnArgs &a_, const Work &w_, const Row &r_)
        : a(a_), w(w_), row(r_), c(a_.scale == 0.f ? 1.f : fabsf(a_.scale)), lane(threadIdx.x & 63), i(lane & 15),
          g(lane >> 4), koff(i * a_.c.dim), voff(4 * g * a_.c.dim + min(NB * i, a_.c.dim - NB)),
          table(a_.n.table + int64_t(w_.b) * a_.n.tld) {
        const float sign = a.scale < 0.f ? -1.f : a.scale > 0.f ? 1.f : 0.f;
#pragma unroll
        for (int x = 0; x < DB; ++x) {
            Op part[P::QP];
            load_q1<T>(a, row, 64 * (x >> 1) + 16 * g + 8 * (x & 1), kFoldK ? sign : 1.f, part);
#pragma unroll
            for (int p = 0; p < P::QP; ++p) q[p][x] = part[p];
        }
        m = -INFINITY;
        l = 0.f;
#pragma unroll
        for (int blk = 0; blk < NB; ++blk) o[blk] = floatx4{};
    }

    __device__ __forceinline__ Pages pages(int key0) const {
        return {page_ref(a, table, w.len, key0), page_ref(a, table, w.len, key0 + 16)};
    }

    __device__ __forceinline__ void load(Tile &t, const Pages &from, int key0) const {
        const int dim = a.c.dim;
        int64_t se[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const int id = page_of(a, from.p[b]);
            t.valid[b] = id >= 0 ? min(16, max(w.len - key0 - 16 * b, 0)) : 0;
            const int64_t page = max(id, 0), at = w.head * a.c.page + from.p[b].off;
            const uint8_t *k = a.c.k + page * a.c.stride + at * dim, *v = a.c.v + page * a.c.stride + at * dim;
#pragma unroll
            for (int x = 0; x < DB / 2; ++x)
                t.k[b][x] = *reinterpret_cast<const intx4 *>(k + koff + min(64 * x + 16 * g, dim - 16));
            // V's whole lines pass the caches by: where a sequence's rows are one tile, as the form is chosen for, no other
            // workgroup reads them (a sequence of more rows than the average does, and reads them from memory again for each
            // tile).  The halves of K's that two loads share do not (64 sequences of up to 8192 keys 126.5 -> 120.3 us, K's
            // too 137; of 8192 each 260 -> 241, 245; four waves a workgroup)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint8_t *vp = v + e * dim + voff;
                if constexpr (W == 1) {
                    t.v[4 * b + e][0] = __builtin_nontemporal_load(reinterpret_cast<const unsigned *>(vp));
                } else {
                    typedef int intw __attribute__((ext_vector_type(W)));
                    const intw x = __builtin_nontemporal_load(reinterpret_cast<const intw *>(vp));
#pragma unroll
                    for (int word = 0; word < W; ++word) t.v[4 * b + e][word] = x[word];
                }
            }
            se[b] = page * a.c.sstride + at;
        }
        t.s = load_scale(lane < 32 ? a.c.ks : a.c.vs, POW2 ? DS_SCALE_POW2 : DS_SCALE_F32, (lane & 16 ? se[1] : se[0]) + i);
    }

    __device__ __forceinline__ void follow(float top) {
        if (__any(top > m + kLoose || (m == -INFINITY && top > -INFINITY))) {
            const float now = fmaxf(m, top);
            const float by = now == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - now);
            m = now;
            l *= by;
#pragma unroll
            for (int blk = 0; blk < NB; ++blk) o[blk] *= by;
        }
    }
    // Whether a sum of the wave's is no number.
    __device__ __forceinline__ bool none() const {
        bool is = l != l;
#pragma unroll
        for (int blk = 0; blk < NB; ++blk)
#pragma unroll
            for (int r = 0; r < 4; ++r) is |= o[blk][r] != o[blk][r];
        return __any(is);
    }
    __device__ __forceinline__ float largest(const float (&x)[8]) const {
        const float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
        return over_groups(top, [](float y, float z) { return fmaxf(y, z); }) * (kFoldK ? c : 1.f);
    }

    // One tile of 32 keys; edge: some row does not see some key of it, or some key does not exist.  False where that
    // needs slow_sums.  begun: all rows have a maximum.
    __device__ __forceinline__ bool step(Tile &t, int key0, bool edge, bool &begun, float *lds) {
        float sc = scale_of(t.s, POW2 ? DS_SCALE_POW2 : DS_SCALE_F32);
        if (edge) sc = i < (lane & 16 ? t.valid[1] : t.valid[0]) ? sc : 0.f;
        lds[lane] = kFoldK || lane >= 32 ? sc : sc * a.scale;
        __builtin_amdgcn_wave_barrier();
        if (a.c.dim < 32 * DB)                // (a number that is none times Q's 0 is no 0)
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int x = 0; x < DB / 2; ++x)
                    if (64 * x + 16 * g >= a.c.dim) t.k[b][x] = intx4{};
        floatx4 sum[2] = {};
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const float by = kFoldK ? lds[16 * b + i] : 1.f;
#pragma unroll
            for (int x = 0; x < DB; ++x) {
                const Op k = decode_k<FMT, Op>(t.k[b][x >> 1][2 * (x & 1)], t.k[b][x >> 1][2 * (x & 1) + 1], by);
#pragma unroll
                for (int p = P::QP - 1; p >= 0; --p) sum[b] = mma16(k, q[p][x], sum[b]);
            }
        }
        float x[8];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            floatx4 sk;
            if constexpr (!kFoldK) sk = *reinterpret_cast<const floatx4 *>(lds + 16 * b + 4 * g);
#pragma unroll
            for (int r = 0; r < 4; ++r) x[4 * b + r] = kFoldK ? sum[b][r] : sum[b][r] * sk[r];
        }
        if (edge) {
            int low = row.low - key0 - 4 * g, lim = row.lim - key0 - 4 * g, has[2] = {t.valid[0] - 4 * g, t.valid[1] - 4 * g};
            __asm__ volatile("" : "+v"(low), "+v"(lim), "+v"(has[0]), "+v"(has[1]));
            unsigned bad = lane >= 32 && !(fabsf(sc) < INFINITY);    // (values' scales)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int k = 16 * (e >> 2) + (e & 3);
                x[e] = k >= low && k < lim && (e & 3) < has[e >> 2] ? x[e] : -INFINITY;
#pragma unroll
                for (int word = 0; word < W; ++word) {
                    if ((e & 3) >= has[e >> 2]) t.v[e][word] = 0;
                    bad |= not_finite<FMT>(t.v[e][word]);
                }
            }
            if (__any(bad != 0)) return false;
        }
        if (edge || !begun) {
            follow(largest(x));
            begun = __all(m > -INFINITY);
        }
        const floatx4 sv[2] = {*reinterpret_cast<const floatx4 *>(lds + 32 + 4 * g),
                               *reinterpret_cast<const floatx4 *>(lds + 48 + 4 * g)};
        __builtin_amdgcn_wave_barrier();
        bf16x8 pt[PP];
        float part = 0.f;
        const auto weigh = [&]() {
            const float off = m == -INFINITY ? 0.f : m;
            part = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float p = __builtin_amdgcn_exp2f(kFoldK ? __builtin_fmaf(x[e], c, -off) : x[e] - off);
                part += p;
                put_weight<PP, FMT>(pt, e, p * sv[e >> 2][e & 3]);
            }
        };
        weigh();
        // (see Tiles::weights)
        if (__any(part >= float(1 << int(kLoose)))) {
            follow(largest(x));
            weigh();
        }
        l += part;
#pragma unroll
        for (int blk = 0; blk < NB; ++blk) {
            const int word = blk >> 2, j = blk & 3;
            bf16x8 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const unsigned pair = __builtin_amdgcn_perm(t.v[2 * e + 1][word], t.v[2 * e][word], j & 2 ? 0x07030602u : 0x05010400u);
                const bf16x2 y = j & 1 ? decode2<FMT, true>(pair, 1.f) : decode2<FMT, false>(pair, 1.f);
                v[2 * e] = y[0];
                v[2 * e + 1] = y[1];
            }
#pragma unroll
            for (int p = PP - 1; p >= 0; --p) o[blk] = mma16(v, pt[p], o[blk]);
        }
        return true;
    }

    template <int STEP>
    __device__ __forceinline__ bool walk(int key, int until, int every, int since, float *lds) {
        bool fine = true, begun = false;
        const auto edge = [&](const Tile &t) {
            return key + kKeys > every || key < since || (t.valid[0] & t.valid[1]) != 16;
        };
        if (key >= until) return true;
        Tile t[2];
        load(t[0], pages(key), key);
        Pages next = pages(key + STEP);
        while (true) {
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const Pages after = pages(key + 2 * STEP);
                if (key + STEP < until) load(t[x ^ 1], next, key + STEP);
                next = after;
                fine = step(t[x], key, edge(t[x]), begun, lds);
                key += STEP;
                if (!fine || key >= until) return fine;
            }
        }
    }
};

// As attn8_share, for up to 16 rows, of four waves or eight (figures above).
template <typename T, int FMT, bool POW2, int PP, int DB>
__global__ __launch_bounds__(attn8_threads(kAttnFew, DB), (attn8_groups(kAttnFew, sizeof(T) == 4, DB) * attn8_threads(kAttnFew, DB) / 256)) void attn8_few(AttnArgs a) {
    constexpr int kWaves = attn8_threads(kAttnFew, DB) / 64;
    constexpr int kJoin = DB >= 4 ? 8 : 16, kLine = 32 * DB + 4;      // rows at a time, floats between them
    __shared__ __attribute__((aligned(16))) float scales[kWaves * 64];
    __shared__ __attribute__((aligned(16))) float sums[kWaves][kJoin][kLine];
    __shared__ float2 ml[kWaves][16];
    Work w;
    if (!find_work<16>(a, w)) return;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Row row = find_row(a, w, w.row0 + (lane & 15));
    int from, until;
    w.keys(a, w.row0 + 15, from, until);
    if (a.splits > 1 && from >= until) {   // a split past the sequence's end
        if (wave == 0 && lane < 16 && row.is)
            a.ml[(int64_t(w.split) * a.n.tokens + row.tok) * a.heads + row.head] = make_float2(-INFINITY, 0.f);
        return;
    }
    Few<T, FMT, POW2, PP, DB> s(a, w, row);
    bool fine = s.template walk<kWaves * kKeys>(from + wave * kKeys, until, w.lim(a, w.token(a, w.row0)),
                                                 w.low(a, w.token(a, w.row0 + 15)), scales + wave * 64);
    if constexpr (kPartsApart<T, FMT>) fine = fine && !s.none();
    const AttnArgs al = late_args();
    if (__syncthreads_or(!fine)) {        // then the first wave takes all keys, in the other form's order
        if (wave > 0) return;
        row = find_row(al, w, w.row0 + (lane & 31));
        row.is = row.is && (lane & 31) < 16;
        HeldQ<T, DB> held;
        load_q<T, DB>(al, row, lane >> 5, 1.f, held.q);
        Sums<DB> all;
        slow_sums<T, FMT, DB, HeldQ<T, DB>>(al, w, row, held, lane >> 5, from, until, all);
        all.l += other_half(all.l);
        finish<T, DB>(al, w, row, all, lane >> 5);
        return;
    }
    s.l = over_groups(s.l, [](float x, float y) { return x + y; });
    if (lane < 16) ml[wave][lane] = make_float2(s.m, s.l);
    join_waves<T, kJoin, kLine>(al, w, sums, ml, min(16, w.rows - w.row0), [&](int r0) {
        if (s.i >= r0 && s.i < r0 + kJoin) {
            float *to = sums[wave][s.i - r0];
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int blk = 0; blk < 2 * DB; blk += 4)
                    *reinterpret_cast<floatx4 *>(to + 2 * DB * (4 * s.g + r) + blk) =
                        floatx4{s.o[blk][r], s.o[blk + 1][r], s.o[blk + 2][r], s.o[blk + 3][r]};
        }
    });
}

// ---- keys and values decoded in LDS ---------------------------------------------------------------------

constexpr int kTileKeys = 64;

// Where unit c of row r lies among rows of N 16-byte units: 16 lanes that read the same unit of rows side by side
// meet all 64 banks (rows of 128 bytes lie two in a line of banks).
template <int N>
__device__ __forceinline__ int unit_at(int r, int c) {
    return r * N + (c ^ (N == 8 ? r >> 1 & 7 : r & 15));
}

// A tile as operands of 16 bytes.  K: unit c of row r has values 8 c and on of key r; V: unit 2 st + h of row blk * 32 + i
// has value DB i + blk of the keys of step st and half h, in key_of's order.
template <int DB>
struct TileLds {
    intx4 k[kTileKeys * 4 * DB];
    intx4 v[32 * DB * 8];
    float sk[kTileKeys], sv[kTileKeys];   // fp32 scales, K's times a.scale
    int note[4];                          // of each 16 keys: those that exist, and 1 << 16 if V holds no number
};

// Powers of two go into the operands: into V's (bf16), and into K's if those are bf16 too.
template <typename T, int FMT, bool POW2, int PP, int DB>
struct Tiles {
    using P = Parts<T>;
    using Op = typename P::Op;
    static constexpr bool kFoldK = POW2 && std::is_same_v<Op, bf16x8>, kFoldV = POW2;
    static constexpr int W = DB == 8 ? 2 : 1;
    static constexpr int kPieces = 2 * DB;                         // 16-byte pieces of a row of K
    static constexpr int kLoads = DB / 2;                          // of a thread
    static_assert(kLoads <= 2, "a thread holds two scales");
    static constexpr bool kEarly = PP == 1 && POW2;                // registers for V's operands before the weights are there

    const AttnArgs &a;
    const Work &w;
    const int lane, i, h, wave;

    // What a thread holds of a tile.  Waves 0 to 3 take K's keys 16 wave and on, waves 4 to 7 V's: one page each.
    struct Stage {
        unsigned raw[8 * W];
        unsigned sc0, sc1;                // scales as stored: of a K thread's loads, of a V thread's keys
        int valid;
    };
    // What does not change from tile to tile: where the wave's head begins in page 0, and the lane's bytes there.
    struct Where {
        const uint8_t *rows;
        const void *scales;
        const int32_t *table;
        unsigned lane;
        int part;                         // the wave's keys of a tile: 16 part and on
    };
    __device__ __forceinline__ Where where() const {
        const int64_t head = int64_t(w.head) * a.c.page;
        const int dim = a.c.dim, part = wave & 3;
        const void *sp = wave < 4 ? a.c.ks : a.c.vs;
        const unsigned at = wave < 4 ? unsigned(lane / kPieces * dim + min(16 * (lane % kPieces), dim - 16))
                                     : unsigned(4 * h * dim + v_column<DB>(i, dim));
        return {(wave < 4 ? a.c.k : a.c.v) + head * dim,
                POW2 ? static_cast<const void *>(static_cast<const uint8_t *>(sp) + head)
                     : static_cast<const void *>(static_cast<const unsigned *>(sp) + head),
                a.n.table + int64_t(w.b) * a.n.tld, at, part};
    }
    // The page that the wave loads of a tile: a tile ahead of the loads.
    __device__ __forceinline__ PageRef page(const Where &to, int key0) const {
        return page_ref(a, to.table, w.len, key0 + 16 * to.part);
    }

    __device__ __forceinline__ void load(Stage &st, const Where &to, const PageRef &from, int key0) const {
        const int dim = a.c.dim, id = page_of(a, from);
        st.valid = id >= 0 ? min(16, max(w.len - key0 - 16 * to.part, 0)) : 0;
        const int64_t page = max(id, 0);
        const uint8_t *rows = to.rows + page * a.c.stride + from.off * dim;
        const int64_t se = page * a.c.sstride + from.off;
        if (wave < 4) {
#pragma unroll
            for (int j = 0; j < kLoads; ++j) {
                const intx4 x = *reinterpret_cast<const intx4 *>(rows + j * (64 / kPieces) * dim + to.lane);
#pragma unroll
                for (int e = 0; e < 4; ++e) st.raw[4 * j + e] = x[e];
                const unsigned sc = load_scale(to.scales, POW2 ? DS_SCALE_POW2 : DS_SCALE_F32, se + j * (64 / kPieces) + lane / kPieces);
                if (j == 0) st.sc0 = sc;
                else st.sc1 = sc;
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                unsigned x[W];
                load_v<DB, false>(rows + (e < 4 ? e : e + 4) * dim, to.lane, x);
#pragma unroll
                for (int word = 0; word < W; ++word) st.raw[e * W + word] = x[word];
            }
            if constexpr (kFoldV) {
                const uint8_t *sp = static_cast<const uint8_t *>(to.scales) + se + 4 * h;
                __builtin_memcpy(&st.sc0, sp, 4);
                __builtin_memcpy(&st.sc1, sp + 8, 4);
            } else {
                st.sc0 = static_cast<const unsigned *>(to.scales)[se + (lane & 15)];
            }
        }
    }

    // edge: some row of the workgroup does not see some key of the tile.
    __device__ __forceinline__ void store(Stage &st, TileLds<DB> &t, bool edge) const {
        const int part = wave & 3;
        if (wave < 4) {
#pragma unroll
            for (int j = 0; j < kLoads; ++j) {
                const int r = 16 * part + j * (64 / kPieces) + lane / kPieces, piece = lane % kPieces;
                if (a.c.dim < 32 * DB && 16 * piece >= a.c.dim)      // (a number that is none times Q's 0 is no 0)
#pragma unroll
                    for (int e = 0; e < 4; ++e) st.raw[4 * j + e] = 0;
                const unsigned sc = j == 0 ? st.sc0 : st.sc1;
                // (the conversion looks at the exponent alone)
                const float by = kFoldK ? __uint_as_float(sc << 23) : scale_of(sc, POW2 ? DS_SCALE_POW2 : DS_SCALE_F32);
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const Op k = decode_k<FMT, Op>(st.raw[4 * j + 2 * u], st.raw[4 * j + 2 * u + 1], kFoldK ? by : 1.f);
                    t.k[unit_at<4 * DB>(r, 2 * piece + u)] = __builtin_bit_cast(intx4, k);
                }
                if (!kFoldK && piece == 0) t.sk[r] = by * a.scale;
            }
        } else {
            float by[8];
            if constexpr (kFoldV) {
                // (alike)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const unsigned sc = e < 4 ? st.sc0 : st.sc1;
                    by[e] = __uint_as_float((e % 4 == 3 ? sc >> 1 : sc << (23 - 8 * (e % 4))) & 0x7f800000u);
                }
            }
            if (st.valid < 16) {
                int has = st.valid - 4 * h;
                __asm__ volatile("" : "+v"(has));
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if ((e < 4 ? e : e + 4) >= has) {
                        by[e] = 1.f;
#pragma unroll
                        for (int word = 0; word < W; ++word) st.raw[e * W + word] = 0;
                    }
            }
            int note = st.valid;
            if (edge) {
                unsigned bad = !kFoldV && (lane & 15) < st.valid && (st.sc0 & 0x7f800000u) == 0x7f800000u;
#pragma unroll
                for (int e = 0; e < 8 * W; ++e) bad |= not_finite<FMT>(st.raw[e]);
                // (and powers of two that take the format's largest number past 2^128, to an infinity as an operand; looking
                // at the operands themselves costs tiles that all rows see 1%)
                constexpr unsigned kPast = (127u + (FMT == DS_Q8_E4M3 ? 120u : 113u)) << 23;
                if constexpr (kFoldV)
#pragma unroll
                    for (int e = 0; e < 8; ++e) bad |= __float_as_uint(by[e]) >= kPast;
                note |= __any(bad != 0) ? 1 << 16 : 0;
            }
#pragma unroll
            for (int word = 0; word < W; ++word)
#pragma unroll
                for (int pair = 0; pair < (DB == 2 ? 1 : 2); ++pair) {
                    unsigned x[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const unsigned raw = st.raw[e * W + word];
                        const float s = kFoldV ? by[e] : 1.f;
                        x[e] = __builtin_bit_cast(unsigned, pair ? decode2<FMT, true>(raw, s) : decode2<FMT, false>(raw, s));
                    }
#pragma unroll
                    for (int odd = 0; odd < 2; ++odd) {
                        intx4 y;
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            y[e] = int(__builtin_amdgcn_perm(x[2 * e + 1], x[2 * e], odd ? 0x07060302u : 0x05040100u));
                        const int blk = 4 * word + 2 * pair + odd;
                        t.v[unit_at<8>(blk * 32 + i, 2 * part + h)] = y;
                    }
                }
            if (!kFoldV && lane < 16) t.sv[16 * part + lane] = lane < st.valid ? __uint_as_float(st.sc0) : 0.f;
            if (lane == 0) t.note[part] = note;
        }
    }

    // K's operands of 32 keys.
    __device__ __forceinline__ void read_k(const TileLds<DB> &t, int sub, Op (&k)[2 * DB]) const {
#pragma unroll
        for (int x = 0; x < 2 * DB; ++x)
            k[x] = __builtin_bit_cast(Op, t.k[unit_at<4 * DB>(32 * sub + i, 4 * (x >> 1) + 2 * h + (x & 1))]);
    }
    __device__ __forceinline__ bf16x8 read_v(const TileLds<DB> &t, int sub, int st, int blk) const {
        return __builtin_bit_cast(bf16x8, t.v[unit_at<8>(blk * 32 + i, 4 * sub + 2 * st + h)]);
    }

    // A step takes 32 keys in two parts, in each of which the matrix unit works on one thing and the vector unit on another:
    // the weights of these keys beside the scores of the next, and the product with V beside the next scores' scales.
    // The row's weights of scores x, and the scores of the next keys.  Weights that come out at 2^kLoose or more say
    // that the running maximum is too far behind, and are taken again; without them it is not looked at.
    __device__ __forceinline__ void weights(const TileLds<DB> &t, int sub, const float (&x)[16], float c,
                                            const Op (&k)[2 * DB], const Op (&q)[P::QP][2 * DB], Sums<DB> &s,
                                            bf16x8 (&pt)[2][PP], floatx16 &next, bf16x8 (&v)[DB][2]) const {
        // V's operands for what follows: half of them in the registers that K's leave
        if constexpr (kEarly)
#pragma unroll
            for (int blk = 0; blk < DB; ++blk) v[blk][0] = read_v(t, sub, 0, blk);
        const float off = s.base();
        next = floatx16{};
        float l[2] = {0.f, 0.f};
        floatx4 sv;
        const auto weigh = [&](int r, float from) {
            if constexpr (!kFoldV)
                if (r % 4 == 0) sv = *reinterpret_cast<const floatx4 *>(t.sv + 32 * sub + 2 * r + 4 * h);
            const float p = __builtin_amdgcn_exp2f(kFoldK ? __builtin_fmaf(x[r], c, -from) : x[r] - from);
            l[r & 1] += p;
            put_weight<PP, FMT>(pt[r >> 3], r & 7, kFoldV ? p : p * sv[r & 3]);
        };
        // (in this order: a wave that waits for its own matrix instructions would leave the vector unit idle)
        constexpr int kEach = 16 / (2 * DB);
#pragma unroll
        for (int y = 0; y < 2 * DB; ++y) {
#pragma unroll
            for (int p = P::QP - 1; p >= 0; --p) next = mma(k[y], q[p][y], next);
            if (kEarly && y >= DB) v[y - DB][1] = read_v(t, sub, 1, y - DB);
#pragma unroll
            for (int r = kEach * y; r < kEach * (y + 1); ++r) weigh(r, off);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (__any(l[0] + l[1] >= float(1 << int(kLoose)))) {
            float top = largest(x);
            top = fmaxf(top, other_half(top));
            s.follow(kFoldK ? top * c : top);
            l[0] = l[1] = 0.f;
            const float now = s.base();
#pragma unroll
            for (int r = 0; r < 16; ++r) weigh(r, now);
        }
        s.l += l[0] + l[1];
        if constexpr (!kEarly)
#pragma unroll
            for (int blk = 0; blk < DB; ++blk)
#pragma unroll
                for (int st = 0; st < 2; ++st) v[blk][st] = read_v(t, sub, st, blk);
    }
    // Their product with V, and x: the next scores, times K's scales.
    __device__ __forceinline__ void product(const bf16x8 (&v)[DB][2], const bf16x8 (&pt)[2][PP], Sums<DB> &s,
                                            const floatx16 &next, const TileLds<DB> &t, int sub, float (&x)[16]) const {
        floatx4 sk;
        constexpr int kEach = 16 / (2 * DB);
#pragma unroll
        for (int y = 0; y < 2 * DB; ++y) {
            const int st = y / DB, blk = y % DB;
#pragma unroll
            for (int part = PP - 1; part >= 0; --part) s.o[blk] = mma(v[blk][st], pt[st][part], s.o[blk]);
#pragma unroll
            for (int r = kEach * y; r < kEach * (y + 1); ++r) {
                if constexpr (!kFoldK)
                    if (r % 4 == 0) sk = *reinterpret_cast<const floatx4 *>(t.sk + 32 * sub + 2 * r + 4 * h);
                x[r] = kFoldK ? next[r] : next[r] * sk[r & 3];
            }
            if constexpr (!kFoldK) __builtin_amdgcn_sched_barrier(0);
        }
    }
    __device__ __forceinline__ float largest(const float (&x)[16]) const {
        float top = fmaxf(x[0], x[1]);
#pragma unroll
        for (int r = 2; r < 16; r += 2) top = fmaxf(fmaxf(top, x[r]), x[r + 1]);
        return top;
    }
    // The scores that the row does not see out of x (edge: there are some in the wave), and the maximum followed.
    // True when all rows of the wave have seen some key.
    __device__ __forceinline__ bool mask(float (&x)[16], int key0, int sub, bool edge, const intx4 &note, float c,
                                         const Row &row, Sums<DB> &s) const {
        if (edge) {
            const int at = key0 + 32 * sub + 4 * h;
            const int low = row.low - at, lim = row.lim - at;
            const int has = (note[2 * sub] & 0xffff) - 4 * h, has1 = (note[2 * sub + 1] & 0xffff) - 4 * h;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int k1 = key_of(r, 0);
                const bool sees = k1 >= low && k1 < lim && (k1 & 15) < (r < 8 ? has : has1);
                x[r] = sees ? x[r] : -INFINITY;
            }
        }
        float top = largest(x);
        top = fmaxf(top, other_half(top));
        s.follow(kFoldK ? top * c : top);
        return __all(s.m > -INFINITY);
    }
};

// Waits for the waves' LDS accesses, and not for loads from memory that are on their way.
__device__ __forceinline__ void lds_barrier() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// Eight waves of 32 rows each, which all walk over the workgroup's keys.  The matrix unit (40% of the time) and the vector
// unit (as much) bound it: a prompt of 8192 tokens of 32 heads over 8 of 128 takes 590 to 602 us in bf16, 888 to 895 with fp32
// scales (weights in two parts, a product a weight and score more), 829 to 845 in fp16 (weights in two parts); of 64
// values 453.  Three tiles in LDS: one is used, the next is written
// (the one after is on its way from memory), and the third may still be read by a wave that is behind: one
// barrier a tile.
template <typename T, int FMT, bool POW2, int PP, int DB>
__global__ __launch_bounds__(512, 2) void attn8_tiles(AttnArgs a) {
    extern __shared__ __attribute__((aligned(16))) unsigned char lds_bytes[];
    TileLds<DB> *lds = reinterpret_cast<TileLds<DB> *>(lds_bytes);
    using Tl = Tiles<T, FMT, POW2, PP, DB>;
    Work w;
    if (!find_work<256>(a, w)) return;
    const int lane = threadIdx.x & 63, i = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row0 = w.row0 + 32 * wave;
    const Row row = find_row(a, w, row0 + i);
    int from, until;
    w.keys(a, w.row0 + 255, from, until);
    // what all rows of the workgroup see, and of the wave
    const int wg_every = w.lim(a, w.token(a, w.row0)), wg_since = w.low(a, w.token(a, w.row0 + 255));
    const int every = w.lim(a, w.token(a, row0)), since = w.low(a, w.token(a, row0 + 31));
    typename Parts<T>::Op q[Parts<T>::QP][2 * DB];
    // powers of two in K's operands leave one factor for all sums; its sign goes into Q, so that the
    // largest sum is the largest score
    const float sign = a.scale < 0.f ? -1.f : a.scale > 0.f ? 1.f : 0.f, c = a.scale == 0.f ? 1.f : fabsf(a.scale);
    load_q<T, DB>(a, row, h, Tl::kFoldK ? sign : 1.f, q);
    Sums<DB> s;
    s.clear();
    const Tl tl{a, w, lane, i, h, wave};
    bool fine = true;
    if (from < until) {
        typename Tl::Stage st;
        const typename Tl::Where to = tl.where();
        const auto wg_edge = [&](int key) { return key + kTileKeys > wg_every || key < wg_since; };
        tl.load(st, to, tl.page(to, from), from);
        PageRef page = tl.page(to, from + kTileKeys);
        tl.store(st, lds[0], wg_edge(from));
        if (from + kTileKeys < until) {
            const PageRef p = page;
            page = tl.page(to, from + 2 * kTileKeys);
            tl.load(st, to, p, from + kTileKeys);
        }
        lds_barrier();
        intx4 note;
        bool edge = false;
        // the notes of the tile at `key`; false if it needs slow_sums
        const auto look = [&](const TileLds<DB> &t, int key) {
            note = *reinterpret_cast<const intx4 *>(t.note);
#pragma unroll
            for (int e = 0; e < 4; ++e) note[e] = __builtin_amdgcn_readfirstlane(note[e]);
            edge = key + kTileKeys > every || key < since || (note[0] & note[1] & note[2] & note[3] & 0xffff) != 16;
            return !((note[0] | note[1] | note[2] | note[3]) >> 16);
        };
        typename Tl::Op k[2 * DB];
        bf16x8 v[DB][2], pt[2][PP];
        floatx16 next = {};
        float x[16];
        bool begun = false;                // all rows have a maximum
        fine = look(lds[0], from);
        tl.read_k(lds[0], 0, k);
#pragma unroll
        for (int y = 0; y < 2 * DB; ++y)
#pragma unroll
            for (int p = Parts<T>::QP - 1; p >= 0; --p) next = mma(k[y], q[p][y], next);
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r] = Tl::kFoldK ? next[r] : next[r] * lds[0].sk[key_of(r, h)];
        tl.read_k(lds[0], 1, k);
        int at = 0;
        for (int key = from; fine; key += kTileKeys) {
            const TileLds<DB> &t = lds[at];
            const int after = at == 2 ? 0 : at + 1;
            const bool more = key + kTileKeys < until;
            if (edge || !begun) begun = tl.mask(x, key, 0, edge, note, c, row, s);
            if (more) {
                tl.store(st, lds[after], wg_edge(key + kTileKeys));
                if (key + 2 * kTileKeys < until) {
                    const PageRef p = page;
                    page = tl.page(to, key + 3 * kTileKeys);
                    tl.load(st, to, p, key + 2 * kTileKeys);
                }
            }
            tl.weights(t, 0, x, c, k, q, s, pt, next, v);
            const bool hidden = edge;
            const intx4 now = note;
            if (more) {
                lds_barrier();
                fine = look(lds[after], key + kTileKeys);
            }
            // (behind the last tile the scores of whatever lies there, which nobody takes)
            if constexpr (Tl::kEarly) tl.read_k(lds[after], 0, k);
            tl.product(v, pt, s, next, t, 1, x);
            if constexpr (!Tl::kEarly) tl.read_k(lds[after], 0, k);
            if (hidden || !begun) begun = tl.mask(x, key, 1, hidden, now, c, row, s);
            tl.weights(t, 1, x, c, k, q, s, pt, next, v);
            if constexpr (Tl::kEarly) tl.read_k(lds[after], 1, k);
            tl.product(v, pt, s, next, lds[after], 0, x);
            if constexpr (!Tl::kEarly) tl.read_k(lds[after], 1, k);
            if (!more) break;
            at = after;
        }
    }
    if constexpr (kPartsApart<T, FMT>) fine = fine && !s.none();
    const AttnArgs al = late_args();
    if (!fine) {
        HeldQ<T, DB> held;
        load_q<T, DB>(al, row, h, 1.f, held.q);
        slow_sums<T, FMT, DB, HeldQ<T, DB>>(al, w, row, held, h, from, until, s);
    }
    s.l += other_half(s.l);
    finish<T, DB>(al, w, row, s, h);
}

}  // namespace

template <typename T>
AttnKernel attn8_kernel(int form, int fmt, int stype, int dim, bool exact) {
    AttnKernel k{nullptr, 0};
    const auto of_parts = [&](auto f, auto pow2, auto parts, auto db) {
        constexpr int FMT = f.value, PP = parts.value, DB = db.value;
        constexpr bool POW2 = pow2.value;
        if (form == kAttnFew) {
            k.func = reinterpret_cast<const void *>(&attn8_few<T, FMT, POW2, PP, DB>);
        } else if (form == kAttnShare) {
            k.func = reinterpret_cast<const void *>(&attn8_share<T, FMT, PP, DB>);
        } else if (form == kAttnOwn) {
            if constexpr (attn8_own_form<T>(DB)) k.func = reinterpret_cast<const void *>(&attn8_own<T, FMT, PP, DB>);
        } else {
            if constexpr (!attn8_own_form<T>(DB)) {
                k.func = reinterpret_cast<const void *>(&attn8_tiles<T, FMT, POW2, PP, DB>);
                k.lds = 3 * int(sizeof(TileLds<DB>));
            }
        }
    };
    // A weight's parts go by the types (and the caller's choice) alone, so that a token's rounding is the same beside any
    // others.  Times an fp32 scale a weight takes two parts for bf16 too: a row of one key comes out as exact as its value,
    // where a power of two loses nothing of a weight of 1.  That costs 64 sequences of up to 8192 keys 5% (one token each) and 10% (four), and a
    // prompt of 8192 tokens 33% (675 us in one part, 895 in two), of heads of 256 13%; over powers of two, where the caller
    // may ask for it, 4%, 11%, 34% (593 and 795) and 10%.
    const auto of_dim = [&](auto f, auto db) {
        constexpr int kLess = Parts<T>::PP, kMore = kLess < 2 ? 2 : kLess;
        if (stype != DS_SCALE_POW2) of_parts(f, std::false_type{}, std::integral_constant<int, kMore>{}, db);
        else if (exact) of_parts(f, std::true_type{}, std::integral_constant<int, kMore>{}, db);
        else of_parts(f, std::true_type{}, std::integral_constant<int, kLess>{}, db);
    };
    const auto of_fmt = [&](auto f) {
        const int db = attn8_dim_blocks(dim);
        if (db == 2) of_dim(f, std::integral_constant<int, 2>{});
        else if (db == 4) of_dim(f, std::integral_constant<int, 4>{});
        else if constexpr (!std::is_same_v<T, float>) of_dim(f, std::integral_constant<int, 8>{});
    };
    if (fmt == DS_Q8_E4M3) of_fmt(std::integral_constant<int, DS_Q8_E4M3>{});
    else of_fmt(std::integral_constant<int, DS_Q8_E5M2>{});
    return k;
}

}  // namespace ds
