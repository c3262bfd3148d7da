// Attention of new tokens over the paged 8-bit cache.
//
// For one cache head a row is a pair of a new token and one of the query heads that share it.  A wave takes 32 (or
// 64) rows and walks over tiles of 32 keys with the running maximum m and sum l of each row's softmax.  It
// computes the products transposed, on 32x32x16 matrix instructions:
//     S^T = K Q^T:  lane (i, h), i = lane % 32, h = lane / 32, has S of row i and 16 of the tile's keys,
//     O^T = V^T P^T: and the same lane needs P of row i and 8 keys an instruction as the second operand:
// those that it holds, if V's keys are taken in the same order.  So weights never leave their lane, and a
// row's maximum is one of 16 registers and one exchange of halves.  Keys and values come from memory
// as they lie: a lane's 16 bytes of a key's row are the first operand of two instructions (Q in the same order of
// values), and its 4 bytes (dims up to 128) of eight keys' rows are those of four, transposed by byte
// permutes, a value and its neighbour key's in one conversion.  There is no LDS on that way and no barrier.
#pragma once

#include <type_traits>

#include "attn8.h"
#include "kern_common.h"
#include "q8.h"

namespace ds {
namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// How the types compute: Q in QP parts of operand type, P in PP parts of bf16.
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

// Eight bytes of a key's row as an operand: exact in both types.
template <int FMT, typename Op>
__device__ __forceinline__ Op decode_k(int lo, int hi) {
    if constexpr (std::is_same_v<Op, bf16x8>) {
        return to_bf16<FMT>(lo, hi);
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

// Any byte of the word that stands for no finite number.
template <int FMT>
__device__ __forceinline__ unsigned not_finite(unsigned w) {
    if constexpr (FMT == DS_Q8_E4M3) return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
    else return ((w & 0x7c7c7c7cu) + 0x04040404u) & 0x80808080u;
}

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

template <typename T, int FMT, int DB, int NQ, bool SHARE>
struct Attn {
    using P = Parts<T>;
    using Op = typename P::Op;
    static constexpr int kRows = 32 * NQ;                          // of a wave
    static constexpr int kTileRows = SHARE ? kRows : kWaves * kRows;

    const AttnArgs &a;
    const int lane, i, h;
    int b, head;                                                   // sequence, cache head (uniform)
    int len;                                                       // its keys that may be seen
    const uint8_t *kbase, *vbase;
    unsigned koff, voff;                                                // of the lane in a 16-key part of a page
    Op q[P::QP][NQ][2 * DB];
    floatx16 o[NQ][DB];
    float m[NQ], l[NQ];
    int lim[NQ], low[NQ];                                          // the row sees keys low .. lim - 1

    __device__ __forceinline__ Attn(const AttnArgs &args) : a(args), lane(threadIdx.x & 63), i(lane & 31), h(lane >> 5) {}

    // The two pages of a tile: numbers (kNoPlace if there is none) and offsets.
    struct Pages {
        int id[2], off[2];
    };
    __device__ __forceinline__ Pages pages(int key0) const {
        Pages p;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int key = key0 + 16 * s;
            const Place at = key < len ? place_at(a.c, a.n, b, key) : Place{kNoPlace, 0};
            p.id[s] = at.page;
            p.off[s] = at.off;
        }
        return p;
    }

    // Loads of a tile.  A part without a page reads page 0 and counts as no key; nothing past a row's dim is
    // read, and the rows of a part past the sequence's end are the page's own.
    __device__ __forceinline__ void load(Tile<DB> &t, const Pages &p, int key0) const {
        const int dim = a.c.dim;
        int valid[2];
        int64_t row[2];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int id = __builtin_amdgcn_readfirstlane(p.id[s]);
            valid[s] = id >= 0 ? min(16, len - key0 - 16 * s) : 0;
            row[s] = max(id, 0);
        }
        t.valid = valid[0] | valid[1] << 16;
        const int at[2] = {head * a.c.page + p.off[0], head * a.c.page + p.off[1]};
        const int64_t byte[2] = {row[0] * a.c.stride + int64_t(at[0]) * dim, row[1] * a.c.stride + int64_t(at[1]) * dim};
        const bool up = i & 16;
        const uint8_t *kp = a.c.k + (up ? byte[1] : byte[0]) + koff;
#pragma unroll
        for (int c = 0; c < DB; ++c) {
            t.k[c] = intx4{};
            if (32 * c + 16 * h < dim) t.k[c] = *reinterpret_cast<const intx4 *>(kp + 32 * c);
        }
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint8_t *vp = a.c.v + byte[s] + (e < 4 ? e : e + 4) * dim;
                if constexpr (DB == 2) t.v[s][e][0] = DB * i < dim ? *reinterpret_cast<const uint16_t *>(vp + voff) : 0;
                else if constexpr (DB == 4) t.v[s][e][0] = DB * i < dim ? *reinterpret_cast<const unsigned *>(vp + voff) : 0;
                else {
                    intx2 w = {};
                    if (DB * i < dim) w = *reinterpret_cast<const intx2 *>(vp + voff);
                    t.v[s][e][0] = w[0];
                    t.v[s][e][1] = w[1];
                }
            }
        const int64_t se = (up ? row[1] : row[0]) * a.c.sstride + (up ? at[1] : at[0]) + (i & 15);
        const void *sp = h ? a.c.vs : a.c.ks;
        t.s = a.c.stype == DS_SCALE_POW2 ? static_cast<const uint8_t *>(sp)[se] : static_cast<const unsigned *>(sp)[se];
    }

    // The operand of block blk and keys of step s: row i of it is value DB i + blk.
    __device__ __forceinline__ bf16x8 decode_v(const Tile<DB> &t, int s, int blk) const {
        const int w = blk >> 2, j = blk & 3;
        bf16x8 r;
        int pair[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            pair[e] = int(__builtin_amdgcn_perm(t.v[s][2 * e + 1][w], t.v[s][2 * e][w], j & 2 ? 0x07030602u : 0x05010400u));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            bf16x2 x;
            if constexpr (FMT == DS_Q8_E4M3)
                x = j & 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(pair[e], 1.f, true)
                          : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(pair[e], 1.f, false);
            else
                x = j & 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(pair[e], 1.f, true)
                          : __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(pair[e], 1.f, false);
            r[2 * e] = x[0];
            r[2 * e + 1] = x[1];
        }
        return r;
    }

    // Key of register r in the tile: the order in which both products take keys.
    __device__ __forceinline__ int key_of(int r) const { return 8 * (r >> 2) + 4 * h + (r & 3); }

    // One tile; edge: some row does not see some key of it, or some key does not exist.  POISON: see poisoned();
    // without it, false where that is needed.
    template <bool POISON>
    __device__ __forceinline__ bool step(Tile<DB> &t, int key0, bool edge, float *lds) {
        // the scales of all 32 keys to every lane that needs them; 0 of keys that do not exist
        const int valid[2] = {t.valid & 0xffff, t.valid >> 16};
        float sc = a.c.stype == DS_SCALE_POW2 ? __uint_as_float(max(t.s << 23, 0x400000u)) : __uint_as_float(t.s);
        if (edge) sc = (i & 15) < (i & 16 ? valid[1] : valid[0]) ? sc : 0.f;
        lds[lane] = h ? sc : sc * a.scale;
        __builtin_amdgcn_wave_barrier();
        floatx16 s[NQ] = {};
#pragma unroll
        for (int c = 0; c < DB; ++c)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const Op k = decode_k<FMT, Op>(t.k[c][2 * u], t.k[c][2 * u + 1]);
#pragma unroll
                for (int p = P::QP - 1; p >= 0; --p)
#pragma unroll
                    for (int n = 0; n < NQ; ++n) s[n] = mma(k, q[p][n][2 * c + u], s[n]);
            }
        __builtin_amdgcn_sched_barrier(0);
        bf16x8 pt[NQ][P::PP][2], seen[NQ][2];
        unsigned bad = 0;
        if (POISON || edge) {
#pragma unroll
            for (int st = 0; st < 2; ++st)
#pragma unroll
                for (int e = 0; e < 8; ++e)
#pragma unroll
                    for (int w = 0; w < Tile<DB>::W; ++w) {
                        unsigned &x = t.v[st][e][w];
                        if (4 * h + (e < 4 ? e : e + 4) >= valid[st]) x = 0;
                        bad |= not_finite<FMT>(x);
                    }
            if (!POISON && __any(bad != 0)) return false;
        }
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            float x[16];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const floatx4 sk = *reinterpret_cast<const floatx4 *>(lds + 8 * j + 4 * h);
#pragma unroll
                for (int e = 0; e < 4; ++e) x[4 * j + e] = s[n][4 * j + e] * sk[e];
            }
            if (POISON || edge)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int k = key_of(r);
                    const bool sees = key0 + k >= low[n] && key0 + k < lim[n] && (k & 15) < valid[r >> 3];
                    x[r] = sees ? x[r] : -INFINITY;
                    if constexpr (POISON) seen[n][r >> 3][r & 7] = __bf16(sees ? 1.f : 0.f);
                }
            float top = fmaxf(x[0], x[1]);
#pragma unroll
            for (int r = 2; r < 16; r += 2) top = fmaxf(fmaxf(top, x[r]), x[r + 1]);
            top = fmaxf(top, other_half(top));
            // the running maximum follows only by steps of 2^8 or more: any number near it serves, as weights
            // of up to 2^8 lose nothing in fp32 or bf16
            if (__any(top > m[n] + 8.f || (m[n] == -INFINITY && top > -INFINITY))) {
                const float now = fmaxf(m[n], top);
                const float by = now == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[n] - now);
                m[n] = now;
                l[n] *= by;
#pragma unroll
                for (int blk = 0; blk < DB; ++blk)
#pragma unroll
                    for (int r = 0; r < 16; ++r) o[n][blk][r] *= by;
            }
            const float off = m[n] == -INFINITY ? 0.f : m[n];
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                x[r] = __builtin_amdgcn_exp2f(x[r] - off);
                l[n] += x[r];
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const floatx4 sv = *reinterpret_cast<const floatx4 *>(lds + 32 + 8 * j + 4 * h);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float w = x[4 * j + e] * sv[e];
#pragma unroll
                    for (int part = 0; part < P::PP; ++part) {
                        const __bf16 top8 = __bf16(w);
                        pt[n][part][j >> 1][4 * (j & 1) + e] = top8;
                        w -= float(top8);
                    }
                }
            }
        }
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (POISON) {
            poisoned(t, pt, seen);
            return true;
        }
#pragma unroll
        for (int blk = 0; blk < DB; ++blk)
#pragma unroll
            for (int st = 0; st < 2; ++st) {
                const bf16x8 v = decode_v(t, st, blk);
#pragma unroll
                for (int part = P::PP - 1; part >= 0; --part)
#pragma unroll
                    for (int n = 0; n < NQ; ++n) o[n][blk] = mma(v, pt[n][part][st], o[n][blk]);
            }
        return true;
    }

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            m[n] = -INFINITY;
            l[n] = 0.f;
#pragma unroll
            for (int blk = 0; blk < DB; ++blk) o[n][blk] = floatx16{};
        }
    }

    // The second product where V holds infinities or NaNs and some row does not see all keys: 0 times those
    // is no 0. They are taken out of V, and a second product counts for each row and value how many
    // that it sees are +infinity (units of 1), -infinity (64) and NaN (4096): sums of up to 32, exact.
    __device__ __forceinline__ void poisoned(const Tile<DB> &t, const bf16x8 (&pt)[NQ][P::PP][2],
                                             const bf16x8 (&seen)[NQ][2]) {
#pragma unroll
        for (int blk = 0; blk < DB; ++blk) {
            floatx16 count[NQ] = {};
#pragma unroll
            for (int st = 0; st < 2; ++st) {
                bf16x8 v = decode_v(t, st, blk), kind;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float f = v[e];
                    const bool fine = fabsf(f) < INFINITY;
                    v[e] = __bf16(fine ? f : 0.f);
                    kind[e] = __bf16(fine ? 0.f : f > 0.f ? 1.f : f < 0.f ? 64.f : 4096.f);
                }
#pragma unroll
                for (int n = 0; n < NQ; ++n) {
#pragma unroll
                    for (int part = P::PP - 1; part >= 0; --part) o[n][blk] = mma(v, pt[n][part][st], o[n][blk]);
                    count[n] = mma(kind, seen[n][st], count[n]);
                }
            }
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float c = count[n][r];
                    const bool nan = c >= 4096.f, minus = c >= 64.f, plus = c - (minus ? 64.f * floorf(c / 64.f) : 0.f) > 0.f;
                    if (nan || (minus && plus)) o[n][blk][r] = NAN;
                    else if (c > 0.f) o[n][blk][r] += minus ? -INFINITY : INFINITY;
                }
        }
    }
};

// Sequence of a tile of rows: the tiles of sequence b begin at starts[b] * group / rows + b, which leaves each at
// least as many as it needs, without a sum over the sequences before it.
__device__ __forceinline__ int64_t first_tile(const AttnArgs &a, int b, int rows) {
    const int s = min(max(a.n.starts[b], 0), a.n.tokens);
    return int64_t(s) * a.group / rows + b;
}

template <typename T, int FMT, int DB, int NQ, bool SHARE>
__device__ __forceinline__ void attn8_body(const AttnArgs &a, float *scales, float *join) {
    using A = Attn<T, FMT, DB, NQ, SHARE>;
    using P = typename A::P;
    A w(a);
    const int lane = w.lane, i = w.i, h = w.h;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int kv = a.c.heads;
    // heads side by side: workgroups go to the chip's eight parts in turn, so the workgroups of a head
    // share the caches of as few parts as the number of heads allows
    int idx = blockIdx.x;
    w.head = idx % kv;
    idx /= kv;
    const int split = idx % a.splits;
    const int tile = idx / a.splits;

    int b = 0;
    for (int n = a.n.seqs; n > 1;) {       // 64 sequences a step
        const int by = (n + 63) / 64;
        const bool ok = lane == 0 || (lane * by < n && first_tile(a, b + lane * by, A::kTileRows) <= tile);
        const int k = 63 - __clzll(__ballot(ok));
        b += k * by;
        n = min(by, n - k * by);
    }
    b = __builtin_amdgcn_readfirstlane(b);
    w.b = b;
    const int s0 = min(max(a.n.starts[b], 0), a.n.tokens), s1 = min(max(a.n.starts[b + 1], s0), a.n.tokens);
    const int64_t rows = int64_t(s1 - s0) * a.group;
    const int64_t mine = tile - first_tile(a, b, A::kTileRows);
    if (mine < 0 || mine * A::kTileRows >= rows) return;
    // the last rows, which see most keys, first
    const int64_t all = (rows + A::kTileRows - 1) / A::kTileRows;
    const int64_t row0 = (a.causal ? all - 1 - mine : mine) * A::kTileRows + (SHARE ? 0 : wave * A::kRows);
    const int length = a.n.lengths[b];
    w.len = min(max(length, 0), a.len);
    // row r is token s0 + r / group at position length - (s1 - s0) + r / group
    const int64_t shift = int64_t(length) - (s1 - s0);
    const auto token = [&](int64_t r) { return int(min(r, rows - 1) / a.group); };
    const auto limit = [&](int t) { return a.causal ? int(min(max(shift + t + 1, int64_t(0)), int64_t(w.len))) : w.len; };
    const auto lowest = [&](int t) { return a.window > 0 ? int(max(min(shift + t + 1 - a.window, int64_t(w.len)), int64_t(0))) : 0; };

    int tok[NQ], hd[NQ];
    bool is[NQ];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        const int64_t r = row0 + 32 * n + i;
        is[n] = r < rows;
        const int t = token(r);
        tok[n] = s0 + t;
        hd[n] = w.head * a.group + int(min(r, rows - 1) - int64_t(t) * a.group);
        w.lim[n] = limit(t);
        w.low[n] = lowest(t);
        const T *qp = static_cast<const T *>(a.q) + tok[n] * a.ldq + hd[n] * a.hldq;
#pragma unroll
        for (int c = 0; c < 2 * DB; ++c) {
            const int d = 32 * (c >> 1) + 16 * h + 8 * (c & 1);
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
            if constexpr (P::QP == 1) {
#pragma unroll
                for (int e = 0; e < 8; ++e) w.q[0][n][c][e] = x[e];
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float rest = x[e];
#pragma unroll
                    for (int p = 0; p < P::QP; ++p) {
                        w.q[p][n][c][e] = __bf16(rest);
                        rest -= float(w.q[p][n][c][e]);
                    }
                }
            }
        }
    }
    w.koff = (i & 15) * a.c.dim + 16 * h;
    w.voff = 4 * h * a.c.dim + DB * i;

    // the wave's keys: those that its rows see, from the tile's first
    const int64_t first = SHARE ? row0 : row0 - wave * A::kRows;
    const int base = lowest(token(first)) & ~(kKeys - 1);
    const int from = max(lowest(token(row0)) & ~(kKeys - 1), int(min(int64_t(base) + int64_t(split) * a.span, kMaxPlaces)) & ~(kKeys - 1));
    const int until = int(min(int64_t(row0 < rows ? limit(token(row0 + A::kRows - 1)) : 0),
                              int64_t(base) + int64_t(split + 1) * a.span));
    // keys that all its rows see
    const int every = limit(token(row0)), since = lowest(token(row0 + A::kRows - 1));
    constexpr int kStep = SHARE ? kWaves * kKeys : kKeys;
    const int begin = from + (SHARE ? wave * kKeys : 0);
    float *lds = scales + wave * 64;
    w.clear();
    bool fine = true;
    const auto edge = [&](int key, const Tile<DB> &t) {
        return key + kKeys > every || key < since || t.valid != (16 | 16 << 16);
    };
    if constexpr (DB == 8) {
        // (the registers hold one tile of 256 values a row)
        for (int key = begin; key < until && fine; key += kStep) {
            Tile<DB> t;
            w.load(t, w.pages(key), key);
            fine = w.template step<false>(t, key, edge(key, t), lds);
        }
    } else if (begin < until) {
        int key = begin;
        Tile<DB> t[2];
        w.load(t[0], w.pages(key), key);
        typename A::Pages next = w.pages(key + kStep);
        const auto one = [&](Tile<DB> &now, Tile<DB> &then) {
            const typename A::Pages after = w.pages(key + 2 * kStep);
            if (key + kStep < until) w.load(then, next, key + kStep);
            next = after;
            fine = w.template step<false>(now, key, edge(key, now), lds);
            key += kStep;
        };
        while (true) {
            one(t[0], t[1]);
            if (key >= until || !fine) break;
            one(t[1], t[0]);
            if (key >= until || !fine) break;
        }
    }
    if (!fine) {
        w.clear();
#pragma unroll 1
        for (int key = begin; key < until; key += kStep) {
            Tile<DB> t;
            w.load(t, w.pages(key), key);
            w.template step<true>(t, key, true, lds);
        }
    }
#pragma unroll
    for (int n = 0; n < NQ; ++n) w.l[n] += other_half(w.l[n]);

    if constexpr (SHARE) {
        // four waves' sums of the same rows: two halves of the waves, then two waves
#pragma unroll
        for (int half = kWaves / 2; half > 0; half /= 2) {
            constexpr int kSlot = 64 + 64 * 16 * DB;
            __syncthreads();
            if (wave >= half && wave < 2 * half) {
                float *to = join + (wave - half) * kSlot;
                if (h == 0) {
                    to[i] = w.m[0];
                    to[32 + i] = w.l[0];
                }
#pragma unroll
                for (int blk = 0; blk < DB; ++blk)
#pragma unroll
                    for (int r = 0; r < 16; ++r) to[64 + (blk * 16 + r) * 64 + lane] = w.o[0][blk][r];
            }
            __syncthreads();
            if (wave < half) {
                const float *of = join + wave * kSlot;
                const float om = of[i], ol = of[32 + i], now = fmaxf(w.m[0], om);
                const float by = w.m[0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(w.m[0] - now);
                const float bo = om == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(om - now);
                w.m[0] = now;
                w.l[0] = w.l[0] * by + ol * bo;
#pragma unroll
                for (int blk = 0; blk < DB; ++blk)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        w.o[0][blk][r] = w.o[0][blk][r] * by + of[64 + (blk * 16 + r) * 64 + lane] * bo;
            }
        }
        if (wave != 0) return;
    }

    // register r of block blk is value DB * row + blk, row = 8 (r / 4) + 4 h + r % 4
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        if (!is[n]) continue;
        const int64_t at = int64_t(tok[n]) * a.heads + hd[n];
        if (a.splits > 1) {
            const int64_t p = int64_t(split) * a.n.tokens * a.heads + at;
            if (h == 0) a.ml[p] = make_float2(w.m[n], w.l[n]);
            if (w.l[n] == 0.f) continue;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int d = DB * (8 * (r >> 2) + 4 * h + (r & 3));
                if (d < a.c.dim)
#pragma unroll
                    for (int blk = 0; blk < DB; ++blk) a.part[p * a.c.dim + d + blk] = w.o[n][blk][r];
            }
            continue;
        }
        const float by = w.l[n] == 0.f ? 0.f : 1.f / w.l[n];
        if (a.lse && h == 0) a.lse[at] = w.l[n] == 0.f ? -INFINITY : (w.m[n] + log2f(w.l[n])) * kLn2;
        T *op = static_cast<T *>(a.out) + tok[n] * a.ldo + hd[n] * a.hldo;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int d = DB * (8 * (r >> 2) + 4 * h + (r & 3));
            if (d < a.c.dim)
#pragma unroll
                for (int blk = 0; blk < DB; ++blk) op[d + blk] = T(w.l[n] == 0.f ? 0.f : w.o[n][blk][r] * by);
        }
    }
}

// Waves of a SIMD unit: two where their registers allow it.
template <typename T, int DB>
constexpr int waves_of = DB <= 4 && !std::is_same_v<T, float> ? 2 : 1;

// Waves that share rows take tiles of keys in turn.
template <typename T, int FMT, int DB>
__global__ __launch_bounds__(256, (waves_of<T, DB>)) void attn8_few(AttnArgs a) {
    __shared__ __attribute__((aligned(16))) float scales[kWaves * 64];
    __shared__ float join[2 * (64 + 64 * 16 * DB)];
    attn8_body<T, FMT, DB, 1, true>(a, scales, join);
}
// Each wave has rows of its own.
template <typename T, int FMT, int DB, int NQ>
__global__ __launch_bounds__(256, (waves_of<T, DB>)) void attn8_many(AttnArgs a) {
    __shared__ __attribute__((aligned(16))) float scales[kWaves * 64];
    attn8_body<T, FMT, DB, NQ, false>(a, scales, nullptr);
}


}  // namespace

template <typename T>
const void *attn8_kernel(int fmt, int dim, bool few) {
    constexpr int NQ = attn8_blocks(std::is_same_v<T, float>, 4);
    constexpr int N8 = attn8_blocks(std::is_same_v<T, float>, 8);
    const int db = attn8_dim_blocks(dim);
    constexpr bool kWide = !std::is_same_v<T, float>;        // more than 128 values a row
#define DS_ATTN8(FMT)                                                                                       \
    if (fmt == FMT && db == 2)                                                                              \
        return few ? reinterpret_cast<const void *>(&attn8_few<T, FMT, 2>)                                  \
                   : reinterpret_cast<const void *>(&attn8_many<T, FMT, 2, NQ>);                            \
    if (fmt == FMT && db == 4)                                                                              \
        return few ? reinterpret_cast<const void *>(&attn8_few<T, FMT, 4>)                                  \
                   : reinterpret_cast<const void *>(&attn8_many<T, FMT, 4, NQ>);                            \
    if constexpr (kWide)                                                                                    \
        if (fmt == FMT && db == 8)                                                                          \
            return few ? reinterpret_cast<const void *>(&attn8_few<T, FMT, 8>)                              \
                       : reinterpret_cast<const void *>(&attn8_many<T, FMT, 8, N8>);
    DS_ATTN8(DS_Q8_E4M3)
    DS_ATTN8(DS_Q8_E5M2)
#undef DS_ATTN8
    return nullptr;
}

}  // namespace ds
