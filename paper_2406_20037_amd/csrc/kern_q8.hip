// Quantization to 8 bits in blocks of 128, and the gated unit with its activations kept
// in 8 bits.  Both move memory and little else: every input is read once and every
// output, transposes too, written once by the same launch.
#include <type_traits>

#include "q8.h"

namespace ds {

int q8_check(const ds_q8 *m, const char *what) {
    if (!m) {
        set_error("%s: null 8-bit matrix", what);
        return DS_EINVAL;
    }
    // (room for a tile past the last row in 32 bits)
    if (m->rows < 0 || m->cols < 0 || m->rows > 0x7ffffe00 || m->cols > 0x7ffffe00) {
        set_error("%s: %lld x %lld values", what, (long long)m->rows, (long long)m->cols);
        return DS_EINVAL;
    }
    if ((m->format != DS_Q8_E4M3 && m->format != DS_Q8_E5M2) ||
        (m->scale_type != DS_SCALE_POW2 && m->scale_type != DS_SCALE_F32) ||
        (m->block_rows != 1 && m->block_rows != kQ8Block) || m->reserved != 0) {
        set_error("%s: format %d, scale type %d, block_rows %d, reserved %d", what, m->format,
                  m->scale_type, m->block_rows, m->reserved);
        return DS_EINVAL;
    }
    if (m->ld < m->cols || m->ld % 16 != 0 || m->ld >= (1 << 24) ||
        m->scale_ld < q8_up(m->cols) || m->scale_ld >= (1 << 22)) {
        set_error("%s: ld %lld of %lld columns (a multiple of 16 below 2^24), scale_ld %lld (below 2^22)", what,
                  (long long)m->ld, (long long)m->cols, (long long)m->scale_ld);
        return DS_EINVAL;
    }
    if (m->rows > 0 && m->cols > 0 &&
        (!m->data || !m->scale || reinterpret_cast<uintptr_t>(m->data) % 16 != 0 ||
         (m->scale_type == DS_SCALE_F32 && reinterpret_cast<uintptr_t>(m->scale) % 4 != 0))) {
        set_error("%s: null or misaligned buffer", what);
        return DS_EINVAL;
    }
    return DS_OK;
}

int launch_check(int64_t groups, int threads, const char *what) {
    if (groups > int64_t(0xffffffffu) / threads) {
        set_error("%s: %lld workgroups of %d threads are more than a launch takes", what, (long long)groups, threads);
        return DS_EUNSUPPORTED;
    }
    return DS_OK;
}

int plain_check(const void *p, int type, int64_t rows, int64_t cols, int64_t ld, const char *what) {
    if (type != DS_TYPE_F32 && type != DS_TYPE_F16 && type != DS_TYPE_BF16) {
        set_error("%s: type %d", what, type);
        return DS_EINVAL;
    }
    if (rows < 0 || cols < 0 || rows > 0x7fffffff || cols > 0x7fffffff || ld < cols) {
        set_error("%s: %lld x %lld, ld %lld", what, (long long)rows, (long long)cols, (long long)ld);
        return DS_EINVAL;
    }
    if (rows > 0 && cols > 0 && (!p || reinterpret_cast<uintptr_t>(p) % type_bytes(type) != 0)) {
        set_error("%s: null or misaligned buffer", what);
        return DS_EINVAL;
    }
    return DS_OK;
}

namespace {

// FULL, here and below: the caller has seen that all rows and columns of a tile exist.

// Eight elements of a row of `cols`, 0 past its end; vec: rows are 16-byte aligned.
template <typename T>
struct Eight {
    T t[8];
    // as loaded: a use after this is not one of values the compiler has already
    __device__ __forceinline__ void forget() {
        intx4 *p = reinterpret_cast<intx4 *>(t);
#pragma unroll
        for (size_t i = 0; i < sizeof(t) / 16; ++i) {
            intx4 w = p[i];
            __asm__ volatile("" : "+v"(w));
            p[i] = w;
        }
    }
};
template <bool FULL, typename T>
__device__ __forceinline__ Eight<T> raw8(const T *row, int c, int cols, bool vec) {
    Eight<T> e;
    if (vec && (FULL || c + 8 <= cols)) {
#pragma unroll
        for (size_t i = 0; i < sizeof(e) / 16; ++i)
            reinterpret_cast<intx4 *>(e.t)[i] = reinterpret_cast<const intx4 *>(row + c)[i];
    } else if (FULL || c + 8 <= cols) {
#pragma unroll
        for (int i = 0; i < 8; ++i) e.t[i] = row[c + i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) e.t[i] = c + i < cols ? row[c + i] : T(0.f);
    }
    return e;
}
template <bool FULL, typename T>
__device__ __forceinline__ void load8(const T *row, int c, int cols, bool vec, float (&v)[8]) {
    const Eight<T> e = raw8<FULL>(row, c, cols, vec);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = float(e.t[i]);
}

// The bits of the largest magnitude, kInf or more where some value is not finite: the largest as
// signed numbers is the largest positive one, as unsigned the most negative one if there is any
// (one instruction for two values each, where taking signs off first would cost one a value).
// SUMS: results of arithmetic, which have no signalling NaNs; of those a floating-point maximum passes
// over the NaNs and takes two values an instruction.
constexpr unsigned kInf = 0x7f800000u;
template <bool SUMS, int N>
__device__ __forceinline__ unsigned max_bits(const float (&v)[N]) {
    if constexpr (SUMS) {
        float m = fmaxf(fabsf(v[0]), fabsf(v[1]));
#pragma unroll
        for (int i = 2; i < N; i += 2) m = fmaxf(fmaxf(m, fabsf(v[i])), fabsf(v[i + 1]));
        return __float_as_uint(m);
    }
    int pos = 0;
    unsigned neg = 0;
#pragma unroll
    for (int i = 0; i < N; i += 2) {
        pos = max(max(pos, __float_as_int(v[i])), __float_as_int(v[i + 1]));
        neg = max(max(neg, __float_as_uint(v[i])), __float_as_uint(v[i + 1]));
    }
    return max(unsigned(pos), neg & 0x7fffffffu);
}
// The same of the finite ones.
template <int N>
__device__ __forceinline__ unsigned max_finite(const float (&v)[N]) {
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float x = v[i];
        __asm__("" : "+v"(x), "+v"(m));                    // one by one, in few registers
        m = max(m, finite_abs(x));
    }
    return m;
}

// Eight bytes to columns c .. of a row that ends at `cols`.
template <bool FULL>
__device__ __forceinline__ void store8(uint8_t *row, int c, int cols, intx2 q) {
    if (FULL || c + 8 <= cols) {
        *reinterpret_cast<intx2 *>(row + c) = q;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i < cols) row[c + i] = uint8_t(unsigned(q[i >> 2]) >> (8 * (i & 3)));
    }
}

template <int FMT, bool FULL>
__device__ __forceinline__ void store_values(uint8_t *row, int c, int cols, const float (&v)[8], float inv) {
    store8<FULL>(row, c, cols, intx2{pack4<FMT>(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv),
                                     pack4<FMT>(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv)});
}

// One 1x128 block of row r at columns c0 .. c0+127, held by 16 lanes of eight values each.
template <int FMT, bool FULL, bool SUMS>
__device__ __forceinline__ void emit_block(const Q8View &m, int r, int blk, int cl, const float (&v)[8]) {
    unsigned top = max_bits<SUMS>(v);
    // what is not finite sets no scale: only a wave that holds some looks at each value
    if (__any(top >= kInf)) top = max_finite(v);
    const BlockScale s = block_scale(max16(top), FMT, m.stype);
    store_values<FMT, FULL>(m.data + int64_t(r) * m.ld, blk * kQ8Block + 8 * cl, m.cols, v, s.inv);
    if (cl == 0) store_scale(m, int64_t(r) * m.sld + blk, s.bits);
}

// Calls fn with the format as a constant.
template <typename Fn>
__device__ __forceinline__ void by_fmt(int fmt, Fn fn) {
    if (fmt == DS_Q8_E4M3) fn(std::integral_constant<int, DS_Q8_E4M3>{});
    else fn(std::integral_constant<int, DS_Q8_E5M2>{});
}

// Rows alone, or one plain matrix read once and written in a half to a quarter of its bytes: bound by
// the memory.  16 lanes a block, so that the largest magnitude meets in one row of lanes, without LDS,
// and a wave's loads cover whole lines: 16384x8192 bf16 in 74 us (5.4 TB/s, of which the caches
// serve a part); of rows that are not 16-byte aligned 89.
template <typename T>
__global__ __launch_bounds__(256) void q8_rows(const T *x, int64_t ldx, int vec, Q8View m, int nb,
                                               int64_t total) {
    const int cl = threadIdx.x & 15;
    const int64_t step = int64_t(gridDim.x) * 16;
    for (int64_t i = int64_t(blockIdx.x) * 16 + (threadIdx.x >> 4); i < total; i += step) {
        const int r = int(i / nb), b = int(i - int64_t(r) * nb);
        float v[8];
        load8<false>(x + int64_t(r) * ldx, b * kQ8Block + 8 * cl, m.cols, vec, v);
        by_fmt(m.fmt, [&](auto f) { emit_block<f.value, false, false>(m, r, b, cl, v); });
    }
}

// ---- tiles of 128 x 128 -----------------------------------------------------------
// Both directions from one read: bound by the memory, if enough of it is on its way.  A tile stays in
// registers while its rows' and its columns' largest magnitudes are found (rows by lanes, columns
// by lanes, then over the waves through LDS), and its transpose goes through LDS as bytes, so that it
// is written in whole lines too.  16384x8192 bf16 both ways in 115 us (4.7 TB/s), fp32 151 us (5.3), and in
// squares 152; 16384x8191 bf16, whose rows load element by element, 147.
// 512 threads; thread t holds rows 4 (t / 16) .. + 3 of columns 8 (t % 16) .. + 7.
constexpr int kTileThreads = 512, kRows = 4, kTileWaves = kTileThreads / 64;

struct TileLds {
    unsigned colmax[kTileWaves][128];
    float inv[128];
    // transposed bytes: column c's 16 rows of wave w are the 16 bytes at c * 8 + (w ^ c / 8 % 8), so
    // that the 16 columns a wave writes at once lie in different banks
    intx4 t[128 * 8];
};

// Largest over the wave's four rows of lanes of eight columns: row of lanes q keeps columns 2 q and
// 2 q + 1.  Each swap brings two columns' values together at once.
__device__ __forceinline__ void over_rows(unsigned (&m)[8]) {
    typedef unsigned uintx2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int c = 0; c < 4; ++c) {                          // lower lanes c, upper lanes c + 4
        const uintx2 a = __builtin_amdgcn_permlane32_swap(m[c], m[c + 4], false, false);
        m[c] = max(a[0], a[1]);
    }
#pragma unroll
    for (int c = 0; c < 2; ++c) {                          // rows of lanes c, c + 2, c + 4, c + 6
        const uintx2 a = __builtin_amdgcn_permlane16_swap(m[c], m[c + 2], false, false);
        m[c] = max(a[0], a[1]);
    }
}

// One tile and where it goes: to `row` at (r0, c0) and transposed to `col` at (rc0, r0); either has
// data == null when not wanted.
struct TileOut {
    Q8View row, col;
    int c0, rc0;
};

template <int CTRL>
__device__ __forceinline__ unsigned dpp(unsigned v) {
    return unsigned(__builtin_amdgcn_update_dpp(0, int(v), CTRL, 0xF, 0xF, false));
}

// The thread's four rows: lane l of 16 gathers the largest magnitude of row l % 4, so that one scale a
// lane is formed and stored, and each group of four lanes has all four.
template <bool FULL, bool SUMS>
__device__ __forceinline__ void emit_rows(const float (&v)[kRows][8], const TileOut &o, int r0) {
    const int cl = threadIdx.x & 15, rg = threadIdx.x >> 4;
    unsigned m[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) m[r] = max_bits<SUMS>(v[r]);
    if (__any(max(max(m[0], m[1]), max(m[2], m[3])) >= kInf))
#pragma unroll
        for (int r = 0; r < kRows; ++r) m[r] = max_finite(v[r]);
    const bool odd = cl & 1, high = cl & 2;
    const unsigned a = max(odd ? m[1] : m[0], dpp<0xB1>(odd ? m[0] : m[1]));   // with lane ^ 1
    const unsigned b = max(odd ? m[3] : m[2], dpp<0xB1>(odd ? m[2] : m[3]));
    unsigned top = max(high ? b : a, dpp<0x4E>(high ? a : b));                 // with lane ^ 2
    top = max(top, dpp<0x124>(top));                                           // lanes turned by 4, by 8
    top = max(top, dpp<0x128>(top));
    const BlockScale s = block_scale(top, o.row.fmt, o.row.stype);
    const int rr = r0 + kRows * rg;
    if (cl < kRows && (FULL || rr + cl < o.row.rows))
        store_scale(o.row, int64_t(rr + cl) * o.row.sld + (o.c0 >> 7), s.bits);
    const unsigned inv = __float_as_uint(s.inv);
    const float by[kRows] = {__uint_as_float(dpp<0x00>(inv)), __uint_as_float(dpp<0x55>(inv)),
                             __uint_as_float(dpp<0xAA>(inv)), __uint_as_float(dpp<0xFF>(inv))};
#pragma unroll
    for (int r = 0; r < kRows; ++r)
        if (FULL || rr + r < o.row.rows)
            by_fmt(o.row.fmt, [&](auto f) {                // row by row: scaled values of one at a time
                store_values<f.value, FULL>(o.row.data + int64_t(rr + r) * o.row.ld, o.c0 + 8 * cl, o.row.cols, v[r],
                                            by[r]);
            });
}

// The thread's largest magnitudes of its eight columns, then the wave's to `lds`.
template <bool SUMS>
__device__ __forceinline__ void column_max(const float (&v)[kRows][8], unsigned (*lds)[128]) {
    const int tid = threadIdx.x;
    unsigned m[8], any = 0;
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        const float u[kRows] = {v[0][c], v[1][c], v[2][c], v[3][c]};
        m[c] = max_bits<SUMS>(u);
        any = max(any, m[c]);
    }
    if (__any(any >= kInf))
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            const float u[kRows] = {v[0][c], v[1][c], v[2][c], v[3][c]};
            m[c] = max_finite(u);
        }
    over_rows(m);
    *reinterpret_cast<intx2 *>(lds[tid >> 6] + 8 * (tid & 15) + 2 * (tid >> 4 & 3)) = intx2{int(m[0]), int(m[1])};
}

// The columns' scales, once the waves' column_max are in.
__device__ __forceinline__ void column_scales(const TileOut &o, int r0, TileLds &lds) {
    const int c = threadIdx.x;
    if (c >= 128) return;
    unsigned top = 0;
#pragma unroll
    for (int i = 0; i < kTileWaves; ++i) top = max(top, lds.colmax[i][c]);
    const BlockScale s = block_scale(top, o.col.fmt, o.col.stype);
    lds.inv[c] = s.inv;
    if (o.rc0 + c < o.col.rows) store_scale(o.col, int64_t(o.rc0 + c) * o.col.sld + (r0 >> 7), s.bits);
}

// The tile's columns times inv, as bytes to `t`; inv the same for all where `one` is not 0.
__device__ __forceinline__ void transpose_in(const float (&v)[kRows][8], const float *inv, float one, int fmt,
                                             intx4 *t) {
    const int cl = threadIdx.x & 15, rg = threadIdx.x >> 4, w = threadIdx.x >> 6;
    by_fmt(fmt, [&](auto f) {
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            const int cc = 8 * cl + c;
            const float s = one != 0.f ? one : inv[cc];
            reinterpret_cast<int *>(t)[(cc * 8 + (w ^ (cl & 7))) * 4 + (rg & 3)] =
                pack4<f.value>(v[0][c] * s, v[1][c] * s, v[2][c] * s, v[3][c] * s);
        }
    });
}

template <bool FULL>
__device__ __forceinline__ void transpose_out(const TileOut &o, int r0, const intx4 *t) {
#pragma unroll
    for (int j = 0; j < 1024 / kTileThreads; ++j) {
        const int i = j * kTileThreads + threadIdx.x, c = i >> 3, g = i & 7, at = r0 + 16 * g;
        if (!FULL && (o.rc0 + c >= o.col.rows || at >= o.col.cols)) continue;
        uint8_t *p = o.col.data + int64_t(o.rc0 + c) * o.col.ld;
        const intx4 q = t[c * 8 + (g ^ (c >> 3 & 7))];
        if (FULL || at + 16 <= o.col.cols) {
            *reinterpret_cast<intx4 *>(p + at) = q;
        } else {
            store8<false>(p, at, o.col.cols, intx2{q[0], q[1]});
            store8<false>(p, at + 8, o.col.cols, intx2{q[2], q[3]});
        }
    }
}

// Column by column: a tile's transpose.  The LDS is free again after a barrier that follows.
template <bool FULL, bool SUMS>
__device__ __forceinline__ void emit_columns(const float (&v)[kRows][8], const TileOut &o, int r0, TileLds &lds) {
    column_max<SUMS>(v, lds.colmax);
    __syncthreads();
    column_scales(o, r0, lds);
    __syncthreads();
    transpose_in(v, lds.inv, 0.f, o.col.fmt, lds.t);
    __syncthreads();
    transpose_out<FULL>(o, r0, lds.t);
}

template <bool FULL, typename T>
__device__ __forceinline__ void tile_body(const T *x, int64_t ldx, int vec, int rows, int cols, int tr, int tc,
                                          const Q8View &row, const Q8View &col, TileLds &lds) {
    const int cl = threadIdx.x & 15, rg = threadIdx.x >> 4;
    const int r0 = tr * 128, c0 = tc * 128;
    const TileOut o = {row, col, c0, c0};
    float v[kRows][8];
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        const int rr = r0 + kRows * rg + r;
        if (FULL || rr < rows) {
            load8<FULL>(x + int64_t(rr) * ldx, c0 + 8 * cl, cols, vec, v[r]);
        } else {
#pragma unroll
            for (int c = 0; c < 8; ++c) v[r][c] = 0.f;
        }
    }
    if (!(row.data ? row.shift : col.shift)) {
        if (row.data) emit_rows<FULL, false>(v, o, r0);
        if (!col.data) return;
        emit_columns<FULL, false>(v, o, r0, lds);
        return;
    }
    // one scale for the square
    column_max<false>(v, lds.colmax);
    __syncthreads();
    unsigned all = 0;
#pragma unroll
    for (int c = 0; c < 8; ++c)
#pragma unroll
        for (int i = 0; i < kTileWaves; ++i) all = max(all, lds.colmax[i][8 * cl + c]);
    all = max16(all);
    if (row.data) {
        const BlockScale s = block_scale(all, row.fmt, row.stype);
        if (threadIdx.x == 0) store_scale(row, int64_t(tr) * row.sld + tc, s.bits);
        by_fmt(row.fmt, [&](auto f) {
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                const int rr = r0 + kRows * rg + r;
                if (FULL || rr < row.rows)
                    store_values<f.value, FULL>(row.data + int64_t(rr) * row.ld, c0 + 8 * cl, row.cols, v[r], s.inv);
            }
        });
    }
    if (!col.data) return;
    const BlockScale s = block_scale(all, col.fmt, col.stype);
    if (threadIdx.x == 0) store_scale(col, int64_t(tc) * col.sld + tr, s.bits);
    transpose_in(v, nullptr, s.inv, col.fmt, lds.t);
    __syncthreads();
    transpose_out<FULL>(o, r0, lds.t);
}

// WHOLE, here and below: all tiles are whole and rows 16-byte aligned.  That kernel has the one body
// without divergent branches, and fits the registers of more waves: six a SIMD unit hide the
// memory's latency here, and five take 7 % longer.  No instance may spill registers: the compiler
// has been seen to reload one at the end of a divergent branch for a part of the lanes only.
template <typename T, bool WHOLE>
__global__ __launch_bounds__(kTileThreads, WHOLE ? 6 : 5) void q8_tile(const T *x, int64_t ldx, int vec, int rows,
                                                                       int cols, int tiles_c, Q8View row,
                                                                       Q8View col) {
    __shared__ TileLds lds;
    const int tr = blockIdx.x / tiles_c, tc = blockIdx.x - tr * tiles_c;
    if (WHOLE)
        tile_body<true>(x, ldx, true, rows, cols, tr, tc, row, col, lds);
    else if (tr * 128 + 128 <= rows && tc * 128 + 128 <= cols)
        tile_body<true>(x, ldx, vec, rows, cols, tr, tc, row, col, lds);
    else
        tile_body<false>(x, ldx, vec, rows, cols, tr, tc, row, col, lds);
}

// ---- gated unit -----------------------------------------------------------------

// 1 / (1 + exp(-g)).  exp(-g) = 2^(hi + lo), hi the rounded product with log2(e) and lo what the
// rounding and the constant leave out, so the error does not grow with |g|.  Beyond +-88.5, where
// the result is 1 or less than any normal number, g is taken as that, and all steps are finite; the
// reciprocal instruction gives 0 in place of a subnormal number, so that g sigmoid(g) is 0 there too,
// however large |g| is (tests/test_gpu_q8_tails.py).
__device__ __forceinline__ float sigmoid(float g) {
    const float L = 1.44269502f, L2 = 1.92596299e-8f;      // log2(e) in two parts
    g = __builtin_amdgcn_fmed3f(g, -88.5f, 88.5f);
    const float hi = -g * L;
    const float lo = fmaf(-g, L2, fmaf(-g, L, -hi));
    const float e = __builtin_amdgcn_exp2f(hi);
    return __builtin_amdgcn_rcpf(1.f + fmaf(e, lo * 0.693147181f, e));
}

// h = g sigmoid(g) u, with g and u kept in 8 bits: bound by the memory, the sigmoid's arithmetic
// beside it.  As q8_rows: 16 lanes a block, which write up to three blocks of one read.  8192x8192 bf16
// with its checkpoint in 85 us (5.5 TB/s).  VEC: rows are 16-byte aligned (8192x8191, which are not,
// 105 us, and 142 with the columns looked at one by one).
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void swiglu8_rows(const T *gu, int64_t ldg, int hidden, int up,
                                                    Q8View h, Q8View saved, int nb, int64_t total) {
    const int cl = threadIdx.x & 15;
    const int64_t step = int64_t(gridDim.x) * 16;
    for (int64_t i = int64_t(blockIdx.x) * 16 + (threadIdx.x >> 4); i < total; i += step) {
        const int r = int(i / nb), b = int(i - int64_t(r) * nb);
        const T *p = gu + int64_t(r) * ldg;
        const int c = b * kQ8Block + 8 * cl;
        float g[8], u[8], v[8];
        load8<false>(p, c, hidden, VEC, g);
        load8<false>(p + up, c, hidden, VEC, u);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = g[k] * sigmoid(g[k]) * u[k];
        const bool in = b * kQ8Block < hidden;             // not a block between the two
        if (in) by_fmt(h.fmt, [&](auto f) { emit_block<f.value, false, true>(h, r, b, cl, v); });
        if (saved.data)
            by_fmt(saved.fmt, [&](auto f) {
                emit_block<f.value, false, false>(saved, r, b, cl, g);
                if (in) emit_block<f.value, false, false>(saved, r, b + up / kQ8Block, cl, u);
            });
    }
}

// Eight 8-bit values times their scale.
__device__ __forceinline__ void values8(intx2 q, float s, int fmt, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        typedef float f2 __attribute__((ext_vector_type(2)));
        f2 a, b;
        if (fmt == DS_Q8_E4M3) {
            a = __builtin_amdgcn_cvt_pk_f32_fp8(q[i], false);
            b = __builtin_amdgcn_cvt_pk_f32_fp8(q[i], true);
        } else {
            a = __builtin_amdgcn_cvt_pk_f32_bf8(q[i], false);
            b = __builtin_amdgcn_cvt_pk_f32_bf8(q[i], true);
        }
        v[4 * i] = a[0] * s;
        v[4 * i + 1] = a[1] * s;
        v[4 * i + 2] = b[0] * s;
        v[4 * i + 3] = b[1] * s;
    }
}

// Eight bytes of a row that ends at `cols`, 0 past it.
template <bool FULL>
__device__ __forceinline__ intx2 bytes8(const uint8_t *row, int c, int cols) {
    if (FULL || c + 8 <= cols) return *reinterpret_cast<const intx2 *>(row + c);
    intx2 q = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (c + i < cols) q[i >> 2] |= int(unsigned(row[c + i]) << (8 * (i & 3)));
    return q;
}

template <bool FULL, typename T>
__device__ __forceinline__ void grad_body(const Q8View &saved, const T *dh, int64_t ldh, int vec, int hidden,
                                          int up, int tr, int tc, const Q8View &dgu, const Q8View &dgu_t,
                                          const Q8View &h_t, TileLds &lds) {
    const int cl = threadIdx.x & 15, rg = threadIdx.x >> 4;
    const int r0 = tr * 128, c0 = tc * 128, c = c0 + 8 * cl;
    // The gate's columns end at `up` here, zeros from `hidden` on; a tile past `hidden` has those alone.
    const bool in = FULL || c0 < hidden;
    TileOut o[3] = {{dgu, dgu_t, c0, c0}, {dgu, dgu_t, up + c0, up + c0}, {Q8View{}, h_t, c0, c0}};
    o[0].row.cols = up;
    o[0].col.rows = up;
    if (!in) o[1].row.data = o[1].col.data = o[2].col.data = nullptr;

    struct Raw {
        intx2 g, u;
        float sg, su;
        Eight<T> d;
    };
    auto fetch = [&](int rr) {
        Raw x{};
        if (FULL || (in && rr < saved.rows)) {
            const uint8_t *q = saved.data + int64_t(rr) * saved.ld;
            const int64_t si = int64_t(rr) * saved.sld + tc;
            x.g = bytes8<FULL>(q, c, hidden);
            x.u = bytes8<FULL>(q + up, c, hidden);
            x.sg = scale_at(saved.scale, saved.stype, si);
            x.su = scale_at(saved.scale, saved.stype, si + up / kQ8Block);
            x.d = raw8<FULL>(dh + int64_t(rr) * ldh, c, hidden, FULL || vec);
        }
        return x;
    };
    Raw x[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) x[r] = fetch(r0 + kRows * rg + r);
    // One output after another, with silu(g) and the loaded bytes held: all three at once do not fit
    // the registers of two workgroups a CU.
    float silu[kRows][8], v[kRows][8];
    auto emit = [&](int n) {
        if (o[n].row.data) emit_rows<FULL, true>(v, o[n], r0);
        // (the tile before is read out of LDS before the first of these barriers and written after)
        if (o[n].col.data) emit_columns<FULL, true>(v, o[n], r0, lds);
    };
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        float g[8], u[8];
        values8(x[r].g, x[r].sg, saved.fmt, g);
        values8(x[r].u, x[r].su, saved.fmt, u);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float s = sigmoid(g[k]);
            silu[r][k] = g[k] * s;
            v[r][k] = float(x[r].d.t[k]) * u[k] * fmaf(silu[r][k], 1.f - s, s);
        }
    }
    emit(0);
    // (decoded again below: kept, the decoded values would not fit)
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        x[r].d.forget();
        __asm__ volatile("" : "+v"(x[r].u));
    }
#pragma unroll
    for (int r = 0; r < kRows; ++r)
#pragma unroll
        for (int k = 0; k < 8; ++k) v[r][k] = float(x[r].d.t[k]) * silu[r][k];
    emit(1);
    if (!o[2].col.data) return;
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        float u[8];
        values8(x[r].u, x[r].su, saved.fmt, u);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[r][k] = silu[r][k] * u[k];
    }
    emit(2);
}

// A tile of g, u and dh gives three outputs in five layouts.  Its 602 MB at 8192x8192 would take
// 116 us; bound by the vector unit (51 instructions a value: the sigmoid, three products, and five
// maxima, scalings and roundings) and by how few waves the registers leave to hide latency: bf16 dh
// 150 us with 16 waves a CU; fp32 dh, whose loaded rows take twice the registers, 241 with 8.
template <typename T, bool WHOLE>
__global__ __launch_bounds__(kTileThreads, sizeof(T) == 4 ? 3 : 4) void swiglu8_grad_tile(
    Q8View saved, const T *dh, int64_t ldh, int vec, int hidden, int up, int tiles_c, Q8View dgu, Q8View dgu_t,
    Q8View h_t) {
    __shared__ TileLds lds;
    const int tr = blockIdx.x / tiles_c, tc = blockIdx.x - tr * tiles_c;
    if (WHOLE || (vec && tr * 128 + 128 <= saved.rows && tc * 128 + 128 <= hidden))
        grad_body<true>(saved, dh, ldh, true, hidden, up, tr, tc, dgu, dgu_t, h_t, lds);
    else
        grad_body<false>(saved, dh, ldh, vec, hidden, up, tr, tc, dgu, dgu_t, h_t, lds);
}

bool rows16(const void *p, int type, int64_t ld) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld * type_bytes(type) % 16 == 0;
}

// Calls fn with a null pointer of the element type.
template <typename Fn>
int by_type(int type, Fn fn) {
    if (type == DS_TYPE_F32) fn(static_cast<const float *>(nullptr));
    else if (type == DS_TYPE_F16) fn(static_cast<const _Float16 *>(nullptr));
    else fn(static_cast<const __bf16 *>(nullptr));
    return hip_ok(hipGetLastError(), "8-bit kernel launch") ? DS_OK : DS_EHIP;
}

// One workgroup a tile.
int tile_grid(int64_t rows, int64_t cols, unsigned *grid) {
    const int64_t n = q8_up(rows) * q8_up(cols);
    *grid = unsigned(n);
    return launch_check(n, kTileThreads, "tiles of 128 x 128");
}

// Workgroups of 16 blocks each, at most what fills the chip several times over.
unsigned row_grid(int64_t blocks) { return unsigned(std::min<int64_t>((blocks + 15) / 16, 16384)); }

int shape_error(const char *what, const ds_q8 *m, int64_t rows, int64_t cols) {
    set_error("%s is %lld x %lld, not %lld x %lld", what, (long long)m->rows, (long long)m->cols,
              (long long)rows, (long long)cols);
    return DS_EINVAL;
}

// Checks an output of the given shape with 1x128 blocks.
int check_out(const ds_q8 *m, const char *what, int64_t rows, int64_t cols) {
    const int rc = q8_check(m, what);
    if (rc != DS_OK) return rc;
    if (m->rows != rows || m->cols != cols) return shape_error(what, m, rows, cols);
    if (m->block_rows != 1) {
        set_error("%s: block_rows %d, not 1", what, m->block_rows);
        return DS_EINVAL;
    }
    return DS_OK;
}

int check_hidden(int64_t hidden, int64_t up) {
    if (hidden < 0 || up < hidden || up % kQ8Block != 0 || up > 0x3fffffff) {
        set_error("hidden %lld, up %lld (a multiple of 128, at least hidden)", (long long)hidden,
                  (long long)up);
        return DS_EINVAL;
    }
    return DS_OK;
}

}  // namespace
}  // namespace ds

using namespace ds;

extern "C" {

int ds_q8_quantize(const void *x, int type, int64_t rows, int64_t cols, int64_t ldx, const ds_q8 *row,
                   const ds_q8 *col, hipStream_t stream) {
    int rc = plain_check(x, type, rows, cols, ldx, "x");
    if (rc != DS_OK) return rc;
    if (!row && !col) {
        set_error("ds_q8_quantize has nothing to write");
        return DS_EINVAL;
    }
    if (row && (rc = q8_check(row, "row")) != DS_OK) return rc;
    if (col && (rc = q8_check(col, "col")) != DS_OK) return rc;
    if (row && (row->rows != rows || row->cols != cols)) return shape_error("row", row, rows, cols);
    if (col && (col->rows != cols || col->cols != rows)) return shape_error("col", col, cols, rows);
    if (row && col && row->block_rows != col->block_rows) {
        set_error("row has block_rows %d, col %d", row->block_rows, col->block_rows);
        return DS_EINVAL;
    }
    if (rows == 0 || cols == 0) return DS_OK;
    const Q8View vr = q8_view(row), vc = q8_view(col);
    const int vec = rows16(x, type, ldx);
    if (!col && row->block_rows == 1) {
        const int nb = int(q8_up(cols));
        const int64_t total = rows * nb;
        return by_type(type, [&](auto *t) {
            using T = std::remove_cv_t<std::remove_pointer_t<decltype(t)>>;
            q8_rows<T><<<row_grid(total), 256, 0, stream>>>(static_cast<const T *>(x), ldx, vec, vr, nb,
                                                            total);
        });
    }
    unsigned grid;
    if ((rc = tile_grid(rows, cols, &grid)) != DS_OK) return rc;
    return by_type(type, [&](auto *t) {
        using T = std::remove_cv_t<std::remove_pointer_t<decltype(t)>>;
        (vec && rows % 128 == 0 && cols % 128 == 0 ? q8_tile<T, true> : q8_tile<T, false>)
            <<<grid, kTileThreads, 0, stream>>>(static_cast<const T *>(x), ldx, vec, int(rows), int(cols),
                                                int(q8_up(cols)), vr, vc);
    });
}

int ds_swiglu8(const void *gu, int type, int64_t rows, int64_t hidden, int64_t up, int64_t ldg,
               const ds_q8 *h, const ds_q8 *saved, hipStream_t stream) {
    int rc = check_hidden(hidden, up);
    if (rc != DS_OK) return rc;
    if ((rc = plain_check(gu, type, rows, up + hidden, ldg, "gu")) != DS_OK) return rc;
    if ((rc = check_out(h, "h", rows, hidden)) != DS_OK) return rc;
    if (saved && (rc = check_out(saved, "saved", rows, up + hidden)) != DS_OK) return rc;
    const Q8View vh = q8_view(h), vs = q8_view(saved);
    const int vec = rows16(gu, type, ldg);
    // without a checkpoint nothing is written between the two factors
    const int nb = int(saved ? up / kQ8Block : q8_up(hidden));
    const int64_t total = rows * nb;
    if (total == 0) return DS_OK;
    return by_type(type, [&](auto *t) {
        using T = std::remove_cv_t<std::remove_pointer_t<decltype(t)>>;
        // the gate's block that reaches past hidden ends at `up` in the checkpoint
        (vec ? swiglu8_rows<T, true> : swiglu8_rows<T, false>)<<<row_grid(total), 256, 0, stream>>>(
            static_cast<const T *>(gu), ldg, int(hidden), int(up), vh, vs, nb, total);
    });
}

int ds_swiglu8_grad(const ds_q8 *saved, const void *dh, int type, int64_t hidden, int64_t up, int64_t ldh,
                    const ds_q8 *dgu, const ds_q8 *dgu_t, const ds_q8 *h_t, hipStream_t stream) {
    int rc = check_hidden(hidden, up);
    if (rc != DS_OK) return rc;
    if ((rc = q8_check(saved, "saved")) != DS_OK) return rc;
    const int64_t rows = saved->rows;
    if ((rc = check_out(saved, "saved", rows, up + hidden)) != DS_OK) return rc;
    if ((rc = plain_check(dh, type, rows, hidden, ldh, "dh")) != DS_OK) return rc;
    if (!dgu && !dgu_t && !h_t) {
        set_error("ds_swiglu8_grad has nothing to write");
        return DS_EINVAL;
    }
    if (dgu && (rc = check_out(dgu, "dgu", rows, up + hidden)) != DS_OK) return rc;
    if (dgu_t && (rc = check_out(dgu_t, "dgu_t", up + hidden, rows)) != DS_OK) return rc;
    if (h_t && (rc = check_out(h_t, "h_t", hidden, rows)) != DS_OK) return rc;
    if (rows == 0 || up == 0) return DS_OK;
    unsigned grid;
    if ((rc = tile_grid(rows, up, &grid)) != DS_OK) return rc;
    const Q8View vs = q8_view(saved), vd = q8_view(dgu), vt = q8_view(dgu_t), vh = q8_view(h_t);
    const int vec = rows16(dh, type, ldh);
    return by_type(type, [&](auto *t) {
        using T = std::remove_cv_t<std::remove_pointer_t<decltype(t)>>;
        (vec && rows % 128 == 0 && hidden == up ? swiglu8_grad_tile<T, true> : swiglu8_grad_tile<T, false>)
            <<<grid, kTileThreads, 0, stream>>>(vs, static_cast<const T *>(dh), ldh, vec, int(hidden), int(up),
                                                int(up / kQ8Block), vd, vt, vh);
    });
}

}  // extern "C"
