// Quantization to 8 bits in blocks of 128, and the gated unit with its activations kept
// in 8 bits.  Both move memory and little else: every input is read once and every
// output, transposes too, written once by the same launch.
#include "q8.h"

namespace ds {

int q8_check(const ds_q8 *m, const char *what) {
    if (!m) {
        set_error("%s: null 8-bit matrix", what);
        return DS_EINVAL;
    }
    if (m->rows < 0 || m->cols < 0 || m->rows > 0x7fffffff || m->cols > 0x7fffffff) {
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

// Loads eight elements of a row of `cols` as fp32, 0 past its end; vec: rows are 16-byte aligned.
template <typename T>
__device__ __forceinline__ void load8(const T *row, int c, int cols, bool vec, float (&v)[8]) {
    if (vec && c + 8 <= cols) {
        T t[8];
#pragma unroll
        for (size_t i = 0; i < sizeof(t) / 16; ++i)
            reinterpret_cast<intx4 *>(t)[i] = reinterpret_cast<const intx4 *>(row + c)[i];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = float(t[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = c + i < cols ? float(row[c + i]) : 0.f;
    }
}

// The largest magnitude of the values as bits, NaN and infinities above all.
template <int N>
__device__ __forceinline__ unsigned max_bits(const float (&v)[N]) {
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
    return m;
}
// The same of the finite ones.
template <int N>
__device__ __forceinline__ unsigned max_finite(const float (&v)[N]) {
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) m = max(m, finite_abs(v[i]));
    return m;
}

__device__ __forceinline__ intx2 pack8(const float (&v)[8], float inv, int fmt) {
    return intx2{pack4(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv, fmt),
                 pack4(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv, fmt)};
}

// Eight bytes to columns c .. of a row that ends at `cols`.
__device__ __forceinline__ void store8(uint8_t *row, int c, int cols, intx2 q) {
    if (c + 8 <= cols) {
        *reinterpret_cast<intx2 *>(row + c) = q;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i < cols) row[c + i] = uint8_t(unsigned(q[i >> 2]) >> (8 * (i & 3)));
    }
}

// One 1x128 block of row r at columns c0 .. c0+127, held by 16 lanes of eight values each.
__device__ __forceinline__ void emit_block(const Q8View &m, int r, int blk, int cl, const float (&v)[8]) {
    unsigned top = max16(max_bits(v));
    // what is not finite sets no scale: only a wave that holds some looks at each value
    if (__any(top >= 0x7f800000u)) top = max16(max_finite(v));
    const BlockScale s = block_scale(top, m.fmt, m.stype);
    store8(m.data + int64_t(r) * m.ld, blk * kQ8Block + 8 * cl, m.cols, pack8(v, s.inv, m.fmt));
    if (cl == 0) store_scale(m, int64_t(r) * m.sld + blk, s.bits);
}

// Rows alone: 16 lanes a block.
template <typename T>
__global__ __launch_bounds__(256) void q8_rows(const T *x, int64_t ldx, int vec, Q8View m, int nb,
                                               int64_t total) {
    const int cl = threadIdx.x & 15;
    const int64_t step = int64_t(gridDim.x) * 16;
    for (int64_t i = int64_t(blockIdx.x) * 16 + (threadIdx.x >> 4); i < total; i += step) {
        const int r = int(i / nb), b = int(i - int64_t(r) * nb);
        float v[8];
        load8(x + int64_t(r) * ldx, b * kQ8Block + 8 * cl, m.cols, vec, v);
        emit_block(m, r, b, cl, v);
    }
}

// ---- tiles of 128 x 128 -----------------------------------------------------------
// 512 threads; thread t holds rows 4 (t / 16) .. + 3 of columns 8 (t % 16) .. + 7.
constexpr int kTileThreads = 512, kRows = 4, kTileWaves = kTileThreads / 64;

struct TileLds {
    unsigned colmax[kTileWaves][128];
    BlockScale cs[128];
    // transposed bytes: column c's 16 rows of wave w are the 16 bytes at c * 8 + (w ^ c / 8 % 8), so
    // that the 16 columns a wave writes at once lie in different banks
    intx4 t[128 * 8];
};

// Largest over the wave's 16 rows of column 8 (lane % 16) + c, for each c.
__device__ __forceinline__ unsigned over_rows(unsigned m) {
    m = max(m, unsigned(__shfl_xor(int(m), 16)));
    return max(m, unsigned(__shfl_xor(int(m), 32)));
}

// Writes a tile's values to `row` at (r0, c0) and transposed to `col` at (rc0, r0); either has
// data == null when not wanted.  Elements outside the matrices hold 0.
__device__ __forceinline__ void emit_tile(const float (&v)[kRows][8], const Q8View &row, const Q8View &col,
                                          int r0, int c0, int rc0, TileLds &lds) {
    const int tid = threadIdx.x, cl = tid & 15, rg = tid >> 4, w = tid >> 6;
    const bool square = (row.data ? row.shift : col.shift) != 0;
    if (row.data && !square)
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const int rr = r0 + kRows * rg + r;
            if (rr < row.rows) emit_block(row, rr, c0 >> 7, cl, v[r]);
        }
    if (!col.data && !square) return;
    unsigned m[8], any = 0;
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        const float u[kRows] = {v[0][c], v[1][c], v[2][c], v[3][c]};
        m[c] = max_bits(u);
        any = max(any, m[c]);
    }
    if (__any(any >= 0x7f800000u))
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            const float u[kRows] = {v[0][c], v[1][c], v[2][c], v[3][c]};
            m[c] = max_finite(u);
        }
#pragma unroll
    for (int c = 0; c < 8; ++c) m[c] = over_rows(m[c]);
    if ((tid & 48) == 0) {
        unsigned *p = lds.colmax[w] + 8 * cl;
        reinterpret_cast<intx4 *>(p)[0] = intx4{int(m[0]), int(m[1]), int(m[2]), int(m[3])};
        reinterpret_cast<intx4 *>(p)[1] = intx4{int(m[4]), int(m[5]), int(m[6]), int(m[7])};
    }
    __syncthreads();
    unsigned all = 0;
    if (square) {
#pragma unroll
        for (int c = 0; c < 8; ++c)
#pragma unroll
            for (int i = 0; i < kTileWaves; ++i) all = max(all, lds.colmax[i][8 * cl + c]);
        all = max16(all);
        if (row.data) {
            const BlockScale s = block_scale(all, row.fmt, row.stype);
            if (tid == 0) store_scale(row, int64_t(r0 >> 7) * row.sld + (c0 >> 7), s.bits);
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                const int rr = r0 + kRows * rg + r;
                if (rr < row.rows)
                    store8(row.data + int64_t(rr) * row.ld, c0 + 8 * cl, row.cols, pack8(v[r], s.inv, row.fmt));
            }
        }
        if (!col.data) return;
        if (tid == 0) {
            const BlockScale s = block_scale(all, col.fmt, col.stype);
            store_scale(col, int64_t(rc0 >> 7) * col.sld + (r0 >> 7), s.bits);
        }
    }
    if (tid < 128) {
        unsigned top = all;
        if (!square)
#pragma unroll
            for (int i = 0; i < kTileWaves; ++i) top = max(top, lds.colmax[i][tid]);
        const BlockScale s = block_scale(top, col.fmt, col.stype);
        lds.cs[tid] = s;
        if (!square && rc0 + tid < col.rows)
            store_scale(col, int64_t(rc0 + tid) * col.sld + (r0 >> 7), s.bits);
    }
    __syncthreads();
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        const int cc = 8 * cl + c;
        const float inv = lds.cs[cc].inv;
        reinterpret_cast<int *>(lds.t)[(cc * 8 + (w ^ (cl & 7))) * 4 + (rg & 3)] =
            pack4(v[0][c] * inv, v[1][c] * inv, v[2][c] * inv, v[3][c] * inv, col.fmt);
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int i = j * kTileThreads + tid, c = i >> 3, g = i & 7, at = r0 + 16 * g;
        if (rc0 + c < col.rows && at < col.cols) {
            uint8_t *p = col.data + int64_t(rc0 + c) * col.ld;
            const intx4 q = lds.t[c * 8 + (g ^ (c >> 3 & 7))];
            if (at + 16 <= col.cols) {
                *reinterpret_cast<intx4 *>(p + at) = q;
            } else {
                store8(p, at, col.cols, intx2{q[0], q[1]});
                store8(p, at + 8, col.cols, intx2{q[2], q[3]});
            }
        }
    }
    // the next tile's first writes here come after a barrier that follows these reads
}

template <typename T>
__global__ __launch_bounds__(kTileThreads) void q8_tile(const T *x, int64_t ldx, int vec, int rows, int cols,
                                                        int tiles_c, Q8View row, Q8View col) {
    __shared__ TileLds lds;
    const int cl = threadIdx.x & 15, rg = threadIdx.x >> 4;
    const int tr = blockIdx.x / tiles_c, tc = blockIdx.x - tr * tiles_c;
    const int r0 = tr * 128, c0 = tc * 128;
    float v[kRows][8];
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        const int rr = r0 + kRows * rg + r;
        if (rr < rows) {
            load8(x + int64_t(rr) * ldx, c0 + 8 * cl, cols, vec, v[r]);
        } else {
#pragma unroll
            for (int c = 0; c < 8; ++c) v[r][c] = 0.f;
        }
    }
    emit_tile(v, row, col, r0, c0, c0, lds);
}

// ---- gated unit -----------------------------------------------------------------

// 1 / (1 + exp(-g)).  exp(-g) = 2^(hi + lo), hi the rounded product with log2(e) and lo
// what the rounding and the constant leave out, so the error does not grow with |g|;
// the quotient by one Newton step on the reciprocal.
__device__ __forceinline__ float sigmoid(float g) {
    const float L = 1.44269502f, L2 = 1.92596299e-8f;      // log2(e) in two parts
    const float hi = -g * L;
    const float lo = fmaf(-g, L, -hi) - g * L2;
    float e = __builtin_amdgcn_exp2f(hi);
    // e * 2^lo; where e is 0 or infinite the result is 1 or 0 whatever lo says
    e = fabsf(hi) < 127.9f ? fmaf(e, lo * 0.693147181f, e) : e;
    const float d = 1.f + e;
    const float r = __builtin_amdgcn_rcpf(d);
    const float n = fmaf(fmaf(-d, r, 1.f), r, r);
    return d < 1e38f ? n : r;                              // infinite d: r is 0 already
}

template <typename T>
__global__ __launch_bounds__(256) void swiglu8_rows(const T *gu, int64_t ldg, int vec, int hidden, int up,
                                                    Q8View h, Q8View saved, int nb, int64_t total) {
    const int cl = threadIdx.x & 15;
    const int64_t step = int64_t(gridDim.x) * 16;
    for (int64_t i = int64_t(blockIdx.x) * 16 + (threadIdx.x >> 4); i < total; i += step) {
        const int r = int(i / nb), b = int(i - int64_t(r) * nb);
        const T *p = gu + int64_t(r) * ldg;
        const int c = b * kQ8Block + 8 * cl;
        float g[8], u[8], v[8];
        load8(p, c, hidden, vec, g);
        load8(p + up, c, hidden, vec, u);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = g[k] * sigmoid(g[k]) * u[k];
        const bool in = b * kQ8Block < hidden;             // not a block between the two
        if (in) emit_block(h, r, b, cl, v);
        if (saved.data) {
            emit_block(saved, r, b, cl, g);
            if (in) emit_block(saved, r, b + up / kQ8Block, cl, u);
        }
    }
}

// Eight 8-bit values times their scale; columns from `cols` on are 0.
__device__ __forceinline__ void values8(intx2 q, float s, int fmt, int c, int cols, float (&v)[8]) {
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
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = c + i < cols ? v[i] : 0.f;
}

// Eight bytes of a row that ends at `cols`, 0 past it.
__device__ __forceinline__ intx2 bytes8(const uint8_t *row, int c, int cols) {
    if (c + 8 <= cols) return *reinterpret_cast<const intx2 *>(row + c);
    intx2 q = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (c + i < cols) q[i >> 2] |= int(unsigned(row[c + i]) << (8 * (i & 3)));
    return q;
}

template <typename T>
__global__ __launch_bounds__(kTileThreads, 4) void swiglu8_grad_tile(Q8View saved, const T *dh, int64_t ldh,
                                                                  int vec, int hidden, int up, int tiles_c,
                                                                  Q8View dgu, Q8View dgu_t, Q8View h_t) {
    __shared__ TileLds lds;
    const int cl = threadIdx.x & 15, rg = threadIdx.x >> 4;
    const int tr = blockIdx.x / tiles_c, tc = blockIdx.x - tr * tiles_c;
    const int r0 = tr * 128, c0 = tc * 128, c = c0 + 8 * cl;
    float dg[kRows][8], du[kRows][8], h[kRows][8];
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        const int rr = r0 + kRows * rg + r;
        if (rr < saved.rows && c0 < hidden) {
            const uint8_t *q = saved.data + int64_t(rr) * saved.ld;
            const int64_t si = int64_t(rr) * saved.sld + tc;
            float g[8], u[8], d[8];
            values8(bytes8(q, c, hidden), scale_at(saved.scale, saved.stype, si), saved.fmt, c, hidden, g);
            values8(bytes8(q + up, c, hidden), scale_at(saved.scale, saved.stype, si + up / kQ8Block), saved.fmt,
                    c, hidden, u);
            load8(dh + int64_t(rr) * ldh, c, hidden, vec, d);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float s = sigmoid(g[k]), silu = g[k] * s;
                dg[r][k] = d[k] * u[k] * (s * (1.f + g[k] * (1.f - s)));
                du[r][k] = d[k] * silu;
                h[r][k] = silu * u[k];
            }
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) dg[r][k] = du[r][k] = h[r][k] = 0.f;
        }
    }
    if (dgu.data || dgu_t.data) {
        // the gate's columns end at `up` here, zeros from `hidden` on
        Q8View a = dgu, b = dgu_t;
        a.cols = up;
        b.rows = up;
        emit_tile(dg, a, b, r0, c0, c0, lds);
        if (c0 < hidden) emit_tile(du, dgu, dgu_t, r0, up + c0, up + c0, lds);
    }
    if (h_t.data && c0 < hidden) {
        Q8View none = h_t;
        none.data = nullptr;
        emit_tile(h, none, h_t, r0, c0, c0, lds);
    }
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

// One workgroup a tile; DS_EUNSUPPORTED past the grid's limit.
int tile_grid(int64_t rows, int64_t cols, unsigned *grid) {
    const int64_t n = q8_up(rows) * q8_up(cols);
    if (n > kGridLimit) {
        set_error("%lld tiles of 128 x 128 are more than a launch takes", (long long)n);
        return DS_EUNSUPPORTED;
    }
    *grid = unsigned(n);
    return DS_OK;
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
        q8_tile<T><<<grid, kTileThreads, 0, stream>>>(static_cast<const T *>(x), ldx, vec, int(rows), int(cols),
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
        swiglu8_rows<T><<<row_grid(total), 256, 0, stream>>>(static_cast<const T *>(gu), ldg, vec,
                                                             int(hidden), int(up), vh, vs, nb, total);
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
        swiglu8_grad_tile<T><<<grid, kTileThreads, 0, stream>>>(vs, static_cast<const T *>(dh), ldh, vec,
                                                       int(hidden), int(up), int(up / kQ8Block), vd, vt, vh);
    });
}

}  // extern "C"
