// The 8-bit formats and block scales on the device, and the host checks of ds_q8,
// shared by kern_q8.hip and kern_q8_matmul.hip.
#pragma once

#include <hip/hip_runtime.h>

#include "ds_internal.h"

namespace ds {

// ---- host -------------------------------------------------------------------
constexpr int kQ8Block = DS_Q8_BLOCK;

// DS_OK, or DS_EINVAL with the error set: `what` names the operand.
int q8_check(const ds_q8 *m, const char *what);
// The same for a plain matrix of DS_TYPE_* elements, ld elements between rows.
int plain_check(const void *p, int type, int64_t rows, int64_t cols, int64_t ld, const char *what);

// DS_OK, or DS_EUNSUPPORTED with the error set where a launch, whose work-items are counted in 32 bits,
// does not take so many workgroups.
int launch_check(int64_t groups, int threads, const char *what);

inline int64_t q8_up(int64_t n) { return (n + kQ8Block - 1) / kQ8Block; }
inline int type_bytes(int type) { return type == DS_TYPE_F32 ? 4 : 2; }

// ---- device -----------------------------------------------------------------
typedef int intx2 __attribute__((ext_vector_type(2)));
typedef int intx4 __attribute__((ext_vector_type(4)));
typedef int intx8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

// An 8-bit matrix as kernels take it.
struct Q8View {
    uint8_t *data;
    void *scale;
    int64_t ld, sld;
    int rows, cols;
    int fmt, stype;
    int shift;                 // log2(block_rows): scale row of row r is r >> shift
};

inline Q8View q8_view(const ds_q8 *m) {
    if (!m) return Q8View{};
    return Q8View{static_cast<uint8_t *>(m->data), m->scale, m->ld, m->scale_ld, int(m->rows),
                  int(m->cols), m->format, m->scale_type, m->block_rows == 1 ? 0 : 7};
}

// The fp32 value of scale (row, block); scale rows are rows >> shift.
__device__ __forceinline__ float scale_at(const void *s, int stype, int64_t i) {
    if (stype == DS_SCALE_F32) return static_cast<const float *>(s)[i];
    const unsigned b = static_cast<const uint8_t *>(s)[i];
    return __uint_as_float(max(b << 23, 0x400000u));   // 2^-127 is the subnormal 0x00400000
}

struct BlockScale {
    float inv;                 // 1 / scale, what values are multiplied by
    unsigned bits;             // as stored: an exponent byte or fp32 bits
};

// The scale of a block whose largest magnitude is amax (fp32 bits, finite).  448 and
// 57344 are 1.75 * 2^8 and 1.75 * 2^15, so the power of two is amax's exponent less 8
// or 15, one more if its fraction is over 1.75; no rounding is involved.
__device__ __forceinline__ BlockScale block_scale(unsigned amax, int fmt, int stype) {
    if (stype == DS_SCALE_POW2) {
        const int e = max(int((amax + 0x1FFFFFu) >> 23) - (fmt == DS_Q8_E4M3 ? 8 : 15), 1);
        return {__uint_as_float(unsigned(254 - e) << 23), unsigned(e)};
    }
    const float s = fmaxf(__uint_as_float(amax) / (fmt == DS_Q8_E4M3 ? 448.f : 57344.f),
                          __uint_as_float(0x800000u));
    return {1.f / s, __float_as_uint(s)};
}

// A stored scale of a cache's row.  The byte 255 stands for no number, and a conversion by 2^(255 - 127) makes none of
// any byte.
__device__ __forceinline__ float scale_of(unsigned stored, int stype) {
    if (stype != DS_SCALE_POW2) return __uint_as_float(stored);
    return __uint_as_float(stored == 255u ? 0x7fc00000u : max(stored << 23, 0x400000u));
}

__device__ __forceinline__ void store_scale(const Q8View &m, int64_t i, unsigned bits) {
    if (m.stype == DS_SCALE_POW2) static_cast<uint8_t *>(m.scale)[i] = uint8_t(bits);
    else static_cast<unsigned *>(m.scale)[i] = bits;
}

// |v| as ordered bits, 0 where v is not finite: such values set no scale.
__device__ __forceinline__ unsigned finite_abs(float v) {
    const unsigned u = __float_as_uint(v) & 0x7fffffffu;
    return u < 0x7f800000u ? u : 0u;
}

// Four values to 8 bits, nearest even, first in the low byte.
template <int FMT>
__device__ __forceinline__ int pack4(float a, float b, float c, float d) {
    int r;
    __asm__("" : "=v"(r));                       // both halves are written: no need to clear it
    if constexpr (FMT == DS_Q8_E4M3) {
        r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, r, false);
        return __builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
    } else {
        r = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, r, false);
        return __builtin_amdgcn_cvt_pk_bf8_f32(c, d, r, true);
    }
}

// Eight 8-bit values times a power of two as bf16: exact where the results are normal numbers (both
// formats have fewer bits).
template <int FMT>
__device__ __forceinline__ bf16x8 to_bf16(int lo, int hi, float scale = 1.f) {
    const int w[2] = {lo, hi};
    bf16x8 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        bf16x2 t;
        if constexpr (FMT == DS_Q8_E4M3) {
            t = (i & 1) ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i >> 1], scale, true)
                        : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i >> 1], scale, false);
        } else {
            t = (i & 1) ? __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w[i >> 1], scale, true)
                        : __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w[i >> 1], scale, false);
        }
        r[2 * i] = t[0];
        r[2 * i + 1] = t[1];
    }
    return r;
}

// Largest of the 16 lanes of each row of lanes, in all of them.
__device__ __forceinline__ unsigned max16(unsigned v) {
    v = max(v, unsigned(__builtin_amdgcn_update_dpp(0, int(v), 0xB1, 0xF, 0xF, false)));   // lane ^ 1
    v = max(v, unsigned(__builtin_amdgcn_update_dpp(0, int(v), 0x4E, 0xF, 0xF, false)));   // lane ^ 2
    v = max(v, unsigned(__builtin_amdgcn_update_dpp(0, int(v), 0x141, 0xF, 0xF, false)));  // other quad
    v = max(v, unsigned(__builtin_amdgcn_update_dpp(0, int(v), 0x140, 0xF, 0xF, false)));  // other eight
    return v;
}

}  // namespace ds
