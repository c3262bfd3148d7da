// C = A B^T of 8-bit matrices with a scale for each block of 128 along the reduction.
#include <type_traits>

#include "kern_common.h"
#include "q8.h"

namespace ds {
namespace {

struct Q8MatArgs {
    Q8View a, b;
    void *c;
    int64_t ldc;
    int type;
    int M, N, K, nkt;
};

__device__ __forceinline__ void store_c(void *c, int type, int64_t i, float v) {
    if (type == DS_TYPE_F32) static_cast<float *>(c)[i] = v;
    else if (type == DS_TYPE_F16) static_cast<_Float16 *>(c)[i] = _Float16(v);
    else static_cast<__bf16 *>(c)[i] = __bf16(v);
}

// 32 bytes of a row from k on, 0 from K on.
__device__ __forceinline__ intx8 load32(const uint8_t *row, int k, int K) {
    intx8 v = {0, 0, 0, 0, 0, 0, 0, 0};
    if (k + 32 <= K) {
        const intx4 *p = reinterpret_cast<const intx4 *>(row + k);
        const intx4 x = p[0], y = p[1];
        v = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
#pragma unroll
        for (int i = 0; i < 32; ++i)
            if (k + i < K) v[i >> 2] |= int(unsigned(row[k + i]) << (8 * (i & 3)));
    }
    return v;
}

// One 128-long step of a 16 x 16 product, lane l holding bytes 32 (l / 16) .. + 31 of row
// l % 16 of either operand: the same 8 bytes of both make one bf16 instruction, so it does
// not matter which k those are.  Result: row 4 (l / 16) + i of `b`, row l % 16 of `a`.
template <int FA, int FB>
__device__ __forceinline__ floatx4 dot128(intx8 a, intx8 b) {
    floatx4 p = {0, 0, 0, 0};
#pragma unroll
    for (int u = 0; u < 4; ++u)
        p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(to_bf16<FB>(b[2 * u], b[2 * u + 1]),
                                                    to_bf16<FA>(a[2 * u], a[2 * u + 1]), p, 0, 0, 0);
    return p;
}

// 16 x 16 of C a workgroup; its waves take the steps of the reduction in turn.
template <int FA, int FB>
__global__ __launch_bounds__(1024) void q8_few(Q8MatArgs a) {
    __shared__ float red[16 * 256];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, nw = blockDim.x >> 6;
    const int li = lane & 15, lg = lane >> 4;
    const int n0 = blockIdx.x * 16, m0 = blockIdx.y * 16;
    const int m = min(m0 + li, a.M - 1), n = min(n0 + li, a.N - 1);
    const uint8_t *pa = a.a.data + int64_t(m) * a.a.ld, *pb = a.b.data + int64_t(n) * a.b.ld;
    const int64_t sa = int64_t(m >> a.a.shift) * a.a.sld;
    int64_t sb[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        sb[i] = int64_t(min(n0 + 4 * lg + i, a.N - 1) >> a.b.shift) * a.b.sld;
    floatx4 acc = {0, 0, 0, 0};
    for (int kt = w; kt < a.nkt; kt += nw) {
        const int k = kt * kQ8Block + 32 * lg;
        const floatx4 p = dot128<FA, FB>(load32(pa, k, a.K), load32(pb, k, a.K));
        const float s = scale_at(a.a.scale, a.a.stype, sa + kt);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] += p[i] * (s * scale_at(a.b.scale, a.b.stype, sb[i] + kt));
    }
    *reinterpret_cast<floatx4 *>(red + w * 256 + li * 16 + 4 * lg) = acc;
    __syncthreads();
    for (int e = threadIdx.x; e < 256; e += blockDim.x) {
        float v = 0.f;
        for (int i = 0; i < nw; ++i) v += red[i * 256 + e];
        const int r = m0 + (e >> 4), c = n0 + (e & 15);
        if (r < a.M && c < a.N) store_c(a.c, a.type, int64_t(r) * a.ldc + c, v);
    }
}

template <int V>
using Fmt = std::integral_constant<int, V>;

// Calls fn with the operands' formats as constants.
template <typename Fn>
int by_formats(int fa, int fb, Fn fn) {
    if (fa == DS_Q8_E4M3) fb == DS_Q8_E4M3 ? fn(Fmt<0>{}, Fmt<0>{}) : fn(Fmt<0>{}, Fmt<1>{});
    else fb == DS_Q8_E4M3 ? fn(Fmt<1>{}, Fmt<0>{}) : fn(Fmt<1>{}, Fmt<1>{});
    return hip_ok(hipGetLastError(), "8-bit matmul launch") ? DS_OK : DS_EHIP;
}

}  // namespace
}  // namespace ds

using namespace ds;

extern "C" int ds_q8_matmul(const ds_q8 *a, const ds_q8 *b, void *c, int type, int64_t ldc,
                            hipStream_t stream) {
    int rc;
    if ((rc = q8_check(a, "a")) != DS_OK || (rc = q8_check(b, "b")) != DS_OK) return rc;
    if (a->cols != b->cols || a->scale_type != b->scale_type) {
        set_error("a has %lld columns and scale type %d, b %lld and %d", (long long)a->cols,
                  a->scale_type, (long long)b->cols, b->scale_type);
        return DS_EINVAL;
    }
    if ((rc = plain_check(c, type, a->rows, b->rows, ldc, "c")) != DS_OK) return rc;
    if (a->rows == 0 || b->rows == 0) return DS_OK;
    Q8MatArgs g{q8_view(a), q8_view(b), c, ldc, type, int(a->rows), int(b->rows), int(a->cols),
                int(q8_up(a->cols))};
    const int64_t tm = (a->rows + 15) / 16, tn = (b->rows + 15) / 16;
    if (tm > 65535) {
        set_error("ds_q8_matmul: %lld rows", (long long)a->rows);
        return DS_EUNSUPPORTED;
    }
    const int waves = std::clamp(g.nkt, 1, 8);
    return by_formats(g.a.fmt, g.b.fmt, [&](auto fa, auto fb) {
        q8_few<fa.value, fb.value><<<dim3(unsigned(tn), unsigned(tm)), 64 * waves, 0, stream>>>(g);
    });
}
