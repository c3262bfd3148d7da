// C = A B^T of 8-bit matrices with a scale for each block of 128 along the reduction.
#include <climits>
#include <new>
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
    int tiles_m, tiles_n, group;   // tiles of C; workgroups walk `group` rows of tiles at a time
    int ks, kps;                   // splits of the reduction, steps of 128 in each
    float *part;                   // ks > 1: ks partial products, M x N each
    int words;                     // power-of-two scales: words of four are aligned
    int cvec, pvec;                // rows of C, of a partial product, are 16-byte aligned
};

__device__ __forceinline__ void store_c(void *c, int type, int64_t i, float v) {
    if (type == DS_TYPE_F32) static_cast<float *>(c)[i] = v;
    else if (type == DS_TYPE_F16) static_cast<_Float16 *>(c)[i] = _Float16(v);
    else static_cast<__bf16 *>(c)[i] = __bf16(v);
}

// Four columns from `col` on of the row at `at`, as far as the row goes.
__device__ __forceinline__ void store4(void *c, int type, int64_t at, int col, int cols, int vec, floatx4 v) {
    if (vec && col + 4 <= cols) {
        if (type == DS_TYPE_F32) {
            *reinterpret_cast<floatx4 *>(static_cast<float *>(c) + at + col) = v;
        } else if (type == DS_TYPE_F16) {
            *reinterpret_cast<f16x4 *>(static_cast<_Float16 *>(c) + at + col) =
                f16x4{_Float16(v[0]), _Float16(v[1]), _Float16(v[2]), _Float16(v[3])};
        } else {
            *reinterpret_cast<bf16x4 *>(static_cast<__bf16 *>(c) + at + col) =
                bf16x4{__bf16(v[0]), __bf16(v[1]), __bf16(v[2]), __bf16(v[3])};
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (col + i < cols) store_c(c, type, at + col + i, v[i]);
    }
}

// The first n of 16 bytes.
__device__ __forceinline__ intx4 mask16(int n) {
    intx4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = n >= 4 * i + 4 ? -1 : n > 4 * i ? (1 << (8 * (n - 4 * i))) - 1 : 0;
    return v;
}

// 16 bytes from a 16-byte aligned p, zeros from the n-th on.  They are loaded whole where one of
// them exists: an aligned 16 bytes never reach past the page, or the allocation, of any one.
__device__ __forceinline__ intx4 first16(const uint8_t *p, int n) {
    intx4 v = {0, 0, 0, 0};
    if (n > 0) v = *reinterpret_cast<const intx4 *>(p);
    return v & mask16(n);
}
__device__ __forceinline__ intx8 whole32(const uint8_t *p) {
    const intx4 x = reinterpret_cast<const intx4 *>(p)[0], y = reinterpret_cast<const intx4 *>(p)[1];
    return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
}
__device__ __forceinline__ intx8 first32(const uint8_t *p, int n) {
    const intx4 x = first16(p, n), y = first16(p + 16, n - 16);
    return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
}

// Scales i .. i + 3 as fp32.
__device__ __forceinline__ floatx4 scales4(const void *s, int stype, int64_t i) {
    floatx4 v;
    if (stype == DS_SCALE_F32) {
        __builtin_memcpy(&v, static_cast<const float *>(s) + i, 16);   // aligned to 4
        return v;
    }
    unsigned w;
    __builtin_memcpy(&w, static_cast<const uint8_t *>(s) + i, 4);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = __uint_as_float(max((w >> (8 * k) & 255u) << 23, 0x400000u));
    return v;
}

// One 128-long step of a 16 x 16 product, lane l holding bytes 32 (l / 16) .. + 31 of row
// l % 16 of either operand: the same 8 bytes of both make one bf16 instruction, so it does
// not matter which k those are.  Result: row 4 (l / 16) + i of `b`, row l % 16 of `a`.
template <int FB>
__device__ __forceinline__ floatx4 dot128(const bf16x8 (&a)[4], intx8 b) {
    floatx4 p = {0, 0, 0, 0};
#pragma unroll
    for (int u = 0; u < 4; ++u)
        p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(to_bf16<FB>(b[2 * u], b[2 * u + 1]), a[u], p, 0, 0, 0);
    return p;
}

constexpr int kFewWaves = 8;

// C's 16 x 16 NT blocks for few rows of A: every byte of the weight is used once, so it passes once
// from memory to registers, in the layout of the matrix instructions, and bounds the time; LDS
// in between would only add to it.  A workgroup has 16 NT columns; each of its waves takes a run of
// the reduction's steps, two at a time in flight, and their sums meet in LDS.  Each step's sum is
// scaled by its two scales in fp32.  16x16384x8192 in 28 us (4.8 TB/s), 1x4096x4096 in 6.0, of which
// 3 are the launch's.
// SQ: B's scales are of squares, one for the workgroup's columns.
template <int NT, bool SQ, int FA, int FB>
__global__ __launch_bounds__(64 * kFewWaves) void q8_few(Q8MatArgs a) {
    constexpr int U = 2, SB = SQ ? 1 : 4 * NT;
    __shared__ float red[kFewWaves * 256];
    const int lane = threadIdx.x & 63, li = lane & 15, lg = lane >> 4, nw = blockDim.x >> 6;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n0 = blockIdx.x * 16 * NT, m0 = blockIdx.y * 16;
    const int m = min(m0 + li, a.M - 1);
    const uint8_t *const pa = a.a.data + int64_t(m) * a.a.ld + 32 * lg;
    const uint8_t *pb[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) pb[j] = a.b.data + int64_t(min(n0 + 16 * j + li, a.N - 1)) * a.b.ld + 32 * lg;
    const int64_t sa = int64_t(m >> a.a.shift) * a.a.sld;
    auto sb = [&](int i) {
        return int64_t(min(n0 + (SQ ? 0 : 16 * (i / 4) + 4 * lg + i % 4), a.N - 1) >> a.b.shift) * a.b.sld;
    };

    floatx4 acc[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[j] = floatx4{0, 0, 0, 0};
    // a wave's run of steps in whole fours, whose scales are read together
    const int z = blockIdx.z, kz = min(a.nkt, (z + 1) * a.kps);
    const int per = ((a.kps + nw - 1) / nw + 3) & ~3, k0 = z * a.kps + w * per, k1 = min(kz, k0 + per);
    auto add = [&](intx8 va, const intx8 (&vb)[NT], float s, auto t) {
        bf16x8 da[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) da[i] = to_bf16<FA>(va[2 * i], va[2 * i + 1]);
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const floatx4 p = dot128<FB>(da, vb[j]);
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[j][i] = fmaf(p[i], s * t(SQ ? 0 : 4 * j + i), acc[j][i]);
        }
    };
    int kt = k0;
#pragma unroll 1
    for (; kt + 4 <= k1 && (kt + 4) * kQ8Block <= a.K; kt += 4) {
        const floatx4 s = scales4(a.a.scale, a.a.stype, sa + kt);
        floatx4 t[SB];
#pragma unroll
        for (int i = 0; i < SB; ++i) t[i] = scales4(a.b.scale, a.b.stype, sb(i) + kt);
#pragma unroll
        for (int h = 0; h < 4; h += U) {
            intx8 va[U], vb[U][NT];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t k = int64_t(kt + h + u) * kQ8Block;
#pragma unroll
                for (int j = 0; j < NT; ++j) vb[u][j] = whole32(pb[j] + k);
                va[u] = whole32(pa + k);
            }
            // every load is under way before the first value is used: the compiler would wait for the
            // scales first (16x16384x8192 with 1x128 scales 43 -> 33 us)
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int u = 0; u < U; ++u) add(va[u], vb[u], s[h + u], [&](int i) { return t[i][h + u]; });
        }
    }
#pragma unroll 1
    for (; kt < k1; ++kt) {                                // the last steps, which may reach past K
        const int k = kt * kQ8Block, n = a.K - k - 32 * lg;
        intx8 vb[NT];
#pragma unroll
        for (int j = 0; j < NT; ++j) vb[j] = first32(pb[j] + k, n);
        float t[SB];
#pragma unroll
        for (int i = 0; i < SB; ++i) t[i] = scale_at(a.b.scale, a.b.stype, sb(i) + kt);
        add(first32(pa + k, n), vb, scale_at(a.a.scale, a.a.stype, sa + kt), [&](int i) { return t[i]; });
    }
    // the waves' sums, in their order, 16 columns at a time
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        if (j) __syncthreads();
        *reinterpret_cast<floatx4 *>(red + (w * 16 + li) * 16 + 4 * lg) = acc[j];
        __syncthreads();
        for (int e = threadIdx.x; e < 256; e += blockDim.x) {
            float v = 0.f;
#pragma unroll
            for (int i = 0; i < kFewWaves; ++i) v += i < nw ? red[i * 256 + e] : 0.f;
            const int r = m0 + e / 16, c = n0 + 16 * j + e % 16;
            if (r >= a.M || c >= a.N) continue;
            if (a.part) a.part[(int64_t(z) * a.M + r) * a.N + c] = v;
            else store_c(a.c, a.type, int64_t(r) * a.ldc + c, v);
        }
    }
}

// ---- tiles -----------------------------------------------------------------------

#define DS_GLOBAL(p) ((const __attribute__((address_space(1))) void *)(p))
#define DS_LOCAL(p) ((__attribute__((address_space(3))) void *)(p))

// Waits for all but the wave's newest N copies and for its LDS accesses, then for the workgroup.
template <int N>
__device__ __forceinline__ void stage_barrier() {
    __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | (N >> 4 << 14));   // vmcnt(N)
    __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0)
    __asm__ volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    __asm__ volatile("" ::: "memory");
}

// A buffer descriptor of n bytes from p on: loads past them give zeros.
__device__ __forceinline__ intx4 buffer_of(const uint8_t *p, unsigned n) {
    const uint64_t u = reinterpret_cast<uint64_t>(p);
    return intx4{int(unsigned(u)), int(unsigned(u >> 32) & 0xffffu), int(n), 0x00020000};
}

// Copies 16 bytes a lane from d at off to LDS at dst + 16 lane.  The compiler does not see
// an LDS write here that later reads would have to wait for: stage_barrier's wait and the
// memory clobbers order the two.  One instruction has to lie between a write of m0, where dst is
// taken from, and the copy: the compiler, which writes m0 before, puts none in front of a statement.
__device__ __forceinline__ void copy16(intx4 d, unsigned off, unsigned dst) {
    __asm__ volatile("s_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds"
                     :: "v"(off), "s"(d), "{m0}"(dst) : "memory");
}

// The same for four bytes a lane.
__device__ __forceinline__ void copy4(intx4 d, unsigned off, unsigned dst) {
    __asm__ volatile("s_nop 0\n\tbuffer_load_dword %0, %1, 0 offen lds"
                     :: "v"(off), "s"(d), "{m0}"(dst) : "memory");
}

// How a tile's products are formed.
enum {
    MM_POW2 = 0,   // scaled 8-bit instructions, power-of-two scales in the instruction
    MM_F32 = 1,    // 8-bit instructions block by block, each block's sum times fp32 scales
    // the same through bf16 instructions on the decoded values, whose sums are exact to fp32
    MM_EXACT_POW2 = 2,
    MM_EXACT_F32 = 3
};
constexpr bool mm_exact(int mode) { return mode >= MM_EXACT_POW2; }
constexpr bool mm_words(int mode) { return mode == MM_POW2 || mode == MM_EXACT_POW2; }

// 32 FM x 32 FN of C a workgroup of four waves, 16 FM x 16 FN a wave.
template <int FM, int FN, int MODE>
struct MmShape {
    static constexpr int BM = 32 * FM, BN = 32 * FN, ROWS = BM + BN;
    static constexpr int STAGE = ROWS * kQ8Block;          // bytes of one 128-long step
    // the scales of four steps: a word of exponents or four fp32 numbers a row
    static constexpr int SCALES = ROWS * (mm_words(MODE) ? 4 : 16);
    static constexpr int LDS = 2 * STAGE + 2 * SCALES;
};

// C = sum over steps of 128 of (A's scales x B's scales) * (A's bytes B's bytes^T), in a tile of C that
// stays in registers.  Bound by the matrix instructions: a step of a 256 x 256 tile is 16.8 MFLOP for
// 64 KB, more than the caches' rate asks for.  Operands go from memory to LDS without registers, in
// two stages, each step's copies issued a step and a half before their use, in two parts, as
// each half of a stage has been read; fragments are read from LDS between the products of the
// quarter before.  8192x16384x8192 to bf16: 810 us (2.7 PFLOP/s; the instructions alone, on random
// bytes in registers, reach 3.2 to 4.2 at the clock that the power leaves them).  Exact to fp32:
// 4096x8192x8192 475 us (1.2 PFLOP/s; bf16 instructions alone 2.0 to 2.2, and each byte is first decoded).
// SQ: B's scales are of squares, one for all columns of a wave.  A tile of 256 columns or rows leaves
// one wave a SIMD unit; the smaller ones two.
template <int FM, int FN, int MODE, bool SQ, int FA, int FB>
__global__ __launch_bounds__(256, FM * FN > 16 ? 1 : 2) void q8_mm(Q8MatArgs a) {
    using S = MmShape<FM, FN, MODE>;
    constexpr bool EXACT = mm_exact(MODE), WORDS = mm_words(MODE);
    constexpr int BM = S::BM, BN = S::BN, ROWS = S::ROWS, STAGE = S::STAGE, HM = FM / 2, HN = FN / 2;
    constexpr int LA = BM / 32, LB = BN / 32;              // copies a thread makes of either operand
    extern __shared__ __align__(16) uint8_t smem[];

    const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, lg = lane >> 4;
    const int wid = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wid >> 1, wn = wid & 1;
    // (quotients of scalars come out of the vector unit)
    const auto scalar = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
    int t = xcd_tile(blockIdx.x, gridDim.x);
    const int tiles = a.tiles_m * a.tiles_n, z = scalar(t / tiles);
    t -= z * tiles;
    const int per = a.group * a.tiles_n, g = scalar(t / per), first = g * a.group;
    const int gm = min(a.tiles_m - first, a.group), r = t - g * per, rn = scalar(r / gm);
    const int m0 = (first + r - rn * gm) * BM, n0 = rn * BN;
    const int kt0 = z * a.kps, kt1 = min(a.nkt, kt0 + a.kps);
    const int last = a.K % kQ8Block ? a.nkt - 1 : INT_MAX; // the step that reaches past K, if any

    // A wave's copy j brings rows 32 j + 8 wid .. + 7 of the stage: lane l the 16 bytes at slot
    // l % 8 of row l / 8.  Slot s of row r holds bytes 16 (s ^ (r / 2) % 8) .. + 15 of the step, so that
    // 16 lanes that read one column of 16 rows use each of the 64 banks once.  Rows past the
    // matrix are past the descriptor's end and arrive as zeros.
    const int cr = 8 * wid + (lane >> 3), ck = 16 * ((lane & 7) ^ ((cr >> 1) & 7));
    const unsigned oa = unsigned(cr) * unsigned(a.a.ld) + ck, ob = unsigned(cr) * unsigned(a.b.ld) + ck;
    const uint8_t *const pa = a.a.data + int64_t(m0) * a.a.ld, *const pb = a.b.data + int64_t(n0) * a.b.ld;
    const unsigned na = unsigned(min(BM, a.M - m0) - 1) * unsigned(a.a.ld) + kQ8Block;
    const unsigned nb = unsigned(min(BN, a.N - n0) - 1) * unsigned(a.b.ld) + kQ8Block;
    const unsigned lds0 = unsigned(uintptr_t(DS_LOCAL(smem))) + wid * 1024;

    // One of a step's copies, given its operands' descriptors.  MM_EXACT_POW2, whose two bodies leave the
    // fewest registers, forms an offset where it is used; the compiler would keep one for each copy.
    auto copy1 = [&](intx4 da, intx4 db, unsigned st, int j) {
        unsigned o = j < LA ? oa : ob, ld = unsigned(j < LA ? a.a.ld : a.b.ld);
        if constexpr (MODE == MM_EXACT_POW2) __asm__ volatile("" : "+v"(o), "+s"(ld));
        copy16(j < LA ? da : db, o + 32 * (j < LA ? j : j - LA) * ld, lds0 + st + j * 4096);
    };
    // Of the step that reaches past K, rows end with the 16 bytes that hold their last value; a step past
    // the run has no bytes, and its copies read nothing.
    auto desc = [&](const uint8_t *p, unsigned n, int kt) {
        const unsigned cut = unsigned(kQ8Block - min(kQ8Block, a.K - kt * kQ8Block)) & ~15u;
        return buffer_of(p + int64_t(kt) * kQ8Block, kt < kt1 ? n - cut : 0u);
    };
    // A step's copies in two parts: what the waves' first halves of rows and columns need, and the rest.
    constexpr int PART = (LA + LB) / 2;
    static_assert(PART % 2 == 0);
    auto part_copy = [](int r, int hi) {                   // copy r of a part
        const int h = r < LA / 2 ? HM / 2 : HN / 2, x = r < LA / 2 ? r : r - LA / 2;
        return (r < LA / 2 ? 0 : LA) + x / h * 2 * h + x % h + hi * h;
    };
    auto copy_all = [&](int kt, unsigned st) {
        const intx4 da = desc(pa, na, kt), db = desc(pb, nb, kt);
#pragma unroll
        for (int j = 0; j < 2 * PART; ++j) copy1(da, db, st, part_copy(j % PART, j / PART));
    };
    // Step kt, copied to stage st, waits for its copies if it reaches past K, and each lane clears what lies
    // past K in what it copied itself: none waits for another, and no branch divides a wave.
    auto clear_past = [&](int kt, unsigned st) {
        if (kt != last) return;
        __builtin_amdgcn_s_waitcnt(0x0F70);                // vmcnt(0)
        __asm__ volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        const intx4 keep = mask16(a.K - kt * kQ8Block - ck);
#pragma unroll 1
        for (int j = 0; j < 2 * PART; ++j)
            *reinterpret_cast<intx4 *>(smem + st + wid * 1024 + j * 4096 + lane * 16) &= keep;
    };

    // Fragment f of an operand: lane l holds bytes 32 (l / 16) .. + 31 of row 16 f + l % 16, in halves.
    const int slot = 16 * ((2 * lg) ^ (li >> 1));
    const int fa0 = (16 * FM * wm + li) * kQ8Block + slot, fb0 = (BM + 16 * FN * wn + li) * kQ8Block + slot;
    auto half = [&](unsigned st, int at, int f, int h) {
        return *reinterpret_cast<const intx4 *>(smem + st + (h ? at ^ 16 : at) + f * 16 * kQ8Block);
    };
    struct Frag {
        intx4 h[2];
        __device__ operator intx8() const {
            return __builtin_shufflevector(h[0], h[1], 0, 1, 2, 3, 4, 5, 6, 7);
        }
    };

    // Scales go through LDS four steps at a time: a word of four exponents a row, or four planes of
    // fp32 numbers; a wave copies those of 64 rows at once.
    uint8_t *const sbuf = smem + 2 * STAGE;
    constexpr int ES = WORDS ? 1 : 4;           // bytes of a scale
    auto copy_scales = [&](int kt, int s) {
        if (kt >= a.nkt) return;
        int ln = lane;
        __asm__ volatile("" : "+v"(ln));                   // addresses are formed here, not kept through all steps
#pragma unroll
        for (int i = 0; i < (ROWS / 64 + 3) / 4; ++i) {
            const int r0 = 64 * (4 * i + wid);             // rows of the stage, all of A or all of B
            if (r0 >= ROWS) break;
            const bool isa = r0 < BM;
            const Q8View &v = isa ? a.a : a.b;
            const int o0 = isa ? m0 : n0, left = (isa ? a.M : a.N) - o0, row = (isa ? r0 : r0 - BM) + ln;
            const int s0 = o0 >> v.shift;                  // scale rows from here on
            const unsigned sld = unsigned(v.sld) * ES;
            const int64_t at = int64_t(s0) * sld + int64_t(kt) * ES;
            const unsigned end = unsigned(((o0 + min(isa ? BM : BN, left) - 1) >> v.shift) - s0) * sld +
                                 (!WORDS ? unsigned(a.nkt - kt) * 4u
                                         : a.words ? (unsigned(a.nkt - kt) + 3u) & ~3u : unsigned(a.nkt - kt));
            uint8_t *const p = static_cast<uint8_t *>(v.scale) + at;
            const unsigned off = unsigned(((o0 + row) >> v.shift) - s0) * sld;
            uint8_t *const dst = sbuf + s * S::SCALES + 4 * r0;
            if (WORDS && !a.words) {             // not in whole words: byte by byte
                const auto d = __builtin_amdgcn_make_buffer_rsrc(p, 0, int(end), 0x00020000);
                int w = 0;
#pragma unroll 1
                for (int k = 0; k < 4; ++k)
                    w |= int(__builtin_amdgcn_raw_buffer_load_b8(d, int(off) + k, 0, 0)) << (8 * k);
                *reinterpret_cast<int *>(dst + 4 * ln) = w;
                continue;
            }
            const intx4 d = buffer_of(p, end);
            const unsigned to = unsigned(uintptr_t(DS_LOCAL(dst)));
#pragma unroll
            for (int k = 0; k < (WORDS ? 1 : 4); ++k) copy4(d, off + 4 * k, to + 4 * k * ROWS);
        }
    };

    // whether an exponent of the thread's row of the stage is over 167, the byte of 2^40
    auto scales_past_2_40 = [&]() {
        static_assert(ROWS == 256 || MODE != MM_EXACT_POW2, "a row a thread");
        const bool isa = tid < BM;
        const Q8View &v = isa ? a.a : a.b;
        const int row = isa ? min(m0 + tid, a.M - 1) : min(n0 + tid - BM, a.N - 1);
        const uint8_t *const p = static_cast<const uint8_t *>(v.scale) + int64_t(row >> v.shift) * v.sld;
        unsigned bad = 0;
        int k = kt0;
        if (a.words)
#pragma unroll 4
            for (; k + 4 <= kt1; k += 4) {
                const unsigned w = *reinterpret_cast<const unsigned *>(p + k);
                bad |= ((w & 0x7f7f7f7fu) + 0x58585858u) & w & 0x80808080u;   // 168 = 128 + 40
            }
#pragma unroll 1
        for (; k < kt1; ++k) bad |= p[k] > 167;
        return int(bad != 0);
    };

    floatx4 acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = floatx4{0, 0, 0, 0};
    Frag alo[HM], ahi[HM], b0[HN], b1[HN];
    // The present step's scales: of A's rows and of B's columns.  MM_POW2: exponents in the low
    // bytes, xn the words of the step after as read.  Otherwise fp32.
    constexpr int XN = FM + (WORDS ? FN : 0);
    int xs[XN], xn[MODE == MM_POW2 ? XN : 1];
    floatx4 sb[WORDS || SQ ? 1 : FN];
    float sq = 0.f, sqn = 0.f;
    auto scales_of = [&](int u) {
        return reinterpret_cast<const int *>(sbuf + ((u >> 2) & 1) * S::SCALES) + (WORDS ? 0 : (u & 3) * ROWS);
    };
    auto word_of = [&](const int *sc, int f) {             // of fragment f, B's after A's
        return f < FM ? sc[16 * (FM * wm + f) + li] : sc[BM + 16 * (FN * wn + f - FM) + li];
    };
    // as fp32 bits; sh: the step's byte of the word
    auto value = [](int v, int sh) { return WORDS ? int(max((unsigned(v) >> sh & 255u) << 23, 0x400000u)) : v; };
    auto scale_of_a = [&](const int *sc, int f, int sh) { return value(sc[16 * (FM * wm + f) + li], sh); };
    auto scale_of_b = [&](const int *sc, int f, int sh) {
        const intx4 v = *reinterpret_cast<const intx4 *>(sc + BM + 16 * (FN * wn + f) + 4 * lg);
        return floatx4{__int_as_float(value(v[0], sh)), __int_as_float(value(v[1], sh)),
                       __int_as_float(value(v[2], sh)), __int_as_float(value(v[3], sh))};
    };
    auto scale_of_square = [&](const int *sc, int sh) {
        return __int_as_float(value(sc[BM + 16 * FN * wn], sh));
    };

    // FOLD: the scales go into the decoded operands.  LATE: sums of blocks wait for D more to be issued
    // before they are scaled and added.
    constexpr bool FOLD = MODE == MM_EXACT_POW2, LATE = !WORDS;
    constexpr int NQ = HM * HN, D = EXACT ? 1 : 2;
    floatx4 wp[D], ws[D];
#pragma unroll
    for (int d = 0; d < D; ++d) wp[d] = ws[d] = floatx4{0, 0, 0, 0};
    auto add_block = [&](int i, int j, floatx4 p, floatx4 w) {
#pragma unroll
        for (int v = 0; v < 4; ++v) acc[i][j][v] = fmaf(p[v], SQ ? w[0] : w[v], acc[i][j][v]);
    };
    // place of a quarter's q-th product; EXACT: down a column, so that B's next fragment is decoded late
    auto qi = [](int q) { return EXACT ? q % HM : q / HN; };
    auto qj = [](int q) { return EXACT ? q / HM : q % HN; };
    bf16x8 da[EXACT ? HM : 1][4], db[EXACT ? FN : 1][4];   // EXACT: decoded fragments, once a step
    // A quarter of the wave's tile, fragments i0 .. of A by j0 .. of B; beside(q) issues what goes
    // between its products q and q + 1.  wi, wj: the quarter before.
    auto quarter = [&]<int U4>(std::integral_constant<int, U4>, const Frag (&fa)[HM], const Frag (&fb)[HN], int i0,
                               int j0, auto beside, int wi, int wj) {
        if constexpr (EXACT)
            if (j0 == 0)
#pragma unroll
                for (int i = 0; i < HM; ++i)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        da[i][k] = to_bf16<FA>(fa[i].h[k >> 1][2 * (k & 1)], fa[i].h[k >> 1][2 * (k & 1) + 1],
                                               FOLD ? __int_as_float(xs[i0 + i]) : 1.f);
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
            const int i = qi(q), j = qj(q);
            if constexpr (MODE == MM_POW2) {
                acc[i0 + i][j0 + j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
                    fb[j], fa[i], acc[i0 + i][j0 + j], FB, FA, U4 > 0 ? U4 : 0,
                    xs[FM + j0 + j], U4 > 0 ? U4 : 0, xs[i0 + i]);
            } else {
                floatx4 p = {0, 0, 0, 0};
                if constexpr (EXACT) {
                    if (i == 0 && i0 == 0)
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            db[j0 + j][k] = to_bf16<FB>(fb[j].h[k >> 1][2 * (k & 1)],
                                                        fb[j].h[k >> 1][2 * (k & 1) + 1],
                                                        FOLD ? __int_as_float(xs[FM + j0 + j]) : 1.f);
                    if constexpr (FOLD) p = acc[i0 + i][j0 + j];
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(db[j0 + j][k], da[i][k], p, 0, 0, 0);
                } else {
                    p = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb[j], fa[i], p, FB, FA, 0, 0, 0, 0);
                }
                if constexpr (FOLD) {
                    acc[i0 + i][j0 + j] = p;
                } else {
                    const int o = q < D ? NQ - D + q : q - D;  // place of the block that is due
                    add_block((q < D ? wi : i0) + qi(o), (q < D ? wj : j0) + qj(o), wp[0], ws[0]);
                    if constexpr (D == 2) {
                        wp[0] = wp[D - 1];
                        ws[0] = ws[D - 1];
                    }
                    wp[D - 1] = p;
                    const float x = __int_as_float(xs[i0 + i]);
                    if constexpr (SQ) ws[D - 1][0] = x * sq;
                    else ws[D - 1] = x * sb[j0 + j];
                }
            }
            beside(q);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // Step kt, whose first fragments are in alo and b0; step kt + 2 is copied.
    // U4: its place among the four steps of a word of scales, -1 if that is not a constant (MM_POW2:
    // a constant picks the word's byte in the instruction, else words are read and shifted each step).
    auto step = [&]<int U4>(std::integral_constant<int, U4> u4, int kt) {
        const int u = kt - kt0;
        const unsigned cur = (u & 1) * STAGE, nxt = STAGE - cur;
        if (U4 < 0 ? (u & 3) == 0 : U4 == 0) copy_scales(kt + 4, ((u >> 2) & 1) ^ 1);
        __builtin_amdgcn_sched_barrier(0);
        // n parts spread over a quarter's first products, at most two after each
        auto spread = [](int q, int n, auto part) {
            const int each = 2 * NQ < n ? (n + NQ - 1) / NQ : n > NQ ? 2 : 1;
#pragma unroll
            for (int r = q * each; r < (q + 1) * each; ++r)
                if (r < n) part(r);
        };
        // A part is copied a step and a half before it is needed: the two parts copied since may be
        // on their way (the scales' copies among them only make a wait longer).
        constexpr int LEFT = 2 * PART;
        const intx4 da = desc(pa, na, kt + 2), db = desc(pb, nb, kt + 2);
        const int *const sc = scales_of(u), *const scn = scales_of(u + 1);
        const int sh = 8 * (u & 3), shn = 8 * ((u + 1) & 3);
        // Each half of the fragments and scales is replaced once its last product is issued
        quarter(u4, alo, b0, 0, 0, [&](int q) {
            spread(q, 2 * HN, [&](int r) { b1[r >> 1].h[r & 1] = half(cur, fb0, HN + (r >> 1), r & 1); });
            spread(q, PART, [&](int r) { copy1(da, db, cur, part_copy(r, 0)); });
            if constexpr (U4 == 0) {
                spread(q, HN, [&](int f) { xs[FM + HN + f] = word_of(sc, FM + HN + f); });
                spread(q, HM, [&](int f) { xs[HM + f] = word_of(sc, HM + f); });
            } else if constexpr (U4 > 0) {
            } else if constexpr (MODE == MM_POW2) {
                spread(q, HM, [&](int f) { xs[HM + f] = int(unsigned(xn[HM + f]) >> sh); });
                spread(q, HN, [&](int f) { xs[FM + HN + f] = int(unsigned(xn[FM + HN + f]) >> sh); });
            } else {
                if constexpr (FOLD) spread(q, HN, [&](int f) { xs[FM + HN + f] = value(word_of(sc, FM + HN + f), sh); });
                else if constexpr (!SQ) spread(q, HN, [&](int f) { sb[HN + f] = scale_of_b(sc, HN + f, sh); });
                spread(q, HM, [&](int f) { xs[HM + f] = scale_of_a(sc, HM + f, sh); });
            }
        }, HM, HN);
        quarter(u4, alo, b1, 0, HN, [&](int q) {
            spread(q, 2 * HM, [&](int r) { ahi[r >> 1].h[r & 1] = half(cur, fa0, HM + (r >> 1), r & 1); });
            if constexpr (MODE == MM_POW2 && U4 < 0) spread(q, XN, [&](int f) { xn[f] = word_of(scn, f); });
        }, 0, 0);
        // Every wave has read the second part of this step, which is copied over now, and the first
        // part of the next has arrived.
        stage_barrier<LEFT>();
        quarter(u4, ahi, b0, HM, 0, [&](int q) {
            spread(q, PART, [&](int r) { copy1(da, db, cur, part_copy(r, 1)); });
            spread(q, 2 * HM, [&](int r) { alo[r >> 1].h[r & 1] = half(nxt, fa0, r >> 1, r & 1); });
            if constexpr (U4 == 3) spread(q, HM, [&](int f) { xs[f] = word_of(scn, f); });
            if constexpr (MODE != MM_POW2) {
                spread(q, HM, [&](int f) { xs[f] = scale_of_a(scn, f, shn); });
                if (SQ && q == 0) sqn = scale_of_square(scn, shn);
            }
        }, 0, HN);
        quarter(u4, ahi, b1, HM, HN, [&](int q) {
            spread(q, 2 * HN, [&](int r) { b0[r >> 1].h[r & 1] = half(nxt, fb0, r >> 1, r & 1); });
            if constexpr (U4 >= 0) {
                if constexpr (U4 == 3) spread(q, HN, [&](int f) { xs[FM + f] = word_of(scn, FM + f); });
            } else if constexpr (MODE == MM_POW2) {
                spread(q, HM, [&](int f) { xs[f] = int(unsigned(xn[f]) >> shn); });
                spread(q, HN, [&](int f) { xs[FM + f] = int(unsigned(xn[FM + f]) >> shn); });
            } else if constexpr (FOLD) {
                spread(q, HN, [&](int f) { xs[FM + f] = value(word_of(scn, FM + f), shn); });
            } else if constexpr (!SQ) {
                spread(q, HN, [&](int f) { sb[f] = scale_of_b(scn, f, shn); });
            }
        }, HM, 0);
        if constexpr (SQ) sq = sqn;
        // likewise the first part of the next step, and the second has arrived
        stage_barrier<LEFT>();
    };

    auto run = [&] {
#pragma unroll
        for (int f = 0; f < HM; ++f)
#pragma unroll
            for (int h = 0; h < 2; ++h) alo[f].h[h] = half(0, fa0, f, h);
#pragma unroll
        for (int f = 0; f < HN; ++f)
#pragma unroll
            for (int h = 0; h < 2; ++h) b0[f].h[h] = half(0, fb0, f, h);
        const int *const sc = scales_of(0);
        if constexpr (MODE == MM_POW2) {
#pragma unroll
            for (int f = 0; f < XN; ++f) xs[f] = xn[f] = word_of(sc, f);
        } else {
#pragma unroll
            for (int f = 0; f < FM; ++f) xs[f] = scale_of_a(sc, f, 0);
            if constexpr (FOLD) {
#pragma unroll
                for (int f = FM; f < XN; ++f) xs[f] = value(word_of(sc, f), 0);
            } else if constexpr (SQ) {
                sq = scale_of_square(sc, 0);
            } else {
#pragma unroll
                for (int f = 0; f < FN; ++f) sb[f] = scale_of_b(sc, f, 0);
            }
        }
        int kt = kt0;
        const std::integral_constant<int, -1> any;
        // (in larger tiles four steps in one are more than the register allocator keeps in place)
        if constexpr (MODE == MM_POW2 && FM * FN <= 16) {
#pragma unroll 1
            for (; kt + 4 <= kt1 && kt + 4 < last; kt += 4) {
                step(std::integral_constant<int, 0>{}, kt);
                step(std::integral_constant<int, 1>{}, kt + 1);
                step(std::integral_constant<int, 2>{}, kt + 2);
                step(std::integral_constant<int, 3>{}, kt + 3);
            }
            const int *const next = scales_of(kt - kt0);
#pragma unroll
            for (int f = 0; f < XN; ++f) xn[f] = word_of(next, f);
        }
#pragma unroll 1
        for (; kt < kt1; ++kt) {
            clear_past(kt + 1, ((kt - kt0) & 1 ^ 1) * STAGE);
            step(any, kt);
        }
        // the last step read ahead into a stage of a step past the run; its values are unused
        if constexpr (LATE)
#pragma unroll
            for (int d = 0; d < D; ++d) add_block(HM + qi(NQ - D + d), HN + qj(NQ - D + d), wp[d], ws[d]);
    };
    // MM_EXACT_POW2 with larger scales than fit the decoded operands, which no layer's values have: each
    // step's sums are scaled, nothing overlaps, and fragments are read where they are used.
    auto run_unfolded = [&] {
#pragma unroll 1
        for (int kt = kt0; kt < kt1; ++kt) {
            const int u = kt - kt0, sh = 8 * (u & 3);
            const unsigned cur = (u & 1) * STAGE;
            const int *const sc = scales_of(u);
            if ((u & 3) == 0) copy_scales(kt + 4, ((u >> 2) & 1) ^ 1);
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                bf16x8 ea[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const intx4 v = half(cur, fa0, i, k >> 1);
                    ea[k] = to_bf16<FA>(v[2 * (k & 1)], v[2 * (k & 1) + 1]);
                }
                const float x = __int_as_float(scale_of_a(sc, i, sh));
#pragma unroll
                for (int j = 0; j < FN; ++j) {
                    floatx4 p = {0, 0, 0, 0};
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const intx4 v = half(cur, fb0, j, k >> 1);
                        p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(to_bf16<FB>(v[2 * (k & 1)], v[2 * (k & 1) + 1]),
                                                                    ea[k], p, 0, 0, 0);
                    }
                    const floatx4 w = x * scale_of_b(sc, j, sh);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(p[e], w[e], acc[i][j][e]);
                    __asm__ volatile("" ::: "memory");     // (kept from one i to the next they would not fit)
                }
            }
            clear_past(kt + 1, STAGE - cur);
            stage_barrier<0>();                            // step kt is read, step kt + 1 has arrived
            copy_all(kt + 2, cur);
        }
    };
    if (kt0 < kt1) {
        copy_scales(kt0, 0);
        copy_all(kt0, 0);
        copy_all(kt0 + 1, STAGE);
        // MM_EXACT_POW2: scales of at most 2^40 go into the decoded operands, which then meet neither
        // the largest bf16 number nor, while the values that they stand for are normal fp32 numbers,
        // the smallest; the sums need no scaling any more (4096x8192x8192, both operands 1x128: 455 us, and 505
        // with fp32 scales, whose sums do).
        bool small = true;
        if constexpr (MODE == MM_EXACT_POW2) small = !__syncthreads_or(scales_past_2_40());
        clear_past(kt0, 0);
        stage_barrier<2 * PART>();
        if (small) run();
        else run_unfolded();
        stage_barrier<0>();                                // of the copies for steps past the run
    }

    // Lane l holds columns 4 (l / 16) .. + 3 of row l % 16 of each 16 x 16 block.  Rows of blocks go
    // through the wave's part of LDS (free since the last barrier), so that 16 bytes a lane and whole
    // lines are stored: straight from the registers a store covers 32 bytes of 16 rows each, and
    // 8192x8192x8192 took 414 us in place of 392.
    void *const out = a.part ? a.part + int64_t(z) * a.M * a.N : a.c;
    const int type = a.part ? DS_TYPE_F32 : a.type, vec = a.part ? a.pvec : a.cvec;
    const int64_t ldc = a.part ? a.N : a.ldc;
    const int rm = m0 + 16 * FM * wm, cn = n0 + 16 * FN * wn;
    if (vec && m0 + BM <= a.M && n0 + BN <= a.N) {
        auto whole = [&](auto *c, auto conv) {
            using T = std::remove_pointer_t<decltype(c)>;
            constexpr int RB = 16 * FN * sizeof(T), ROW = RB + 16;   // bytes of a row, with room between
            constexpr int LR = RB / 16, RI = 64 / LR;                // lanes a row, rows a store
            static_assert(4 * 2 * 16 * ROW <= S::LDS, "two rows of blocks of every wave");
            uint8_t *const own = smem + wid * 2 * 16 * ROW;
            const int lr = lane / LR, lc = lane % LR;
            c += (rm + lr) * ldc + cn + lc * int(16 / sizeof(T));
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                uint8_t *const st = own + (i & 1) * 16 * ROW;
#pragma unroll
                for (int j = 0; j < FN; ++j)
                    *reinterpret_cast<decltype(conv(acc[0][0])) *>(st + li * ROW + (16 * j + 4 * lg) * sizeof(T)) =
                        conv(acc[i][j]);
                __builtin_amdgcn_wave_barrier();
#pragma unroll
                for (int r = 0; r < 16; r += RI)
                    *reinterpret_cast<intx4 *>(c + (16 * i + r) * ldc) =
                        *reinterpret_cast<const intx4 *>(st + (r + lr) * ROW + 16 * lc);
                __builtin_amdgcn_wave_barrier();
            }
        };
        if (type == DS_TYPE_BF16)
            whole(static_cast<__bf16 *>(out), [](floatx4 v) {
                return bf16x4{__bf16(v[0]), __bf16(v[1]), __bf16(v[2]), __bf16(v[3])};
            });
        else if (type == DS_TYPE_F16)
            whole(static_cast<_Float16 *>(out), [](floatx4 v) {
                return f16x4{_Float16(v[0]), _Float16(v[1]), _Float16(v[2]), _Float16(v[3])};
            });
        else
            whole(static_cast<float *>(out), [](floatx4 v) { return v; });
        return;
    }
    // Edges and rows that are not 16-byte aligned: through the wave's part of LDS (free since the last
    // barrier), a lane a column.  One copy of the loop: straight-line it would outgrow the
    // instruction cache.
    constexpr int ROW = 16 * FN + 4;                       // floats; 16 bytes aside from bank to bank
    static_assert(4 * 16 * ROW * 4 <= S::LDS, "a row of blocks of every wave");
    float *const own = reinterpret_cast<float *>(smem) + wid * 16 * ROW;
#pragma unroll 1
    for (int i = 0; i < FM; ++i) {
#pragma unroll
        for (int k = 0; k < FM; ++k)
            if (i == k)
#pragma unroll
                for (int j = 0; j < FN; ++j)
                    *reinterpret_cast<floatx4 *>(own + li * ROW + 16 * j + 4 * lg) = acc[k][j];
        __builtin_amdgcn_wave_barrier();
        const int rows = min(16, a.M - rm - 16 * i), cols = min(16 * FN, a.N - cn);
        auto edge = [&](auto *c) {
            using T = std::remove_pointer_t<decltype(c)>;
            c += (rm + 16 * i) * ldc + cn;
#pragma unroll 4
            for (int r = 0; r < rows; ++r)
#pragma unroll
                for (int x = 0; x < FN / 4; ++x)
                    if (64 * x + lane < cols) c[r * ldc + 64 * x + lane] = T(own[r * ROW + 64 * x + lane]);
        };
        if (type == DS_TYPE_BF16) edge(static_cast<__bf16 *>(out));
        else if (type == DS_TYPE_F16) edge(static_cast<_Float16 *>(out));
        else edge(static_cast<float *>(out));
        __builtin_amdgcn_wave_barrier();
    }
}

// C from the partial sums of ks splits, in their order: the same bits at every call, where atomics would
// give others.  Bound by the launch (3 us) and the sums' reading, from the cache mostly.
__global__ __launch_bounds__(256) void q8_join(Q8MatArgs a) {
    const int per = (a.N + 3) / 4;
    const int64_t total = int64_t(a.M) * per, mn = int64_t(a.M) * a.N;
    for (int64_t e = int64_t(blockIdx.x) * 256 + threadIdx.x; e < total; e += int64_t(gridDim.x) * 256) {
        const int row = int(e / per), col = 4 * int(e - int64_t(row) * per);
        const float *p = a.part + int64_t(row) * a.N + col;
        floatx4 v = {0, 0, 0, 0};
        for (int z = 0; z < a.ks; ++z, p += mn) {
            if (a.pvec) {
                v += *reinterpret_cast<const floatx4 *>(p);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (col + i < a.N) v[i] += p[i];
            }
        }
        store4(a.c, a.type, int64_t(row) * a.ldc, col, a.N, a.cvec, v);
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

// Splits the reduction into `ks` runs of a multiple of `unit` steps, whose partial products go to
// the stream's workspace, held until they are joined.
int split(Q8MatArgs &g, int ks, int unit, hipStream_t stream, SplitHold &hold) {
    if (ks <= 1) return DS_OK;
    g.kps = ((g.nkt + ks - 1) / ks + unit - 1) / unit * unit;
    g.ks = (g.nkt + g.kps - 1) / g.kps;
    return g.ks > 1 ? split_workspace(int64_t(g.ks) * g.M * g.N, stream, &g.part, hold) : DS_OK;
}

int join(const Q8MatArgs &g, hipStream_t stream) {
    if (g.ks == 1) return DS_OK;
    const int64_t quads = int64_t(g.M) * ((g.N + 3) / 4);
    q8_join<<<unsigned(std::min<int64_t>((quads + 255) / 256, 4096)), 256, 0, stream>>>(g);
    return hip_ok(hipGetLastError(), "8-bit matmul join") ? DS_OK : DS_EHIP;
}

template <int FM, int FN, int MODE, bool SQ>
int mm_launch(Q8MatArgs &g, hipStream_t stream) {
    using S = MmShape<FM, FN, MODE>;
    g.tiles_m = (g.M + S::BM - 1) / S::BM;
    g.tiles_n = (g.N + S::BN - 1) / S::BN;
    g.group = 4;
    const int64_t grid = int64_t(g.tiles_m) * g.tiles_n * g.ks;
    int rc = launch_check(grid, 256, "ds_q8_matmul");
    if (rc != DS_OK) return rc;
    const int done = by_formats(g.a.fmt, g.b.fmt, [&](auto fa, auto fb) {
        auto *k = &q8_mm<FM, FN, MODE, SQ, fa.value, fb.value>;
        rc = ensure_lds_attr(reinterpret_cast<const void *>(k), S::LDS);
        if (rc == DS_OK) k<<<unsigned(grid), 256, S::LDS, stream>>>(g);
    });
    if (rc != DS_OK || done != DS_OK) return rc != DS_OK ? rc : done;
    return join(g, stream);
}

// SQ: squares, one scale of B for all columns of a wave
template <int FM, int FN, int MODE>
int mm_square(Q8MatArgs &g, hipStream_t stream) {
    return g.b.shift ? mm_launch<FM, FN, MODE, true>(g, stream) : mm_launch<FM, FN, MODE, false>(g, stream);
}

// The split of a reduction over tiles of 128 x 128, by what each took on the chip: a step of 128 about
// `step` us in a workgroup that has its SIMD units to itself, and the join 3 us and the partial sums'
// writing and reading.  33x4096x4096 17.6 -> 12.6 us by eight, 64x16384x8192 32 -> 30 by four;
// 512x4096x4096 would go from 16.6 to 20.5 and stays whole.
int mm_splits(const Q8MatArgs &g, double step) {
    const int64_t tiles = int64_t((g.M + 127) / 128) * ((g.N + 127) / 128);
    const double sums = double(g.M) * g.N * 10 / 4.5e6;
    int best = 1;
    double least = g.nkt * step;
    for (int ks = 2; ks <= 8 && tiles * ks <= 512 && g.nkt >= 4 * ks; ks *= 2) {
        const double t = double(g.nkt) / ks * step + 3 + ks * sums;
        if (t < least) {
            least = t;
            best = ks;
        }
    }
    return best;
}

int mm_tiles(Q8MatArgs &g, bool exact, hipStream_t stream) {
    const bool pow2 = g.a.stype == DS_SCALE_POW2;
    auto tiles = [&](int bm, int bn) { return int64_t((g.M + bm - 1) / bm) * ((g.N + bn - 1) / bn); };
    if (pow2 && !exact) {
        // Rounds of workgroups over 256 CUs times a round's time: a step of 1.31, 0.86, 0.87 us (two
        // workgroups a CU, 0.47 for one) and what comes before and after.  In tiles of 256 x 256, 256 x 128
        // and 128 x 128: 4096x4096x4096 55, 68 and 63 us; 8192x8192x8192 391, 477 and 462; 2048x4096x8192
        // 85, 61 and 61; 1024x4096x4096 46, 30 and 20; 3000x5000x6000 86, 101 and 114; 4096x4096x700 20, 24
        // and 22.  Of the two smaller it is 256 x 128 for reductions from 12700 on: 512x16384x16384 131 and 141.
        const double n = g.nkt;
        const int64_t t = tiles(128, 128);
        const double large = double((tiles(256, 256) + 255) / 256) * (1.31 * n + 12);
        const double tall = double((tiles(256, 128) + 255) / 256) * (0.86 * n + 6);
        const double small = double(t / 512) * (0.87 * n + 5) +
                             (t % 512 > 256 ? 0.87 * n + 5 : t % 512 ? 0.47 * n + 5 : 0);
        if (large <= tall && large <= small) return mm_launch<8, 8, MM_POW2, false>(g, stream);
        if (tall <= small) return mm_launch<8, 4, MM_POW2, false>(g, stream);
    }
    SplitHold hold;
    const int rc = split(g, mm_splits(g, exact ? 1.0 : 0.5), 4, stream, hold);
    if (rc != DS_OK) return rc;
    if (exact) return pow2 ? mm_launch<4, 4, MM_EXACT_POW2, false>(g, stream) : mm_square<4, 4, MM_EXACT_F32>(g, stream);
    return pow2 ? mm_launch<4, 4, MM_POW2, false>(g, stream) : mm_square<4, 4, MM_F32>(g, stream);
}

template <int NT, bool SQ>
int few_launch(Q8MatArgs &g, int waves, hipStream_t stream) {
    const unsigned tn = unsigned((g.N + 16 * NT - 1) / (16 * NT)), tm = unsigned((g.M + 15) / 16);
    int rc = launch_check(tn, 64 * waves, "ds_q8_matmul");
    if (rc != DS_OK) return rc;
    rc = by_formats(g.a.fmt, g.b.fmt, [&](auto fa, auto fb) {
        q8_few<NT, SQ, fa.value, fb.value><<<dim3(tn, tm, unsigned(g.ks)), 64 * waves, 0, stream>>>(g);
    });
    return rc == DS_OK ? join(g, stream) : rc;
}

int few(Q8MatArgs &g, hipStream_t stream) {
    // Few columns under a long reduction leave most CUs idle: it is split over workgroups too
    // (8x512x16384 17.8 -> 10.4 us, 16x2048x8192 12.6 -> 11.5; 16x4096x16384 would go from 25 to 28).
    SplitHold hold;
    if (g.N <= 2048 && g.nkt >= 64) {
        const int rc = split(g, std::min(g.nkt / 16, 8), 4, stream, hold);
        if (rc != DS_OK) return rc;
    }
    // 32 columns a workgroup read A half as often and are enough workgroups in wide layers
    // (16x16384x8192 39 -> 32 us, 16x8192x8192 23.1 -> 21.6; 1x8192x8192 would go from 18.4 to 21.2)
    const bool two = g.N >= 16384 || (g.N >= 8192 && (g.M > 4 || !g.b.shift));
    // at least four steps a wave, and with 32 columns 16 of them
    const int waves = std::clamp((g.kps + 3) / 4, 1, two && g.kps <= 64 ? 4 : kFewWaves);
    if (two) return g.b.shift ? few_launch<2, true>(g, waves, stream) : few_launch<2, false>(g, waves, stream);
    return g.b.shift ? few_launch<1, true>(g, waves, stream) : few_launch<1, false>(g, waves, stream);
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
    const bool exact = (type & DS_EXACT_SUMS) != 0 || type == DS_TYPE_F32;
    type &= ~DS_EXACT_SUMS;
    if ((rc = plain_check(c, type, a->rows, b->rows, ldc, "c")) != DS_OK) return rc;
    if (a->rows == 0 || b->rows == 0) return DS_OK;
    Q8MatArgs g{};
    g.a = q8_view(a);
    g.b = q8_view(b);
    g.c = c;
    g.ldc = ldc;
    g.type = type;
    g.M = int(a->rows);
    g.N = int(b->rows);
    g.K = int(a->cols);
    g.nkt = int(q8_up(a->cols));
    g.ks = 1;
    g.kps = g.nkt;
    g.cvec = reinterpret_cast<uintptr_t>(c) % 16 == 0 && ldc * type_bytes(type) % 16 == 0;
    g.pvec = g.N % 4 == 0;
    auto words = [](const ds_q8 *m) {
        return reinterpret_cast<uintptr_t>(m->scale) % 4 == 0 && m->scale_ld % 4 == 0;
    };
    g.words = words(a) && words(b);
    try {
        // (32 rows of a short reduction too: 32x4096x4096 10.0 us, 33 rows in tiles 12.4)
        return g.M > (g.nkt <= 32 ? 32 : 16) ? mm_tiles(g, exact, stream) : few(g, stream);
    } catch (const std::bad_alloc &) {                     // of the workspaces' table
        set_error("ds_q8_matmul: out of host memory");
        return DS_ENOMEM;
    }
}
