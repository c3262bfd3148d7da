// Attention over the paged 8-bit cache: the launch, and the join of parts.
#include <cmath>

#include "attn8.h"
#include "kern_common.h"
#include "q8.h"

namespace ds {
namespace {

constexpr int kJoinWaves = 4;
constexpr float kLn2 = 0.69314718055994530942f;

// A wave joins the parts of a row: LPR lanes take four values each of every 64 / LPR-th split, four at a
// time (their loads together), and the groups of lanes are added up in order.  One token's 32 rows of 16 splits 4.0
// us, latency; 1024 tokens of 32 heads of 128 in two splits 13.2 us, 44 MB.
template <typename T, int LPR>
__global__ __launch_bounds__(64 * kJoinWaves) void attn8_join(AttnArgs a) {
    const int lane = threadIdx.x & 63;
    const int64_t at = int64_t(blockIdx.x) * kJoinWaves + (threadIdx.x >> 6);
    const int64_t rows = int64_t(a.n.tokens) * a.heads;
    if (at >= rows) return;
    const int t = int(at / a.heads), hd = int(at - int64_t(t) * a.heads);
    float2 ml = make_float2(-INFINITY, 0.f);
    if (lane < a.splits) ml = a.ml[lane * rows + at];
    int b = 0;
    for (int n = a.n.seqs; n > 1;) {
        const int by = (n + 63) / 64;
        const bool ok = lane == 0 || (lane * by < n && a.n.starts[b + lane * by] <= t);
        const int k = 63 - __clzll(__ballot(ok));
        b += k * by;
        n = min(by, n - k * by);
    }
    if (a.n.starts[b] > t || t >= a.n.starts[b + 1]) return;
    float top = ml.x;
#pragma unroll
    for (int x = 32; x > 0; x /= 2) top = fmaxf(top, __shfl_xor(top, x));
    const float by = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - top);
    float l = ml.y * by;
#pragma unroll
    for (int x = 1; x < 64; x *= 2) l += __shfl_xor(l, x);
    constexpr int kGroups = 64 / LPR;
    const int group = lane / LPR, d = 4 * (lane % LPR);
    floatx4 sum = {};
    for (int s0 = 0; s0 < a.splits; s0 += 4 * kGroups) {
        floatx4 x[4];
        float w[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int s = min(s0 + u * kGroups + group, 63);
            w[u] = __shfl(by, s);
            const float ls = __shfl(ml.y, s);              // (of all lanes: none may stay away from a shuffle)
            // a split without a key has left nothing but that
            const bool is = s < a.splits && ls != 0.f && d < a.c.dim;
            x[u] = floatx4{};
            if (is) x[u] = *reinterpret_cast<const floatx4 *>(a.part + (s * rows + at) * a.c.dim + d);
            w[u] = is ? w[u] : 0.f;
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) sum += w[u] * x[u];
    }
#pragma unroll
    for (int x = LPR; x < 64; x *= 2)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] += __shfl_xor(sum[e], x);
    const float inv = l == 0.f ? 0.f : 1.f / l;
    if (a.lse && lane == 0) a.lse[at] = l == 0.f ? -INFINITY : (top + log2f(l)) * kLn2;
    if (group != 0 || d >= a.c.dim) return;
    T *op = static_cast<T *>(a.out) + t * a.ldo + hd * a.hldo + d;
#pragma unroll
    for (int e = 0; e < 4; ++e) op[e] = T(sum[e] * inv);
}

// ---- host ---------------------------------------------------------------------------

struct AttnPlan {
    int form, threads, splits, span;
    int64_t groups, bytes, part;          // part: bytes of the sums, a multiple of 16
};

// q without DS_EXACT_SUMS in its type (null where q is); exact: whether that was there.
const ds_heads *plain_type(const ds_heads *q, ds_heads *of, bool *exact) {
    if (!q) return nullptr;
    *of = *q;
    *exact = (q->type & DS_EXACT_SUMS) != 0;
    of->type &= ~DS_EXACT_SUMS;
    return of;
}

int attn_check(const ds_heads *q, const ds_cache8 *cache, const ds_chunk *chunk, const ds_attn8_cfg *cfg) {
    int rc;
    if ((rc = heads_check(q, "q", false)) != DS_OK || (rc = cache8_check(cache)) != DS_OK ||
        (rc = chunk_check(chunk, cache)) != DS_OK)
        return rc;
    if (q->dim != cache->dim || q->heads % cache->heads != 0) {
        set_error("q has %lld heads of %lld values, the cache %d of %d", (long long)q->heads, (long long)q->dim,
                  cache->heads, cache->dim);
        return DS_EINVAL;
    }
    if (q->type == DS_TYPE_F32 && cache->dim > 128) {
        // (three parts of such queries do not fit the registers beside the sums)
        set_error("fp32 queries of %d values (up to 128; 16-bit ones up to 256)", cache->dim);
        return DS_EUNSUPPORTED;
    }
    if (!cfg || !std::isfinite(cfg->scale) || !std::isfinite(float(cfg->scale * 1.4426950408889634)) ||
        (cfg->causal != 0 && cfg->causal != 1) || cfg->reserved != 0 ||
        cfg->window < 0 || (cfg->window > 0 && !cfg->causal) || cfg->max_len < 0) {
        if (cfg)
            set_error("scale %g, causal %d, window %lld (only with causal), max_len %lld, reserved %d", cfg->scale,
                      cfg->causal, (long long)cfg->window, (long long)cfg->max_len, cfg->reserved);
        else
            set_error("null cfg");
        return DS_EINVAL;
    }
    return DS_OK;
}

int most_keys(const ds_cache8 *cache, const ds_chunk *chunk, const ds_attn8_cfg *cfg) {
    const int64_t held = chunk->table_cols * cache->page;
    return int(cfg->max_len > 0 ? std::min(cfg->max_len, held) : held);
}

// The form and the splits, from what the host knows: tokens, sequences, heads and the most keys.
AttnPlan attn_plan(const ds_heads *q, const ds_cache8 *cache, const ds_chunk *chunk, const ds_attn8_cfg *cfg) {
    AttnPlan p{};
    const int64_t group = q->heads / cache->heads, rows = q->tokens * group;
    const int db = attn8_dim_blocks(cache->dim);
    const bool own = q->type == DS_TYPE_F32 ? attn8_own_form<float>(db) : attn8_own_form<__bf16>(db);
    p.form = rows <= 16 * chunk->seqs ? kAttnFew : rows <= 64 * chunk->seqs ? kAttnShare : own ? kAttnOwn : kAttnTiles;
    const int tile = attn8_rows(p.form);
    const int64_t base = (rows / tile + chunk->seqs) * cache->heads;
    int64_t keys = most_keys(cache, chunk, cfg);
    if (cfg->window > 0) keys = std::min(keys, std::min(cfg->window, kMaxPlaces) + tile / group + 1 + 64);
    // The split that ends first: rounds of workgroups that the chip holds, each as long as its keys and what a
    // workgroup needs beside them (in workgroups of four waves, 64 equal sequences of 8192 keys: 166 us whole, 176 to
    // 188 in two to four parts; of unequal lengths 118 whole, 112 in three parts, 136 and 151 in two and four: full
    // rounds of whole sequences stay whole).
    const bool shares = p.form == kAttnFew || p.form == kAttnShare;
    p.threads = attn8_threads(p.form, db);
    const int64_t unit = shares ? p.threads / 64 * 32 : 64, beside = 4 * unit;
    const int64_t slots = 256 * attn8_groups(p.form, q->type == DS_TYPE_F32, db);
    const int64_t work = std::max((rows + tile - 1) / tile, std::min(q->tokens, chunk->seqs)) * cache->heads;
    int64_t best = INT64_MAX;
    for (const int64_t splits : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64}) {
        static_assert(kMostSplits == 64, "the last of these");
        const int64_t span = std::max(unit, ((keys + splits - 1) / splits + unit - 1) / unit * unit);
        const int64_t n = std::max<int64_t>(1, (keys + span - 1) / span);
        const int64_t time = (work * n + slots - 1) / slots * (span + beside) + (n > 1 ? beside : 0);
        if (time < best) {
            best = time;
            p.span = int(std::min<int64_t>(span, kMaxPlaces));
            p.splits = int(n);
        }
        if (span == unit) break;
    }
    p.groups = base * p.splits;
    if (p.splits > 1) {
        p.part = p.splits * q->tokens * q->heads * cache->dim * 4;
        p.bytes = p.part + p.splits * q->tokens * q->heads * 8;
    }
    return p;
}

template <typename T>
int run(const AttnPlan &p, AttnArgs a, bool exact, hipStream_t stream) {
    const AttnKernel k = attn8_kernel<T>(p.form, a.c.fmt, a.c.stype, a.c.dim, exact);
    if (k.lds) {
        const int rc = ensure_lds_attr(k.func, k.lds);
        if (rc != DS_OK) return rc;
    }
    void *argv[] = {&a};
    if (!hip_ok(hipLaunchKernel(k.func, dim3(unsigned(p.groups)), dim3(p.threads), argv, k.lds, stream), "ds_attn8"))
        return DS_EHIP;
    if (p.splits > 1) {
        const int64_t rows = int64_t(a.n.tokens) * a.heads;
        (a.c.dim <= 64 ? attn8_join<T, 16> : a.c.dim <= 128 ? attn8_join<T, 32> : attn8_join<T, 64>)
            <<<unsigned((rows + kJoinWaves - 1) / kJoinWaves), 64 * kJoinWaves, 0, stream>>>(a);
        if (!hip_ok(hipGetLastError(), "ds_attn8")) return DS_EHIP;
    }
    return DS_OK;
}

}  // namespace
}  // namespace ds

using namespace ds;

extern "C" {

int ds_attn8_work(const ds_heads *q, const ds_cache8 *cache, const ds_chunk *chunk, const ds_attn8_cfg *cfg,
                  int64_t *bytes) {
    ds_heads of;
    bool exact;
    q = plain_type(q, &of, &exact);
    const int rc = attn_check(q, cache, chunk, cfg);
    if (rc != DS_OK) return rc;
    if (!bytes) {
        set_error("null bytes");
        return DS_EINVAL;
    }
    *bytes = q->tokens == 0 || chunk->seqs == 0 ? 0 : attn_plan(q, cache, chunk, cfg).bytes;
    return DS_OK;
}

int ds_attn8(const ds_heads *q, const ds_cache8 *cache, const ds_chunk *chunk, const ds_attn8_cfg *cfg,
             const ds_heads *out, float *lse, void *work, int64_t work_bytes, hipStream_t stream) {
    ds_heads of;
    bool exact;
    q = plain_type(q, &of, &exact);
    int rc = attn_check(q, cache, chunk, cfg);
    if (rc != DS_OK || (rc = heads_check(out, "out", true)) != DS_OK) return rc;
    if (out->tokens != q->tokens || out->heads != q->heads || out->dim != q->dim || out->type != q->type) {
        set_error("out is %lld x %lld x %lld of type %d, q %lld x %lld x %lld of type %d", (long long)out->tokens,
                  (long long)out->heads, (long long)out->dim, out->type, (long long)q->tokens, (long long)q->heads,
                  (long long)q->dim, q->type);
        return DS_EINVAL;
    }
    if (reinterpret_cast<uintptr_t>(lse) % 4 != 0) {
        set_error("misaligned lse");
        return DS_EINVAL;
    }
    if (q->tokens == 0 || chunk->seqs == 0) return DS_OK;
    const AttnPlan p = attn_plan(q, cache, chunk, cfg);
    if (work_bytes < p.bytes || (p.bytes > 0 && (!work || reinterpret_cast<uintptr_t>(work) % 16 != 0))) {
        set_error("a workspace of %lld bytes, 16-byte aligned, not %lld at %p", (long long)p.bytes,
                  (long long)work_bytes, work);
        return DS_EINVAL;
    }
    if (q->tokens * (q->heads / cache->heads) > 0x7ffffe00) {
        set_error("%lld tokens of %lld heads a cache head", (long long)q->tokens, (long long)(q->heads / cache->heads));
        return DS_EUNSUPPORTED;
    }
    if ((rc = launch_check(p.groups, p.threads, "ds_attn8")) != DS_OK ||
        (rc = launch_check((q->tokens * q->heads + kJoinWaves - 1) / kJoinWaves, 256, "ds_attn8")) != DS_OK)
        return rc;
    AttnArgs a{};
    a.c = cache_view(cache);
    a.n = chunk_view(chunk, cache, q->tokens);
    a.q = q->data;
    a.out = out->data;
    a.ldq = q->ld;
    a.hldq = q->head_ld;
    a.ldo = out->ld;
    a.hldo = out->head_ld;
    a.lse = lse;
    a.part = static_cast<float *>(work);
    a.ml = reinterpret_cast<float2 *>(static_cast<char *>(work) + p.part);
    a.scale = float(cfg->scale * 1.4426950408889634);
    a.heads = int(q->heads);
    a.group = int(q->heads / cache->heads);
    a.causal = cfg->causal;
    a.window = int(std::min<int64_t>(cfg->window, kMaxPlaces));
    a.len = most_keys(cache, chunk, cfg);
    a.splits = p.splits;
    a.span = p.span;
    a.f_group = make_fastdiv(a.group);
    a.f_kv = make_fastdiv(cache->heads);
    a.f_splits = make_fastdiv(a.splits);
    a.f_dim4 = make_fastdiv(cache->dim / 4);
    a.vec_q = heads16(q);
    a.vec_o = heads16(out);
    if (q->type == DS_TYPE_F32) return run<float>(p, a, exact, stream);
    if (q->type == DS_TYPE_F16) return run<_Float16>(p, a, exact, stream);
    return run<__bf16>(p, a, exact, stream);
}

}  // extern "C"
