// C-ABI entry points of the attention part: argument checks and launches; the table of rotations.
#include "tl_attn.hpp"

#include <cmath>

namespace tl {
namespace {

inline bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// 128 tokens of less than 2^24 elements each lie within 32-bit offsets (without a sign) of 2-byte numbers.
inline tl_status heads_status(const tl_heads& h, int64_t heads)
{
    if (heads == 0) return TL_OK;
    if (!h.ptr) return TL_ERR_NULL;
    const int64_t lim = int64_t(1) << 24;
    if (h.token_stride < 0 || h.head_stride < 0 || h.token_stride >= lim || h.head_stride >= (int64_t(1) << 40)) return TL_ERR_SHAPE;
    if (!aligned(h.ptr, 16) || h.token_stride % 8 != 0 || h.head_stride % 8 != 0) return TL_ERR_ALIGN;
    return TL_OK;
}

inline Heads heads_of(const tl_heads& h) { return {static_cast<_Float16*>(h.ptr), h.token_stride, h.head_stride}; }

// A grid holds fewer than 2^32 threads in a direction: 2^24 workgroups of 256.
constexpr int64_t kMaxSeqs = int64_t(1) << 20, kMaxTokens = int64_t(1) << 23, kMaxGroups = int64_t(1) << 24;

inline tl_status batch_status(const tl_batch& b)
{
    if (b.seqs < 1 || b.seqs >= kMaxSeqs || b.tokens < 0 || b.tokens >= kMaxTokens) return TL_ERR_SHAPE;
    if (!b.seq_start && b.tokens != b.seqs) return TL_ERR_SHAPE;
    if (!aligned(b.seq_start, 4) || !aligned(b.cached, 4)) return TL_ERR_ALIGN;
    return TL_OK;
}

inline Batch batch_of(const tl_batch& b) { return {b.seq_start, b.cached, int(b.seqs), int(b.tokens)}; }

inline bool dim_ok(int64_t d) { return d >= 16 && d <= 128 && d % 16 == 0; }
constexpr int64_t kMaxHeads = 4096;

inline tl_status heads_number_status(int64_t q_heads, int64_t kv_heads)
{
    if (q_heads < 1 || kv_heads < 1 || q_heads > kMaxHeads || kv_heads > q_heads || q_heads % kv_heads != 0) return TL_ERR_SHAPE;
    return TL_OK;
}

inline tl_status cache_status(const tl_kv_cache& c)
{
    if (!c.k || !c.v || !c.k_scale || !c.v_scale || !c.page_table) return TL_ERR_NULL;
    if (c.type != TL_KV_INT8 && c.type != TL_KV_FP8) return TL_ERR_UNSUPPORTED;
    if (c.kv_heads < 1 || c.kv_heads > kMaxHeads || !dim_ok(c.head_dim)) return TL_ERR_SHAPE;
    const int64_t lim = int64_t(1) << 31;
    if (c.page_tokens < 16 || c.page_tokens > 1024 || (c.page_tokens & (c.page_tokens - 1))) return TL_ERR_SHAPE;
    if (c.pages < 1 || c.pages >= lim || c.pages_per_seq < 1 || c.pages_per_seq > (lim - 1) / c.page_tokens) return TL_ERR_SHAPE;
    if (!aligned(c.k, 16) || !aligned(c.v, 16) || !aligned(c.k_scale, 4) || !aligned(c.v_scale, 4) || !aligned(c.page_table, 4)) return TL_ERR_ALIGN;
    return TL_OK;
}

inline Cache cache_of(const tl_kv_cache& c)
{
    int shift = 0;
    while ((int64_t(16) << shift) < c.page_tokens) ++shift;
    return {static_cast<uint8_t*>(c.k), static_cast<uint8_t*>(c.v), c.k_scale, c.v_scale, c.page_table, c.pages, c.pages_per_seq,
            int(c.kv_heads), int(c.head_dim), shift, c.type == TL_KV_FP8};
}

inline tl_status from_hip(hipError_t e) { return e == hipSuccess ? TL_OK : TL_ERR_HIP; }

constexpr float kLog2e = 1.44269504088896340736f;

}  // namespace
}  // namespace tl

extern "C" {

tl_status tl_rope_table(float* table, int64_t positions, int64_t rot_dim, double base, const tl_rope_scaling* scaling)
{
    if (!table) return TL_ERR_NULL;
    if (positions < 1 || rot_dim < 2 || rot_dim % 2 != 0 || positions > (int64_t(1) << 40) / rot_dim) return TL_ERR_SHAPE;
    const auto positive = [](double x) { return x > 0.0 && std::isfinite(x); };
    if (!positive(base)) return TL_ERR_VALUE;
    const tl_rope_scaling none{TL_ROPE_PLAIN, 1.0, 1.0, 0.0, 1.0, 1.0};
    const tl_rope_scaling& sc = scaling ? *scaling : none;
    if (sc.kind != TL_ROPE_PLAIN && sc.kind != TL_ROPE_LINEAR && sc.kind != TL_ROPE_BY_PARTS) return TL_ERR_UNSUPPORTED;
    if (!positive(sc.magnitude) || (sc.kind != TL_ROPE_PLAIN && !positive(sc.factor))) return TL_ERR_VALUE;
    if (sc.kind == TL_ROPE_BY_PARTS && (!positive(sc.trained) || !(sc.low >= 0.0) || !(sc.low < sc.high) || !std::isfinite(sc.high))) return TL_ERR_VALUE;
    const int64_t half = rot_dim / 2;
    for (int64_t j = 0; j < half; ++j) {
        double f = std::pow(base, -2.0 * double(j) / double(rot_dim));
        if (sc.kind == TL_ROPE_LINEAR) f /= sc.factor;
        if (sc.kind == TL_ROPE_BY_PARTS) {
            const double turns = sc.trained * f / 6.283185307179586476925;
            const double keep = turns <= sc.low ? 0.0 : turns >= sc.high ? 1.0 : (turns - sc.low) / (sc.high - sc.low);
            f = keep * f + (1.0 - keep) * f / sc.factor;
        }
        for (int64_t p = 0; p < positions; ++p) {
            const double x = double(p) * f;
            table[p * rot_dim + j] = float(sc.magnitude * std::cos(x));
            table[p * rot_dim + half + j] = float(sc.magnitude * std::sin(x));
        }
    }
    return TL_OK;
}

tl_status tl_kv_append(const tl_append_job* job, void* stream)
{
    using namespace tl;
    if (!job) return TL_ERR_NULL;
    const tl_append_job& j = *job;
    tl_status e = batch_status(j.batch);
    if (e != TL_OK) return e;
    if (j.q_heads < 0 || j.kv_heads < 0 || j.q_heads > kMaxHeads || j.kv_heads > kMaxHeads || j.q_heads + j.kv_heads == 0 || !dim_ok(j.head_dim)) return TL_ERR_SHAPE;
    AppendArgs a{};
    if (j.cache) {
        if ((e = cache_status(*j.cache)) != TL_OK) return e;
        if (j.cache->kv_heads != j.kv_heads || j.cache->head_dim != j.head_dim) return TL_ERR_SHAPE;
        if ((e = heads_status(j.v, j.kv_heads)) != TL_OK) return e;
        a.c = cache_of(*j.cache);
        a.v = heads_of(j.v);
    }
    if (j.rope) {
        const tl_rope& r = *j.rope;
        if (!r.table) return TL_ERR_NULL;
        if (r.positions < 1 || r.positions >= (int64_t(1) << 40) || r.rot_dim < 2 || r.rot_dim % 2 != 0 || r.rot_dim > j.head_dim) return TL_ERR_SHAPE;
        if (!aligned(r.table, 4)) return TL_ERR_ALIGN;
        const bool pairs = r.pairs != 0;
        const bool wide = aligned(r.table, 16) && r.rot_dim % (pairs ? 8 : 16) == 0;
        a.r = {r.table, r.positions, int(r.rot_dim), pairs, wide};
    }
    if ((e = heads_status(j.q, j.q_heads)) != TL_OK || (e = heads_status(j.k, j.kv_heads)) != TL_OK) return e;
    if (j.q_out.ptr && (e = heads_status(j.q_out, j.q_heads)) != TL_OK) return e;
    if (j.k_out.ptr && (e = heads_status(j.k_out, j.kv_heads)) != TL_OK) return e;
    if (j.batch.tokens == 0) return TL_OK;
    a.q = heads_of(j.q);
    a.k = heads_of(j.k);
    a.q_out = heads_of(j.q_out);
    a.k_out = heads_of(j.k_out);
    a.b = batch_of(j.batch);
    a.q_heads = a.q_out.p ? int(j.q_heads) : 0;
    a.kv_heads = a.c.k || a.k_out.p ? int(j.kv_heads) : 0;
    a.dim = int(j.head_dim);
    if (a.q_heads + a.kv_heads == 0) return TL_OK;
    return from_hip(launch_append(a, static_cast<hipStream_t>(stream)));
}

size_t tl_attn_cached_workspace(int64_t seqs, int64_t tokens, int64_t q_heads, int64_t kv_heads, int64_t head_dim)
{
    if (seqs < 1 || seqs >= tl::kMaxSeqs || tokens < 0 || tokens >= tl::kMaxTokens) return 0;
    if (tl::heads_number_status(q_heads, kv_heads) != TL_OK || !tl::dim_ok(head_dim)) return 0;
    return tl::cached_workspace(seqs, tokens, q_heads, kv_heads, head_dim);
}

tl_status tl_attn_cached(const tl_cached_job* job, void* stream)
{
    using namespace tl;
    if (!job) return TL_ERR_NULL;
    const tl_cached_job& j = *job;
    if (!j.cache) return TL_ERR_NULL;
    tl_status e = batch_status(j.batch);
    if (e != TL_OK || (e = cache_status(*j.cache)) != TL_OK) return e;
    if ((e = heads_number_status(j.q_heads, j.cache->kv_heads)) != TL_OK) return e;
    if (j.longest < 0) return TL_ERR_SHAPE;
    if (!std::isfinite(j.scale * kLog2e)) return TL_ERR_VALUE;
    if ((e = heads_status(j.q, j.q_heads)) != TL_OK || (e = heads_status(j.out, j.q_heads)) != TL_OK) return e;
    if (!j.workspace) return TL_ERR_NULL;
    if (!aligned(j.workspace, 16)) return TL_ERR_ALIGN;
    if (j.workspace_bytes < cached_workspace(j.batch.seqs, j.batch.tokens, j.q_heads, j.cache->kv_heads, j.cache->head_dim)) return TL_ERR_SHAPE;
    if (j.batch.tokens == 0) return TL_OK;
    CachedArgs a{heads_of(j.q), heads_of(j.out), batch_of(j.batch), cache_of(*j.cache), int(j.q_heads), int(j.q_heads / j.cache->kv_heads),
                 j.scale * kLog2e, static_cast<float*>(j.workspace)};
    return from_hip(launch_cached(a, j.longest, static_cast<hipStream_t>(stream)));
}

tl_status tl_attn_prompt(const tl_prompt_job* job, void* stream)
{
    using namespace tl;
    if (!job) return TL_ERR_NULL;
    const tl_prompt_job& j = *job;
    tl_status e = batch_status(j.batch);
    if (e != TL_OK || (e = heads_number_status(j.q_heads, j.kv_heads)) != TL_OK) return e;
    if (!dim_ok(j.head_dim)) return TL_ERR_SHAPE;
    if ((j.batch.seqs + j.batch.tokens / 32) * j.q_heads >= kMaxGroups) return TL_ERR_SHAPE;
    if (!std::isfinite(j.scale * kLog2e)) return TL_ERR_VALUE;
    if ((e = heads_status(j.q, j.q_heads)) != TL_OK || (e = heads_status(j.k, j.kv_heads)) != TL_OK || (e = heads_status(j.v, j.kv_heads)) != TL_OK ||
        (e = heads_status(j.out, j.q_heads)) != TL_OK) return e;
    if (j.batch.tokens == 0) return TL_OK;
    PromptArgs a{heads_of(j.q), heads_of(j.k), heads_of(j.v), heads_of(j.out), batch_of(j.batch), int(j.q_heads), int(j.kv_heads),
                 int(j.q_heads / j.kv_heads), int(j.head_dim), j.scale * kLog2e};
    return from_hip(launch_prompt(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
