// Attention of drafted tokens over a key/value cache (cf_tree_* in include/cfdecode.h).
#include "../../include/cfdecode.h"
#include "cf_cache_device.h"
#include "cf_lanes_device.h"

#include <cmath>
#include <cstring>
#include <new>

namespace {

using namespace cf::cache;

constexpr int kMaxTokens = 256;

struct TreeArgs {
    const uint16_t *q;
    const char *k, *v;
    const float *k_scale, *v_scale, *slopes;
    uint16_t *out;
    Lengths rows;
    const int32_t *depth;
    const uint64_t *tree;
    int depth_stride;              // depths of a batch row: 0 where all share them
    int tree_stride, words;        // words of a batch row's masks (0: shared), of a token's mask
    int nq, nkv, max_seq, window;
    float cap;
};

template <int FMT>
__device__ __forceinline__ float value(const char *row, int i, float scale)
{
    if constexpr (FMT == CF_CACHE_F16)
        return (float)reinterpret_cast<const _Float16 *>(row)[i];
    else {
        float f[4];
        decode4<FMT>((uint32_t)(uint8_t)row[i], f);
        return f[0] * scale;
    }
}

// One wavefront per drafted token and query head: 64 keys at a time, a key to a lane for the scores, a dimension (and the one 64
// further on) to a lane for the values.
template <int HD, int FMT>
__global__ __launch_bounds__(64) void tree_rows(const TreeArgs a)
{
    __shared__ float qs[HD], ps[64];
    const int lane = threadIdx.x, h = blockIdx.x, t = blockIdx.y, b = blockIdx.z;
    const int n = a.rows.fresh(b), len = a.rows.cached(b);
    if (t >= n) return;
    const int g = h / (a.nq / a.nkv);
    const size_t at = (((size_t)b * a.rows.tokens + t) * a.nq + h) * HD, slice = ((size_t)b * a.nkv + g) * a.max_seq;
    for (int i = lane; i < HD; i += 64) qs[i] = (float)__builtin_bit_cast(_Float16, a.q[at + i]);
    __syncthreads();
    const int32_t *depth = a.depth ? a.depth + (size_t)b * a.depth_stride : nullptr;
    const uint64_t *mask = a.tree ? a.tree + (size_t)b * a.tree_stride + (size_t)t * a.words : nullptr;
    const long long mine = (long long)len + (depth ? depth[t] : t);
    const float slope = a.slopes ? a.slopes[h] : 0.f;
    float m = -1e30f, l = 0.f, o[HD / 64] = {};
    for (int j0 = 0; j0 < len + n; j0 += 64) {
        const int j = j0 + lane, u = j - len;
        bool seen = j < len + n && (u < 0 || (mask ? (mask[u >> 6] >> (u & 63)) & 1 : u <= t));
        float s = 0.f;
        if (seen) {
            const long long theirs = u < 0 ? j : (long long)len + (depth ? depth[u] : u);
            if (a.window > 0 && mine - theirs >= a.window) seen = false;
            const char *row = a.k + (slice + j) * HD * kValueBytes<FMT>;
            const float scale = FMT == CF_CACHE_F16 ? 1.f : a.k_scale[slice + j];
            for (int i = 0; i < HD; ++i) s += qs[i] * value<FMT>(row, i, scale);
            s *= HD == 64 ? 0.125f : 0.08838834764831845f;
            if (a.cap > 0.f) s = a.cap * tanhf(s / a.cap);
            s -= slope * (float)(mine - theirs);
        }
        float top = seen ? s : -1e30f;
        top = fmaxf(m, cf::lanes::max_row(cf::lanes::max_groups<16>(top)));
        const float p = seen ? expf(s - top) : 0.f, old = expf(m - top);
        m = top;
        l = l * old + cf::lanes::sum_row(cf::lanes::sum_groups<16>(p));
        __syncthreads();
        ps[lane] = p;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < HD / 64; ++i) {
            o[i] *= old;
            for (int e = 0; e < 64; ++e)
                if (ps[e] != 0.f) {
                    const char *row = a.v + (slice + j0 + e) * HD * kValueBytes<FMT>;
                    o[i] += ps[e] * value<FMT>(row, lane + 64 * i, FMT == CF_CACHE_F16 ? 1.f : a.v_scale[slice + j0 + e]);
                }
        }
    }
#pragma unroll
    for (int i = 0; i < HD / 64; ++i) a.out[at + lane + 64 * i] = __builtin_bit_cast(uint16_t, (_Float16)(l == 0.f ? 0.f : o[i] / l));
}

using KernelFn = void (*)(const TreeArgs);
KernelFn pick(int hd, int fmt)
{
    if (hd == 64) return fmt == CF_CACHE_F16 ? tree_rows<64, CF_CACHE_F16> : fmt == CF_CACHE_E4M3 ? tree_rows<64, CF_CACHE_E4M3> : tree_rows<64, CF_CACHE_INT8>;
    return fmt == CF_CACHE_F16 ? tree_rows<128, CF_CACHE_F16> : fmt == CF_CACHE_E4M3 ? tree_rows<128, CF_CACHE_E4M3> : tree_rows<128, CF_CACHE_INT8>;
}

}  // namespace

struct cf_tree_s {
    cf_tree_config cfg;
    int device = 0;
    int max_splits = 0;
};

extern "C" {

int cf_tree_create(const cf_tree_config *cfg, cf_tree *out)
{
    if (!cfg || !out) return CF_EINVAL;
    *out = nullptr;
    const int rc = check_config(cfg->cache);
    if (rc != CF_OK) return rc;
    if (cfg->max_tokens < 1 || cfg->max_tokens > kMaxTokens || cfg->window < 0 || !(cfg->score_cap >= 0.f) || !(cfg->score_cap <= 3.402823466e38f)) return CF_EINVAL;
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess) return CF_EHIP;
    cf_tree t = new (std::nothrow) cf_tree_s();
    if (!t) return CF_ENOMEM;
    t->cfg = *cfg;
    t->device = dev;
    *out = t;
    return CF_OK;
}

int cf_tree_destroy(cf_tree t)
{
    if (!t) return CF_EINVAL;
    delete t;
    return CF_OK;
}

int cf_tree_attend(cf_tree t, int32_t batch, const void *q, const cf_cache *cache, const cf_draft *draft, const float *slopes,
                   void *out, void *stream)
{
    if (!t) return CF_EINVAL;
    const cf_cache_config &c = t->cfg.cache;
    int rc = check_cache(c, cache, batch);
    if (rc == CF_OK) rc = check_draft(c, draft);
    if (rc != CF_OK) return rc;
    if (!q || !out || !aligned(q, 16) || !aligned(out, 16) || !aligned(slopes, 4) || draft->tokens > t->cfg.max_tokens) return CF_EINVAL;
    const size_t q_bytes = 2 * (size_t)batch * draft->tokens * c.n_q_heads * c.head_dim;
    if (overlap(q, q_bytes, out, q_bytes)) return CF_EINVAL;
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess) return CF_EHIP;
    if (dev != t->device) return CF_EINVAL;
    TreeArgs a;
    std::memset(&a, 0, sizeof a);
    a.q = static_cast<const uint16_t *>(q), a.out = static_cast<uint16_t *>(out);
    a.k = static_cast<const char *>(cache->k), a.v = static_cast<const char *>(cache->v);
    a.k_scale = cache->k_scale, a.v_scale = cache->v_scale, a.slopes = slopes;
    a.rows = lengths_of(*draft);
    a.depth = draft->depth, a.tree = draft->tree;
    a.words = (draft->tokens + 63) / 64;
    a.depth_stride = draft->per_row ? draft->tokens : 0;
    a.tree_stride = draft->per_row ? draft->tokens * a.words : 0;
    a.nq = c.n_q_heads, a.nkv = c.n_kv_heads, a.max_seq = c.max_seq, a.window = t->cfg.window, a.cap = t->cfg.score_cap;
    hipLaunchKernelGGL(pick(c.head_dim, c.format), dim3(c.n_q_heads, draft->tokens, batch), dim3(64), 0, static_cast<hipStream_t>(stream), a);
    return hipGetLastError() == hipSuccess ? CF_OK : CF_EHIP;
}

int cf_tree_set_splits(cf_tree t, int32_t max_splits)
{
    if (!t || max_splits < 0 || max_splits > 64) return CF_EINVAL;
    t->max_splits = max_splits;
    return CF_OK;
}

int64_t cf_tree_algorithmic_bytes(const cf_tree_config *cfg, int32_t batch, int32_t tokens, int32_t len)
{
    if (!cfg) return 0;
    const cf_cache_config &c = cfg->cache;
    const int64_t row = c.format == CF_CACHE_F16 ? 2 * (int64_t)c.head_dim : (int64_t)c.head_dim + 4;
    const int64_t read = cfg->window > 0 && cfg->window < len ? cfg->window : len;      // cached rows that some token may see
    return (int64_t)batch * (2 * c.n_kv_heads * row * (read + tokens) + 4 * (int64_t)tokens * c.n_q_heads * c.head_dim);
}

}  // extern "C"
