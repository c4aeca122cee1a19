// A key/value cache in fp16 or 8 bits: written with the rotated keys and the values of new tokens, read back as fp16, and its rows of
// accepted tokens moved together (cf_cache_* in include/cfdecode.h).  Three kernels without waits between workgroups.
#include "../../include/cfdecode.h"
#include "cf_cache_device.h"
#include "cf_lanes_device.h"
#include "cf_rope_device.h"

#include <cmath>
#include <cstring>

namespace {

using namespace cf::cache;

constexpr int NT = 256;
constexpr int NW = NT / 64;
constexpr int kMaxKept = 256;      // tokens of a cf_cache_keep: their rows are held in LDS, 64 KB of fp16 at head dimension 128

// ---- append ----------------------------------------------------------------------------------------------------------------
//
// Eight dimensions i and their eight partners i + HD / 2 to a lane, so that a row of a head is held by HD / 16 lanes and a wavefront
// takes 64 / (HD / 16) heads of one token at a time.  cos and sin of a token's HD / 2 angles are computed once, one angle to a thread,
// and handed to all heads through LDS.
// Arithmetic: angle, cos, sin and the rotation are fp64 and the result is rounded to fp16 once.  A fp32 rotation is off by 2^-23, which
// moves one value in some thousands to the other fp16 neighbour, and through it one 8-bit code in 10^5; in fp64 the angle is off by some
// 2^-51 of itself (a power, the product of two, the product with the position), at position 32768 by 2^-36, which moves one value in
// 10^7; the vector units are idle beside it all the same (27.6 million instructions of 16384 wavefronts in 70 us).
// Bound: memory.  Two prompts of 8192 and 6144 tokens, 32 + 2 x 8 heads of 128 dimensions, into int8: 324 MB in 70 us, 4.6 TB/s (a copy
// reaches 4.8).  With few tokens the launch: one token 3.6 us on the GPU, so its heads are spread over more workgroups.
struct AppendArgs {
    const uint16_t *qkv;
    uint16_t *q_out;
    char *k, *v;
    float *k_scale, *v_scale;
    Lengths rows;
    const int32_t *depth;
    int depth_stride;              // depths of a batch row: 0 where all share them
    int nq, nkv, max_seq;
    int nt;                        // tokens of a workgroup: 1 or 4
    double theta[64];              // base^(-2i / HD)
};

// x as fp16, rounded once.  (A conversion by way of fp32 alone would round twice: where the fp32 value is not exact its last bit is made odd
// in the direction of x, so that it is no fp16 value and no middle of two.)
__device__ __forceinline__ _Float16 half_once(double x)
{
    const float f = (float)x;
    const double rest = x - (double)f;
    uint32_t bits = __builtin_bit_cast(uint32_t, f);
    if ((rest > 0.0 || rest < 0.0) && !(bits & 1u) && f != 0.f) bits += (rest > 0.0) == (f > 0.f) ? 1u : ~0u;
    return (_Float16)__builtin_bit_cast(float, bits);
}

template <int HD>
__device__ __forceinline__ uint32_t row_top(uint32_t t)      // largest of the HD / 16 lanes that hold a row
{
    t = max(t, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)t, 0xB1, 0xF, 0xF, true));        // lane ^ 1
    t = max(t, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)t, 0x4E, 0xF, 0xF, true));        // lane ^ 2
    return HD == 64 ? t : max(t, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)t, 0x141, 0xF, 0xF, true));   // 7 - lane
}

template <int HD, int FMT>
__global__ __launch_bounds__(NT) void cache_append(const AppendArgs a)
{
    constexpr int LPR = HD / 16, RPW = 64 / LPR, HALF = HD / 2;
    __shared__ double2 turn[4][HALF];
    const int tid = threadIdx.x, wv = tid >> 6, lane = tid & 63;
    const int b = blockIdx.z, t0 = blockIdx.x * a.nt;
    const int n = a.rows.fresh(b), len = a.rows.cached(b);
    if (t0 >= n) return;
    {
        const int slot = tid / 64, i = lane;
        if (slot < a.nt && i < HALF && t0 + slot < n) {
            const int depth = a.depth ? a.depth[(size_t)b * a.depth_stride + t0 + slot] : t0 + slot;
            double c, s;
            cf::rope_cos_sin64((double)len + (double)depth, a.theta[i], c, s);
            turn[slot][i] = make_double2(c, s);
        }
    }
    __syncthreads();
    const int slot = wv % a.nt, t = t0 + slot;
    if (t >= n) return;
    const int H = a.nq + 2 * a.nkv, groups = (H + RPW - 1) / RPW, step = (NW / a.nt) * gridDim.y;
    const int li = lane % LPR;
    for (int grp = wv / a.nt + (NW / a.nt) * blockIdx.y; grp < groups; grp += step) {
        const int head = grp * RPW + lane / LPR;
        if (head >= H) continue;                                   // (whole rows of lanes: the maxima below stay inside a row)
        const uint16_t *src = a.qkv + (((size_t)b * a.rows.tokens + t) * H + head) * HD + 8 * li;
        h8 lo = *reinterpret_cast<const h8 *>(src), hi = *reinterpret_cast<const h8 *>(src + HALF);
        if (head < a.nq + a.nkv) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const double2 cs = turn[slot][8 * li + j];
                const double x = (double)(float)lo[j], y = (double)(float)hi[j];
                lo[j] = half_once(x * cs.x - y * cs.y);
                hi[j] = half_once(y * cs.x + x * cs.y);
            }
        }
        if (head < a.nq) {
            uint16_t *dst = a.q_out + (((size_t)b * a.rows.tokens + t) * a.nq + head) * HD + 8 * li;
            *reinterpret_cast<h8 *>(dst) = lo;
            *reinterpret_cast<h8 *>(dst + HALF) = hi;
            continue;
        }
        const bool key = head < a.nq + a.nkv;
        const size_t row = ((size_t)b * a.nkv + (head - a.nq - (key ? 0 : a.nkv))) * a.max_seq + len + t;
        char *dst = (key ? a.k : a.v) + (row * HD + 8 * li) * kValueBytes<FMT>;
        if constexpr (FMT == CF_CACHE_F16) {
            *reinterpret_cast<h8 *>(dst) = lo;
            *reinterpret_cast<h8 *>(dst + 2 * HALF) = hi;
        } else {
            const Encoder<FMT> enc(row_top<HD>(max(top_bits(lo), top_bits(hi))));
            *reinterpret_cast<u32x2 *>(dst) = enc.codes(lo);
            *reinterpret_cast<u32x2 *>(dst + HALF) = enc.codes(hi);
            if (li == 0) (key ? a.k_scale : a.v_scale)[row] = enc.scale;
        }
    }
}

// ---- read ------------------------------------------------------------------------------------------------------------------

// Sixteen codes of a row and its scale to a thread, 32 bytes out; 8-bit codes are turned into fp32 by the conversion instructions, the product
// with the scale is rounded to fp16 once.  Bound: memory.  16 x 3511 rows, 8 heads of 128 dimensions, e4m3: 349 MB in 75.7 us, 4.6 TB/s
// (a copy reaches 4.8); a small one 3.7 us, the launch.
struct ReadArgs {
    const char *k, *v;
    const float *k_scale, *v_scale;
    uint16_t *k_out, *v_out;
    int max_seq, first, rows;
};
constexpr int kReadPieces = 4;     // pieces of sixteen values to a thread, all requested before the first is used

template <int HD, int FMT>
__global__ __launch_bounds__(NT) void cache_read(const ReadArgs a)
{
    const bool key = blockIdx.z == 0;
    const size_t slice = (size_t)blockIdx.y * a.max_seq + a.first;
    const char *src = (key ? a.k : a.v) + slice * HD * kValueBytes<FMT>;
    const float *scale = (key ? a.k_scale : a.v_scale) + (FMT == CF_CACHE_F16 ? 0 : slice);
    uint16_t *dst = (key ? a.k_out : a.v_out) + (size_t)blockIdx.y * a.rows * HD;
    const uint32_t pieces = (uint32_t)a.rows * (HD / 16), at = blockIdx.x * (NT * kReadPieces) + threadIdx.x;
    if constexpr (FMT == CF_CACHE_F16) {
        u32x4 x[kReadPieces][2];
#pragma unroll
        for (int i = 0; i < kReadPieces; ++i)
            if (at + NT * i < pieces)
                for (int w = 0; w < 2; ++w) x[i][w] = *reinterpret_cast<const u32x4 *>(src + (size_t)(at + NT * i) * 32 + 16 * w);
#pragma unroll
        for (int i = 0; i < kReadPieces; ++i)
            if (at + NT * i < pieces)
                for (int w = 0; w < 2; ++w) *reinterpret_cast<u32x4 *>(dst + (size_t)(at + NT * i) * 16 + 8 * w) = x[i][w];
    } else {
        u32x4 x[kReadPieces];
        float s[kReadPieces];
#pragma unroll
        for (int i = 0; i < kReadPieces; ++i)
            if (at + NT * i < pieces) {
                x[i] = *reinterpret_cast<const u32x4 *>(src + (size_t)(at + NT * i) * 16);
                s[i] = scale[(at + NT * i) / (HD / 16)];
            }
#pragma unroll
        for (int i = 0; i < kReadPieces; ++i)
            if (at + NT * i < pieces) {
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    h8 o;
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        float f[4];
                        decode4<FMT>(x[i][2 * w + q], f);
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[4 * q + e] = (_Float16)(f[e] * s[i]);
                    }
                    *reinterpret_cast<h8 *>(dst + (size_t)(at + NT * i) * 16 + 8 * w) = o;
                }
            }
    }
}

// ---- keep ------------------------------------------------------------------------------------------------------------------

struct KeepArgs {
    char *k, *v;
    float *k_scale, *v_scale;
    Lengths rows;
    const int32_t *kept, *n_kept;
    int32_t *new_len;
    int nkv, max_seq, row_bytes;
};

// One workgroup per head's slice: its kept rows into LDS, a barrier, and out to their places (a place may be another row's source).
// Bound: the launch and one trip to memory and back, 2.8 us for up to 128 slices; a call 6.8 us, which is the host's part.
__global__ __launch_bounds__(NT) void cache_keep(const KeepArgs a)
{
    extern __shared__ char held[];
    const int tid = threadIdx.x, b = blockIdx.y / a.nkv;
    const bool key = blockIdx.z == 0;
    const int n = a.rows.fresh(b), len = a.rows.cached(b);
    const int moved = min(max(a.n_kept[b], 0), n);
    if (a.new_len && tid == 0 && key && blockIdx.y % a.nkv == 0) a.new_len[b] = len + moved;
    const size_t first = (size_t)blockIdx.y * a.max_seq + len;
    char *rows = (key ? a.k : a.v) + first * a.row_bytes;
    float *scale = key ? a.k_scale : a.v_scale;
    const int32_t *kept = a.kept + (size_t)b * a.rows.tokens;
    const int per = a.row_bytes / 16;                              // 4, 8 or 16 pieces of a row
    for (int e = tid; e < moved * per; e += NT) {
        const int from = min(max(kept[e / per], 0), n - 1);
        *reinterpret_cast<u32x4 *>(held + 16 * e) = *reinterpret_cast<const u32x4 *>(rows + (size_t)from * a.row_bytes + 16 * (e % per));
    }
    const float own_scale = scale && tid < moved ? scale[first + min(max(kept[tid], 0), n - 1)] : 0.f;
    __syncthreads();
    for (int e = tid; e < moved * per; e += NT) *reinterpret_cast<u32x4 *>(rows + 16 * (size_t)e) = *reinterpret_cast<const u32x4 *>(held + 16 * e);
    if (scale && tid < moved) scale[first + tid] = own_scale;
}
static_assert(kMaxKept <= NT, "a thread per scale");

// ---- launches --------------------------------------------------------------------------------------------------------------

template <typename Args>
using Kernel = void (*)(const Args);
Kernel<AppendArgs> pick_append(int hd, int fmt)
{
    if (hd == 64) return fmt == CF_CACHE_F16 ? cache_append<64, CF_CACHE_F16> : fmt == CF_CACHE_E4M3 ? cache_append<64, CF_CACHE_E4M3> : cache_append<64, CF_CACHE_INT8>;
    return fmt == CF_CACHE_F16 ? cache_append<128, CF_CACHE_F16> : fmt == CF_CACHE_E4M3 ? cache_append<128, CF_CACHE_E4M3> : cache_append<128, CF_CACHE_INT8>;
}
Kernel<ReadArgs> pick_read(int hd, int fmt)
{
    if (hd == 64) return fmt == CF_CACHE_F16 ? cache_read<64, CF_CACHE_F16> : fmt == CF_CACHE_E4M3 ? cache_read<64, CF_CACHE_E4M3> : cache_read<64, CF_CACHE_INT8>;
    return fmt == CF_CACHE_F16 ? cache_read<128, CF_CACHE_F16> : fmt == CF_CACHE_E4M3 ? cache_read<128, CF_CACHE_E4M3> : cache_read<128, CF_CACHE_INT8>;
}

int launched() { return hipGetLastError() == hipSuccess ? CF_OK : CF_EHIP; }

}  // namespace

extern "C" {

int cf_cache_append(const cf_cache_config *cfg, int32_t batch, const void *qkv, const cf_cache *cache, const cf_draft *draft,
                    void *q_out, void *stream)
{
    if (!cfg) return CF_EINVAL;
    int rc = check_config(*cfg);
    if (rc == CF_OK) rc = check_cache(*cfg, cache, batch);
    if (rc == CF_OK) rc = check_draft(*cfg, draft);
    if (rc != CF_OK) return rc;
    if (!qkv || !q_out || !aligned(qkv, 16) || !aligned(q_out, 16)) return CF_EINVAL;
    const size_t head_values = (size_t)batch * draft->tokens * cfg->head_dim;
    const size_t qkv_bytes = 2 * head_values * (cfg->n_q_heads + 2 * (size_t)cfg->n_kv_heads), q_bytes = 2 * head_values * cfg->n_q_heads;
    if (overlap(qkv, qkv_bytes, q_out, q_bytes) || in_cache(*cfg, *cache, batch, qkv, qkv_bytes) ||
        in_cache(*cfg, *cache, batch, q_out, q_bytes) || tangled(*cfg, *cache, batch))
        return CF_EINVAL;
    AppendArgs a;
    std::memset(&a, 0, sizeof a);
    a.qkv = static_cast<const uint16_t *>(qkv);
    a.q_out = static_cast<uint16_t *>(q_out);
    a.k = static_cast<char *>(cache->k), a.v = static_cast<char *>(cache->v);
    a.k_scale = cache->k_scale, a.v_scale = cache->v_scale;
    a.rows = lengths_of(*draft);
    a.depth = draft->depth, a.depth_stride = draft->per_row ? draft->tokens : 0;
    a.nq = cfg->n_q_heads, a.nkv = cfg->n_kv_heads, a.max_seq = cfg->max_seq;
    // theta_(8 i + j) = theta_(8 i) theta_j, off by 2^-51.4 of it at most (three half steps; a power alone by one): 16 powers on the host in place
    // of 64 (one token 6.8 us a call, 7.2 with 64)
    double of_eight[8], in_eight[8];
    for (int i = 0; i < 8; ++i) {
        of_eight[i] = std::pow((double)cfg->rope_base, -16.0 * i / cfg->head_dim);
        in_eight[i] = std::pow((double)cfg->rope_base, -2.0 * i / cfg->head_dim);
    }
    for (int i = 0; i < cfg->head_dim / 2; ++i) a.theta[i] = of_eight[i / 8] * in_eight[i % 8];
    // Four tokens to a workgroup, a wavefront each, or one token whose heads are spread over all wavefronts of several workgroups.
    const int heads = a.nq + 2 * a.nkv, groups = (heads * cfg->head_dim / 16 + 63) / 64;
    a.nt = (long long)batch * draft->tokens >= 2048 ? 4 : 1;
    const int chunks = a.nt == 4 ? 1 : (groups + NW - 1) / NW;
    hipLaunchKernelGGL(pick_append(cfg->head_dim, cfg->format), dim3((draft->tokens + a.nt - 1) / a.nt, chunks, batch), dim3(NT), 0,
                       static_cast<hipStream_t>(stream), a);
    return launched();
}

int cf_cache_read(const cf_cache_config *cfg, int32_t batch, const cf_cache *cache, int32_t first, int32_t rows, void *k_out,
                  void *v_out, void *stream)
{
    if (!cfg) return CF_EINVAL;
    int rc = check_config(*cfg);
    if (rc == CF_OK) rc = check_cache(*cfg, cache, batch);
    if (rc != CF_OK) return rc;
    if (!k_out || !v_out || !aligned(k_out, 16) || !aligned(v_out, 16) || first < 0 || rows < 0 || (long long)first + rows > cfg->max_seq)
        return CF_EINVAL;
    if (rows == 0) return CF_OK;
    const size_t out_bytes = 2 * (size_t)batch * cfg->n_kv_heads * rows * cfg->head_dim;
    if (overlap(k_out, out_bytes, v_out, out_bytes) || in_cache(*cfg, *cache, batch, k_out, out_bytes) ||
        in_cache(*cfg, *cache, batch, v_out, out_bytes))
        return CF_EINVAL;
    ReadArgs a;
    std::memset(&a, 0, sizeof a);
    a.k = static_cast<const char *>(cache->k), a.v = static_cast<const char *>(cache->v);
    a.k_scale = cache->k_scale, a.v_scale = cache->v_scale;
    a.k_out = static_cast<uint16_t *>(k_out), a.v_out = static_cast<uint16_t *>(v_out);
    a.max_seq = cfg->max_seq, a.first = first, a.rows = rows;
    const uint32_t pieces = (uint32_t)rows * (cfg->head_dim / 16), per = NT * kReadPieces;
    hipLaunchKernelGGL(pick_read(cfg->head_dim, cfg->format), dim3((pieces + per - 1) / per, batch * cfg->n_kv_heads, 2), dim3(NT), 0,
                       static_cast<hipStream_t>(stream), a);
    return launched();
}

int cf_cache_keep(const cf_cache_config *cfg, int32_t batch, const cf_cache *cache, const cf_draft *draft, const int32_t *kept,
                  const int32_t *n_kept, int32_t *new_len, void *stream)
{
    if (!cfg) return CF_EINVAL;
    int rc = check_config(*cfg);
    if (rc == CF_OK) rc = check_cache(*cfg, cache, batch);
    if (rc == CF_OK) rc = check_draft(*cfg, draft);
    if (rc != CF_OK) return rc;
    if (!kept || !n_kept || !aligned(kept, 4) || !aligned(n_kept, 4) || !aligned(new_len, 4)) return CF_EINVAL;
    const size_t a_row = 4 * (size_t)batch;                         // bytes of an int32 for every batch row
    if (new_len && ((draft->row_len && overlap(new_len, a_row, draft->row_len, a_row)) ||
                    (draft->row_tokens && overlap(new_len, a_row, draft->row_tokens, a_row)) || overlap(new_len, a_row, n_kept, a_row) ||
                    overlap(new_len, a_row, kept, a_row * draft->tokens) || in_cache(*cfg, *cache, batch, new_len, a_row)))
        return CF_EINVAL;
    if (tangled(*cfg, *cache, batch)) return CF_EINVAL;
    if (draft->tokens > kMaxKept) return CF_EUNSUPPORTED;
    KeepArgs a;
    std::memset(&a, 0, sizeof a);
    a.k = static_cast<char *>(cache->k), a.v = static_cast<char *>(cache->v);
    if (cfg->format != CF_CACHE_F16) a.k_scale = cache->k_scale, a.v_scale = cache->v_scale;
    a.rows = lengths_of(*draft);
    a.kept = kept, a.n_kept = n_kept, a.new_len = new_len;
    a.nkv = cfg->n_kv_heads, a.max_seq = cfg->max_seq;
    a.row_bytes = cfg->head_dim * (cfg->format == CF_CACHE_F16 ? 2 : 1);
    hipLaunchKernelGGL(cache_keep, dim3(1, batch * cfg->n_kv_heads, 2), dim3(NT), (size_t)draft->tokens * a.row_bytes,
                       static_cast<hipStream_t>(stream), a);
    return launched();
}

}  // extern "C"
