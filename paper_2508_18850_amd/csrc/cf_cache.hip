// A key/value cache in fp16, 8 bits or 4 bits: written with the rotated keys and the values of new tokens, read back as fp16, and its rows of
// accepted tokens moved together (cf_cache_* in include/cfdecode.h).  Three kernels without waits between workgroups.
#include "../../include/cfdecode.h"
#include "cf_cache_device.h"
#include "cf_lanes_device.h"
#include "cf_rope_device.h"

#include <cmath>
#include <cstring>
#include <type_traits>

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
// 10^7; beside memory it costs little where the rarer steps of the roundings are left out (halves_once; two prompts of 4096 tokens, 32 + 2 x 8 heads
// of 128 dimensions, with norms, into fp16: 44.9 us, 57 with all steps for every value and the weights multiplied in head by head).
// With norms (cf_cache_append_normed) every head's row is divided by the root of its mean square, in fp64 too: the squares of fp16 values are exact.
// The weights are multiplied into cos and sin, once for a token and not for each head; a row's norm is common to the pair, so that it comes last.
// Bound: memory; the next heads' rows are requested before these are used (without it 4 % more).  Those prompts: 202 MB in 44.9 us, 4.5 TB/s (a copy
// reaches 5.1); into 4 bits, 177 MB, 40.5 us, 4.4 TB/s.  With few tokens the launch: one token 3.6 us on the GPU, so its heads are spread over more workgroups.
struct AppendArgs {
    const uint16_t *qkv;
    uint16_t *q_out;
    char *k, *v;
    float *k_scale, *v_scale;      // of the 4-bit format: bytes
    const uint16_t *q_weight, *k_weight;   // with norms
    double eps;
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
// The same of N at once.  Rounding twice can only matter where the fp32 value is a middle of two fp16 numbers, and then (or with any other middle
// that fp16's small numbers have) at least its last twelve bits are 0: one value in 4096, else the conversions alone.
template <int N>
__device__ __forceinline__ void halves_once(const double (&x)[N], _Float16 (&h)[N])
{
    uint32_t least = ~0u;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float f = (float)x[i];
        least = min(least, __builtin_bit_cast(uint32_t, f) & 0xfffu);
        h[i] = (_Float16)f;
    }
    if (__any(least == 0))
#pragma unroll
        for (int i = 0; i < N; ++i) h[i] = half_once(x[i]);
}

template <int HD>
__device__ __forceinline__ uint32_t row_top(uint32_t t)      // largest of the HD / 16 lanes that hold a row
{
    t = max(t, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)t, 0xB1, 0xF, 0xF, true));        // lane ^ 1
    t = max(t, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)t, 0x4E, 0xF, 0xF, true));        // lane ^ 2
    return HD == 64 ? t : max(t, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)t, 0x141, 0xF, 0xF, true));   // 7 - lane
}

// of the four lanes that hold a block of the 4-bit format
__device__ __forceinline__ uint32_t block_top(uint32_t t)
{
    t = max(t, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)t, 0xB1, 0xF, 0xF, true));
    return max(t, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)t, 0x4E, 0xF, 0xF, true));
}

template <int CTRL>
__device__ __forceinline__ double moved(double x)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, 0xF, 0xF, true);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), CTRL, 0xF, 0xF, true);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// 1 / sqrt(mean of the squares of a row + eps), in fp64: the squares of fp16 values are exact, their sum is off by HD half steps of 2^-53, and two
// Newton steps take the approximation of v_rsq_f64 (2^-26 or better) to 2^-51.
template <int HD>
__device__ __forceinline__ double row_norm(const h8 &lo, const h8 &hi, double eps)
{
    double s = 0.0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const double x = (double)(float)lo[j], y = (double)(float)hi[j];
        s = fma(x, x, s);
        s = fma(y, y, s);
    }
    s += moved<0xB1>(s);
    s += moved<0x4E>(s);
    if constexpr (HD == 128) s += moved<0x141>(s);
    const double m = s * (1.0 / HD) + eps;
    double r = __builtin_amdgcn_rsq(m);
#pragma unroll
    for (int i = 0; i < 2; ++i) r = fma(0.5 * r, fma(-m * r, r, 1.0), r);
    return m == (double)INFINITY ? 0.0 : r;
}

// The pair (x, y) of a rotation becomes (x xx - y yx, y yy + x xy): cos, sin, cos, sin, with norms each times the weight of what it is multiplied by.
struct alignas(16) Turn {
    double xx, yx;
};
struct alignas(16) WeightedTurn {
    double xx, yx, yy, xy;
};
template <int HD, int FMT, bool NORM>
__global__ __launch_bounds__(NT) void cache_append(const AppendArgs a)
{
    constexpr int LPR = HD / 16, RPW = 64 / LPR, HALF = HD / 2, KINDS = NORM ? 2 : 1;
    // of a token's pair 8 i + j at j LPR + i, so that the lanes of a row read adjacent ones; with norms for queries and for keys
    __shared__ std::conditional_t<NORM, WeightedTurn, Turn> turn[4][KINDS][HALF];
    const int tid = threadIdx.x, wv = tid >> 6, lane = tid & 63;
    const int b = blockIdx.z, t0 = blockIdx.x * a.nt;
    const int n = a.rows.fresh(b), len = a.rows.cached(b);
    if (t0 >= n) return;
    {
        const int slot = tid / 64, i = lane, at = i % 8 * LPR + i / 8;
        if (slot < a.nt && i < HALF && t0 + slot < n) {
            const int depth = a.depth ? a.depth[(size_t)b * a.depth_stride + t0 + slot] : t0 + slot;
            double c, s;
            if constexpr (NORM) {
                double w[2][2];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const uint16_t *of = k ? a.k_weight : a.q_weight;
                    w[k][0] = (double)(float)__builtin_bit_cast(_Float16, of[i]), w[k][1] = (double)(float)__builtin_bit_cast(_Float16, of[i + HALF]);
                }
                cf::rope_cos_sin64((double)len + (double)depth, a.theta[i], c, s);
#pragma unroll
                for (int k = 0; k < 2; ++k) turn[slot][k][at] = {c * w[k][0], s * w[k][1], c * w[k][1], s * w[k][0]};
            } else {
                cf::rope_cos_sin64((double)len + (double)depth, a.theta[i], c, s);
                turn[slot][0][at] = {c, s};
            }
        }
    }
    __syncthreads();
    const int slot = wv % a.nt, t = t0 + slot;
    if (t >= n) return;
    const int H = a.nq + 2 * a.nkv, groups = (H + RPW - 1) / RPW, step = (NW / a.nt) * gridDim.y;
    const int li = lane % LPR;
    const uint16_t *src = a.qkv + ((size_t)b * a.rows.tokens + t) * H * HD + 8 * li;
    int grp = wv / a.nt + (NW / a.nt) * blockIdx.y;
    h8 next_lo = {}, next_hi = {};
    auto load = [&](int of) {
        const int head = of * RPW + lane / LPR;
        if (head < H) next_lo = *reinterpret_cast<const h8 *>(src + (size_t)head * HD), next_hi = *reinterpret_cast<const h8 *>(src + (size_t)head * HD + HALF);
    };
    load(grp);
    for (; grp < groups; grp += step) {
        const int head = grp * RPW + lane / LPR;
        h8 lo = next_lo, hi = next_hi;
        load(grp + step);
        if (head >= H) continue;                                   // (whole rows of lanes: the maxima below stay inside a row)
        if (head < a.nq + a.nkv) {
            const auto *turns = turn[slot][NORM && head >= a.nq] + li;
            double r = 1.0;
            if constexpr (NORM) r = row_norm<HD>(lo, hi, a.eps);
#pragma unroll
            for (int j0 = 0; j0 < 8; j0 += 2) {
                double z[4];
                _Float16 h[4];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const auto cs = turns[(j0 + j) * LPR];
                    const double x = (double)(float)lo[j0 + j], y = (double)(float)hi[j0 + j];
                    if constexpr (NORM) {
                        z[j] = (x * cs.xx - y * cs.yx) * r;
                        z[2 + j] = (y * cs.yy + x * cs.xy) * r;
                    } else {
                        z[j] = x * cs.xx - y * cs.yx;
                        z[2 + j] = y * cs.xx + x * cs.yx;
                    }
                }
                halves_once(z, h);
#pragma unroll
                for (int j = 0; j < 2; ++j) lo[j0 + j] = h[j], hi[j0 + j] = h[2 + j];
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
        char *dst = (key ? a.k : a.v) + row * bytes_of<FMT>(HD) + bytes_of<FMT>(8) * li;
        if constexpr (FMT == CF_CACHE_F16) {
            *reinterpret_cast<h8 *>(dst) = lo;
            *reinterpret_cast<h8 *>(dst + 2 * HALF) = hi;
        } else if constexpr (FMT == CF_CACHE_MXFP4) {
            const uint32_t slo = block_scale(block_top(top_bits(lo))), shi = block_scale(block_top(top_bits(hi)));
            *reinterpret_cast<uint32_t *>(dst) = block_codes(lo, slo);
            *reinterpret_cast<uint32_t *>(dst + HALF / 2) = block_codes(hi, shi);
            if (li % 4 == 0) {
                uint8_t *scale = reinterpret_cast<uint8_t *>(key ? a.k_scale : a.v_scale) + row * (HD / kBlock) + li / 4;
                scale[0] = (uint8_t)slo, scale[HALF / kBlock] = (uint8_t)shi;
            }
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
    const char *src = (key ? a.k : a.v) + slice * bytes_of<FMT>(HD);
    const float *scale = (key ? a.k_scale : a.v_scale) + (FMT == CF_CACHE_F16 || FMT == CF_CACHE_MXFP4 ? 0 : slice);
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
    } else if constexpr (FMT == CF_CACHE_MXFP4) {
        const uint8_t *power = reinterpret_cast<const uint8_t *>(scale) + slice * (HD / kBlock);
        u32x2 x[kReadPieces];
        uint32_t s[kReadPieces];
#pragma unroll
        for (int i = 0; i < kReadPieces; ++i)
            if (at + NT * i < pieces) {
                x[i] = *reinterpret_cast<const u32x2 *>(src + (size_t)(at + NT * i) * 8);
                s[i] = power[(at + NT * i) / 2];
            }
#pragma unroll
        for (int i = 0; i < kReadPieces; ++i)
            if (at + NT * i < pieces)
#pragma unroll
                for (int w = 0; w < 2; ++w) *reinterpret_cast<u32x4 *>(dst + (size_t)(at + NT * i) * 16 + 8 * w) = block_values(x[i][w], scale_of_byte(s[i]));
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
    char *k_scale, *v_scale;
    Lengths rows;
    const int32_t *kept, *n_kept;
    int32_t *new_len;
    int nkv, max_seq, row_bytes;
    int scale_bytes;               // of a row's scales: 0, 2 or 4
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
    char *scale = (key ? a.k_scale : a.v_scale) + first * a.scale_bytes;
    const int32_t *kept = a.kept + (size_t)b * a.rows.tokens;
    const int per = a.row_bytes / 16;                              // 2, 4, 8 or 16 pieces of a row
    for (int e = tid; e < moved * per; e += NT) {
        const int from = min(max(kept[e / per], 0), n - 1);
        *reinterpret_cast<u32x4 *>(held + 16 * e) = *reinterpret_cast<const u32x4 *>(rows + (size_t)from * a.row_bytes + 16 * (e % per));
    }
    const bool scales = a.scale_bytes != 0 && tid < moved;         // (without them nothing more is read before the barrier)
    uint32_t own_scale = 0;
    if (scales) {
        const int mine = min(max(kept[tid], 0), n - 1);
        own_scale = a.scale_bytes == 4 ? reinterpret_cast<const uint32_t *>(scale)[mine] : reinterpret_cast<const uint16_t *>(scale)[mine];
    }
    __syncthreads();
    for (int e = tid; e < moved * per; e += NT) *reinterpret_cast<u32x4 *>(rows + 16 * (size_t)e) = *reinterpret_cast<const u32x4 *>(held + 16 * e);
    if (scales && a.scale_bytes == 4) reinterpret_cast<uint32_t *>(scale)[tid] = own_scale;
    if (scales && a.scale_bytes == 2) reinterpret_cast<uint16_t *>(scale)[tid] = (uint16_t)own_scale;
}
static_assert(kMaxKept <= NT, "a thread per scale");

// ---- launches --------------------------------------------------------------------------------------------------------------

template <typename Args>
using Kernel = void (*)(const Args);
template <int HD, bool NORM>
Kernel<AppendArgs> pick_append_of(int fmt)
{
    return fmt == CF_CACHE_F16 ? cache_append<HD, CF_CACHE_F16, NORM> : fmt == CF_CACHE_E4M3 ? cache_append<HD, CF_CACHE_E4M3, NORM> :
           fmt == CF_CACHE_INT8 ? cache_append<HD, CF_CACHE_INT8, NORM> : cache_append<HD, CF_CACHE_MXFP4, NORM>;
}
Kernel<AppendArgs> pick_append(int hd, int fmt, bool norm)
{
    if (hd == 64) return norm ? pick_append_of<64, true>(fmt) : pick_append_of<64, false>(fmt);
    return norm ? pick_append_of<128, true>(fmt) : pick_append_of<128, false>(fmt);
}
template <int HD>
Kernel<ReadArgs> pick_read_of(int fmt)
{
    return fmt == CF_CACHE_F16 ? cache_read<HD, CF_CACHE_F16> : fmt == CF_CACHE_E4M3 ? cache_read<HD, CF_CACHE_E4M3> :
           fmt == CF_CACHE_INT8 ? cache_read<HD, CF_CACHE_INT8> : cache_read<HD, CF_CACHE_MXFP4>;
}
Kernel<ReadArgs> pick_read(int hd, int fmt) { return hd == 64 ? pick_read_of<64>(fmt) : pick_read_of<128>(fmt); }

int launched() { return hipGetLastError() == hipSuccess ? CF_OK : CF_EHIP; }

// cf_cache_append, and cf_cache_append_normed where there are weights (norm).
int append(const cf_cache_config *cfg, int32_t batch, const void *qkv, bool norm, const void *q_weight, const void *k_weight, float eps,
           const cf_cache *cache, const cf_draft *draft, void *q_out, void *stream)
{
    if (!cfg) return CF_EINVAL;
    int rc = check_config(*cfg);
    if (rc == CF_OK) rc = check_cache(*cfg, cache, batch);
    if (rc == CF_OK) rc = check_draft(*cfg, draft);
    if (rc != CF_OK) return rc;
    if (!qkv || !q_out || !aligned(qkv, 16) || !aligned(q_out, 16)) return CF_EINVAL;
    if (norm && (!q_weight || !k_weight || !aligned(q_weight, 16) || !aligned(k_weight, 16) || !(eps >= 0.f) || !(eps <= 3.402823466e38f))) return CF_EINVAL;
    const size_t head_values = (size_t)batch * draft->tokens * cfg->head_dim;
    const size_t qkv_bytes = 2 * head_values * (cfg->n_q_heads + 2 * (size_t)cfg->n_kv_heads), q_bytes = 2 * head_values * cfg->n_q_heads;
    if (overlap(qkv, qkv_bytes, q_out, q_bytes) || in_cache(*cfg, *cache, batch, qkv, qkv_bytes) ||
        in_cache(*cfg, *cache, batch, q_out, q_bytes) || tangled(*cfg, *cache, batch))
        return CF_EINVAL;
    const size_t weight_bytes = 2 * (size_t)cfg->head_dim;
    if (norm && (overlap(q_weight, weight_bytes, q_out, q_bytes) || overlap(k_weight, weight_bytes, q_out, q_bytes) ||
                 in_cache(*cfg, *cache, batch, q_weight, weight_bytes) || in_cache(*cfg, *cache, batch, k_weight, weight_bytes)))
        return CF_EINVAL;
    AppendArgs a;
    std::memset(&a, 0, sizeof a);
    a.qkv = static_cast<const uint16_t *>(qkv);
    a.q_out = static_cast<uint16_t *>(q_out);
    a.k = static_cast<char *>(cache->k), a.v = static_cast<char *>(cache->v);
    a.k_scale = cache->k_scale, a.v_scale = cache->v_scale;
    a.q_weight = static_cast<const uint16_t *>(q_weight), a.k_weight = static_cast<const uint16_t *>(k_weight), a.eps = eps;
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
    hipLaunchKernelGGL(pick_append(cfg->head_dim, cfg->format, norm), dim3((draft->tokens + a.nt - 1) / a.nt, chunks, batch), dim3(NT), 0,
                       static_cast<hipStream_t>(stream), a);
    return launched();
}

}  // namespace

extern "C" {

int cf_cache_append(const cf_cache_config *cfg, int32_t batch, const void *qkv, const cf_cache *cache, const cf_draft *draft,
                    void *q_out, void *stream)
{
    return append(cfg, batch, qkv, false, nullptr, nullptr, 0.f, cache, draft, q_out, stream);
}

int cf_cache_append_normed(const cf_cache_config *cfg, int32_t batch, const void *qkv, const void *q_weight, const void *k_weight, float eps,
                           const cf_cache *cache, const cf_draft *draft, void *q_out, void *stream)
{
    return append(cfg, batch, qkv, true, q_weight, k_weight, eps, cache, draft, q_out, stream);
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
    a.k_scale = reinterpret_cast<char *>(cache->k_scale), a.v_scale = reinterpret_cast<char *>(cache->v_scale);
    a.scale_bytes = row_scale_bytes(*cfg);
    a.rows = lengths_of(*draft);
    a.kept = kept, a.n_kept = n_kept, a.new_len = new_len;
    a.nkv = cfg->n_kv_heads, a.max_seq = cfg->max_seq;
    a.row_bytes = row_bytes(*cfg);
    hipLaunchKernelGGL(cache_keep, dim3(1, batch * cfg->n_kv_heads, 2), dim3(NT), (size_t)draft->tokens * a.row_bytes,
                       static_cast<hipStream_t>(stream), a);
    return launched();
}

}  // extern "C"
