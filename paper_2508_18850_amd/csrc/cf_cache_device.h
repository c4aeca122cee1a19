// What the kernels on a key/value cache in one of the formats of cf_cache_config share: lengths of the batch rows, encoding and
// decoding of 8-bit rows, the checks of the arguments.
#ifndef CF_CACHE_DEVICE_H
#define CF_CACHE_DEVICE_H

#include "../../include/cfdecode.h"

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace cf {
namespace cache {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// largest value of a code
template <int FMT>
constexpr float kLargest = FMT == CF_CACHE_INT8 ? 127.f : 448.f;
template <int FMT>
constexpr int kValueBytes = FMT == CF_CACHE_F16 ? 2 : 1;

// The batch rows' lengths (cf_draft without its masks).
struct Lengths {
    const int32_t *row_len, *row_tokens;
    int max_len, tokens;
    __device__ __forceinline__ int cached(int b) const { return row_len ? min(max(row_len[b], 0), max_len) : max_len; }
    __device__ __forceinline__ int fresh(int b) const { return row_tokens ? min(max(row_tokens[b], 0), tokens) : tokens; }
};
inline Lengths lengths_of(const cf_draft &d) { return Lengths{d.row_len, d.row_tokens, d.max_len, d.tokens}; }

inline bool aligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

inline bool overlap(const void *p, size_t p_bytes, const void *q, size_t q_bytes)
{
    const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
    return a < b + q_bytes && b < a + p_bytes;
}

inline int check_config(const cf_cache_config &c)
{
    if (c.n_q_heads < 1 || c.n_kv_heads < 1 || c.n_q_heads % c.n_kv_heads || c.max_batch < 1 || c.max_seq < 1 ||
        (c.format != CF_CACHE_F16 && c.format != CF_CACHE_E4M3 && c.format != CF_CACHE_INT8) || !(c.rope_base > 1.0f) ||
        !(c.rope_base <= 3.402823466e38f))
        return CF_EINVAL;
    if (c.head_dim != 64 && c.head_dim != 128) return CF_EUNSUPPORTED;
    // 32-bit offsets, also in bytes of fp16, inside a head's slice of the cache; head counts that no product of sizes overflows with
    if (1ull * (unsigned)c.max_seq * (unsigned)c.head_dim >= 1ull << 30 || c.n_q_heads > 65535) return CF_EUNSUPPORTED;
    return CF_OK;
}
inline int check_cache(const cf_cache_config &c, const cf_cache *p, int32_t batch)
{
    if (!p || !p->k || !p->v || !aligned(p->k, 16) || !aligned(p->v, 16) || batch < 1 || batch > c.max_batch) return CF_EINVAL;
    if (c.format != CF_CACHE_F16 && (!p->k_scale || !p->v_scale || !aligned(p->k_scale, 4) || !aligned(p->v_scale, 4))) return CF_EINVAL;
    if ((long long)batch * c.n_kv_heads > 65535) return CF_EUNSUPPORTED;      // second dimension of the grids
    return CF_OK;
}
// Whether [x, x + bytes) shares memory with a cache of `batch` rows; whether the cache's own buffers do with each other.
inline size_t cached_rows(const cf_cache_config &c, int32_t batch) { return (size_t)batch * c.n_kv_heads * c.max_seq; }
inline size_t buffer_bytes(const cf_cache_config &c, int32_t batch) { return cached_rows(c, batch) * c.head_dim * (c.format == CF_CACHE_F16 ? 2 : 1); }
inline bool in_cache(const cf_cache_config &c, const cf_cache &p, int32_t batch, const void *x, size_t bytes)
{
    const size_t rows = buffer_bytes(c, batch), scales = 4 * cached_rows(c, batch);
    if (overlap(x, bytes, p.k, rows) || overlap(x, bytes, p.v, rows)) return true;
    return c.format != CF_CACHE_F16 && (overlap(x, bytes, p.k_scale, scales) || overlap(x, bytes, p.v_scale, scales));
}
inline bool tangled(const cf_cache_config &c, const cf_cache &p, int32_t batch)
{
    const size_t rows = buffer_bytes(c, batch), scales = 4 * cached_rows(c, batch);
    if (overlap(p.k, rows, p.v, rows)) return true;
    return c.format != CF_CACHE_F16 && (overlap(p.k_scale, scales, p.v_scale, scales) || overlap(p.k_scale, scales, p.k, rows) ||
                                        overlap(p.k_scale, scales, p.v, rows) || overlap(p.v_scale, scales, p.k, rows) || overlap(p.v_scale, scales, p.v, rows));
}
inline int check_draft(const cf_cache_config &c, const cf_draft *d)
{
    if (!d || d->tokens < 1 || d->max_len < 0 || (long long)d->max_len + d->tokens > c.max_seq) return CF_EINVAL;
    if (!aligned(d->row_len, 4) || !aligned(d->row_tokens, 4) || !aligned(d->depth, 4) || !aligned(d->tree, 8)) return CF_EINVAL;
    return CF_OK;
}

// ---- 8-bit rows ------------------------------------------------------------------------------------------------------------

// Largest magnitude among eight fp16 values, as bits (a NaN or an infinity is 0x7c00 or more, all else less).
__device__ __forceinline__ uint32_t top_bits(h8 v)
{
    typedef uint16_t us8 __attribute__((ext_vector_type(8)));
    const us8 m = __builtin_bit_cast(us8, v) & (uint16_t)0x7fff;
    uint32_t t = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) t = max(t, (uint32_t)m[i]);
    return t;
}

// What turns the values of a row into codes.  The exact quotient x Q / top is either on a border between two codes or at least 2^-19
// of itself away from it (numerators and denominators are whole numbers of at most 11 and 8 bits), so that only the quotients on a
// border have to be exact: y0 = x Q * rcp(top) has an error of 2^-22 at most, and y0 + (x Q - y0 top) * rcp(top), whose bracket the fused
// multiply-add computes without an error, is the quotient itself wherever fp32 holds it.
template <int FMT>
struct Encoder {
    float top, rcp;
    bool usable;
    float scale;
    __device__ __forceinline__ explicit Encoder(uint32_t bits)
    {
        usable = bits > 0 && bits < 0x7c00u;
        top = (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
        rcp = usable ? __builtin_amdgcn_rcpf(top) : 0.f;
        scale = bits < 0x7c00u ? top / kLargest<FMT> : __builtin_nanf("");
    }
    __device__ __forceinline__ float quotient(_Float16 x) const
    {
        const float n = (float)x * kLargest<FMT>;                       // exact: 11 + 7 bits
        const float y = n * rcp;
        return fmaf(fmaf(-y, top, n), rcp, y);
    }
    // eight codes, the first in the lowest byte
    __device__ __forceinline__ u32x2 codes(h8 v) const
    {
        u32x2 c = {0u, 0u};
        if (usable) {
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                const float y0 = quotient(v[4 * w]), y1 = quotient(v[4 * w + 1]), y2 = quotient(v[4 * w + 2]), y3 = quotient(v[4 * w + 3]);
                if constexpr (FMT == CF_CACHE_INT8) {
                    const uint32_t i0 = (uint32_t)(int)rintf(y0), i1 = (uint32_t)(int)rintf(y1), i2 = (uint32_t)(int)rintf(y2), i3 = (uint32_t)(int)rintf(y3);
                    const uint32_t lo = __builtin_amdgcn_perm(i1, i0, 0x0c0c0400u), hi = __builtin_amdgcn_perm(i3, i2, 0x04000c0cu);
                    c[w] = lo | hi;
                } else {
                    int p = __builtin_amdgcn_cvt_pk_fp8_f32(y0, y1, 0, false);
                    c[w] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y2, y3, p, true);
                }
            }
        }
        return c;
    }
};

// Four codes as fp32 (before the scale).
template <int FMT>
__device__ __forceinline__ void decode4(uint32_t c, float (&f)[4])
{
    if constexpr (FMT == CF_CACHE_INT8) {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = (float)((int)(c << (24 - 8 * i)) >> 24);
    } else {
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
        f[0] = lo[0], f[1] = lo[1], f[2] = hi[0], f[3] = hi[1];
    }
}

}  // namespace cache
}  // namespace cf

#endif
