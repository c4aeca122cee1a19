// Operands of the matrix products of the tree attention (cf_tree.hip) from a key/value cache in one of its formats.
//
// Both products are taken transposed, so that a lane of 16 g + c has to do with one row c of queries throughout:
//   S^T = K Q^T   16 keys x 16 queries a tile: A = keys, B = queries; the lane gets the scores of its query for keys 4 g .. 4 g + 3
//   O^T = V^T P^T 16 dimensions x 16 queries: A = values, B = weights; the contraction runs over 32 keys in the order in which the
//                 scores of two tiles lie in the lane (keys 4 g .. 4 g + 3 and 16 + 4 g .. 16 + 4 g + 3), so that no weight moves
// NJ = HD / 16 adjacent dimensions of a value row to a lane: dimension NJ c + jj is row c of the jj-th product.
#ifndef CF_TREE_DEVICE_H
#define CF_TREE_DEVICE_H

#include "cf_cache_device.h"
#include "cf_mfma_device.h"
#include "cf_stream_device.h"

namespace cf {
namespace tree {

using cf::mfma::f32x4;
using cf::mfma::h8;
using cf::mfma::mfma16;
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));

// fp16 pair of two codes in the low bytes of the halves.  int8 codes come with their top bit flipped (0 .. 255): such a half is the
// fp16 number code * 2^-24, and one multiply-add makes it (code - 128) * 2^-9, exactly.
constexpr float kInt8Unit = 512.f;          // what a code's operand has to be multiplied with
__device__ __forceinline__ uint32_t pair_of_int8(uint32_t x)
{
    const h2 v = __builtin_bit_cast(h2, x) * h2{(_Float16)32768.f, (_Float16)32768.f} + h2{(_Float16)-0.25f, (_Float16)-0.25f};
    return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ uint32_t pair_of_e4m3(uint32_t x, bool high)
{
    const auto v = high ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)x, 1.f, true) : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)x, 1.f, false);
    return __builtin_bit_cast(uint32_t, v);
}

// Infinities and NaN among the values of a dword: the top bit of each such value, and the dword without them.
template <int FMT>
__device__ __forceinline__ uint32_t unfit_bits(uint32_t x)
{
    if constexpr (FMT == CF_CACHE_F16) return ((x & 0x7c007c00u) + 0x04000400u) & 0x80008000u;
    if constexpr (FMT == CF_CACHE_E4M3) return ((x & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;      // (0x7f and 0xff)
    return 0u;
}
template <int FMT>
__device__ __forceinline__ uint32_t without_unfit(uint32_t x)
{
    const uint32_t bad = unfit_bits<FMT>(x);
    return x & ~(FMT == CF_CACHE_F16 ? (bad >> 15) * 0xffffu : (bad >> 7) * 0xffu);
}

// Eight codes as fp16.
template <int FMT>
__device__ __forceinline__ u32x4 widen(uint32_t a, uint32_t b)
{
    u32x4 o;
    if constexpr (FMT == CF_CACHE_INT8) {
        a ^= 0x80808080u, b ^= 0x80808080u;
        o[0] = pair_of_int8(__builtin_amdgcn_perm(0u, a, 0x0c010c00u)), o[1] = pair_of_int8(__builtin_amdgcn_perm(0u, a, 0x0c030c02u));
        o[2] = pair_of_int8(__builtin_amdgcn_perm(0u, b, 0x0c010c00u)), o[3] = pair_of_int8(__builtin_amdgcn_perm(0u, b, 0x0c030c02u));
    } else {
        o[0] = pair_of_e4m3(a, false), o[1] = pair_of_e4m3(a, true);
        o[2] = pair_of_e4m3(b, false), o[3] = pair_of_e4m3(b, true);
    }
    return o;
}

// The keys of a step of 32: requested row by row, 16 bytes a load, used as A operands.
template <int HD, int FMT>
struct Keys {
    static constexpr int KS = HD / 32, LOADS = FMT == CF_CACHE_F16 ? KS : KS / 2, ROW = HD * cache::kValueBytes<FMT>;
    u32x4 raw[2][LOADS];
    // first dimension of what group g holds for contraction step ks
    static __device__ __forceinline__ int dim(int ks, int g) { return FMT == CF_CACHE_F16 ? 32 * ks + 8 * g : 64 * (ks / 2) + 16 * g + 8 * (ks & 1); }
    static __device__ __forceinline__ uint32_t offset(int c, int g) { return (uint32_t)(c * ROW + 16 * g); }
    __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t r, uint32_t off)
    {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < LOADS; ++i)
                raw[t][i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, off + t * (16 * ROW) + 64 * i, 0, 0));
    }
    __device__ __forceinline__ h8 operand(int t, int ks) const
    {
        if constexpr (FMT == CF_CACHE_F16) {
            return __builtin_bit_cast(h8, raw[t][ks]);
        } else {
            const u32x4 x = raw[t][ks / 2];
            return __builtin_bit_cast(h8, widen<FMT>(x[2 * (ks & 1)], x[2 * (ks & 1) + 1]));
        }
    }
};

// The values of a step of 32: NJ adjacent dimensions of eight rows to a lane, transposed in the lane into NJ A operands, two at a time.
template <int HD, int FMT>
struct Values {
    static constexpr int NJ = HD / 16, ROW = HD * cache::kValueBytes<FMT>, DW = NJ * cache::kValueBytes<FMT> / 4;     // dwords of a load: 1, 2 or 4
    uint32_t raw[8][DW];
    static __device__ __forceinline__ int row(int u, int g) { return u < 4 ? 4 * g + u : 12 + 4 * g + u; }
    static __device__ __forceinline__ uint32_t offset(int c, int g) { return (uint32_t)(4 * g * ROW + c * (4 * DW)); }
    __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t r, uint32_t off)
    {
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const uint32_t at = off + (u < 4 ? u : 12 + u) * ROW;
            if constexpr (DW == 4) {
                const u32x4 x = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, at, 0, 0));
#pragma unroll
                for (int w = 0; w < 4; ++w) raw[u][w] = x[w];
            } else if constexpr (DW == 2) {
                const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(r, at, 0, 0));
                raw[u][0] = x[0], raw[u][1] = x[1];
            } else {
                raw[u][0] = __builtin_amdgcn_raw_buffer_load_b32(r, at, 0, 0);
            }
        }
    }
    // the operands of dimensions NJ c + 2 pair and NJ c + 2 pair + 1
    __device__ __forceinline__ void operands(int pair, h8 (&f)[2]) const
    {
        u32x4 o[2];
        if constexpr (FMT == CF_CACHE_F16) {
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                o[0][w] = __builtin_amdgcn_perm(raw[2 * w + 1][pair], raw[2 * w][pair], 0x05040100u);
                o[1][w] = __builtin_amdgcn_perm(raw[2 * w + 1][pair], raw[2 * w][pair], 0x07060302u);
            }
        } else {
            const int word = pair / 2, high = pair & 1;            // two codes of a dword
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                if constexpr (FMT == CF_CACHE_INT8) {
                    const uint32_t lo = raw[2 * w][word], hi = raw[2 * w + 1][word];       // (top bits flipped: flip())
                    o[0][w] = pair_of_int8(__builtin_amdgcn_perm(hi, lo, high ? 0x0c060c02u : 0x0c040c00u));
                    o[1][w] = pair_of_int8(__builtin_amdgcn_perm(hi, lo, high ? 0x0c070c03u : 0x0c050c01u));
                } else {
                    const uint32_t x = __builtin_amdgcn_perm(raw[2 * w + 1][word], raw[2 * w][word], high ? 0x07030602u : 0x05010400u);
                    o[0][w] = pair_of_e4m3(x, false);
                    o[1][w] = pair_of_e4m3(x, true);
                }
            }
        }
        f[0] = __builtin_bit_cast(h8, o[0]), f[1] = __builtin_bit_cast(h8, o[1]);
    }
    // once before the operands of int8 codes
    __device__ __forceinline__ void flip()
    {
        if constexpr (FMT == CF_CACHE_INT8)
#pragma unroll
            for (int u = 0; u < 8; ++u)
#pragma unroll
                for (int w = 0; w < DW; ++w) raw[u][w] ^= 0x80808080u;
    }
    // Takes infinities and NaN (int8 codes have none) out; not 0 if there were some.
    __device__ __forceinline__ uint32_t take_out_unfit()
    {
        uint32_t odd = 0;
#pragma unroll
        for (int u = 0; u < 8; ++u)
#pragma unroll
            for (int w = 0; w < DW; ++w) {
                odd |= unfit_bits<FMT>(raw[u][w]);
                raw[u][w] = without_unfit<FMT>(raw[u][w]);
            }
        return odd;
    }
};

}  // namespace tree
}  // namespace cf

#endif
