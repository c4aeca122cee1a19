// Rows quantised to 8-bit integers, and the product of such rows with weights quantised by output channel (cf_linear_* in include/cfdecode.h).
#include "../../include/cfdecode.h"
#include "cf_cache_device.h"
#include "cf_lanes_device.h"

#include <algorithm>
#include <cstring>
#include <new>

namespace {

using cf::cache::aligned;
using cf::cache::overlap;
using cf::cache::h8;
using cf::cache::u32x2;
using cf::cache::u32x4;
typedef int i32x4 __attribute__((ext_vector_type(4)));

// ---- rows to codes -----------------------------------------------------------------------------------------------------------
//
// The row in registers, 8 values to a piece: its largest magnitude, then the codes (cf::cache::Encoder: the correctly rounded quotients).
constexpr int kPieces = 8;         // pieces of a thread that stay in registers

template <int T>
__global__ __launch_bounds__(T) void quantize_rows(const uint16_t *x, int8_t *codes, float *scale, int n)
{
    __shared__ uint32_t tops[T / 64];
    const int tid = threadIdx.x, pieces = n / 8;
    const uint16_t *src = x + (size_t)blockIdx.x * n;
    int8_t *dst = codes + (size_t)blockIdx.x * n;
    h8 v[kPieces];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
        const int at = tid + T * i;
        v[i] = *reinterpret_cast<const h8 *>(src + 8 * (size_t)min(at, pieces - 1));
        top = max(top, cf::cache::top_bits(v[i]));
    }
    for (int at = tid + T * kPieces; at < pieces; at += T) top = max(top, cf::cache::top_bits(*reinterpret_cast<const h8 *>(src + 8 * (size_t)at)));
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, s));
    if constexpr (T > 64) {
        if (tid % 64 == 0) tops[tid / 64] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < T / 64; ++w) top = max(top, tops[w]);
    }
    const cf::cache::Encoder<CF_CACHE_INT8> enc(top);
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
        const int at = tid + T * i;
        if (at < pieces) *reinterpret_cast<u32x2 *>(dst + 8 * (size_t)at) = enc.codes(v[i]);
    }
    for (int at = tid + T * kPieces; at < pieces; at += T)
        *reinterpret_cast<u32x2 *>(dst + 8 * (size_t)at) = enc.codes(*reinterpret_cast<const h8 *>(src + 8 * (size_t)at));
    if (tid == 0) scale[blockIdx.x] = enc.scale;
}

// ---- the product -------------------------------------------------------------------------------------------------------------
//
// 16 x 16 x 64 steps of the matrix units, 32-bit sums (exact: 2^31 / 127^2 codes and more).  Operands, lane = 16 g + c: row c, codes 16 g .. 16 g + 15.
struct LinearArgs {
    const int8_t *x, *w;
    const float *x_scale, *w_scale;
    uint16_t *out;
    int rows, n_in, n_out;
};

// A sum times its scales, as fp16.  The fp32 product is made first (the compiler would put it and the conversion into one instruction, which rounds
// once, in some kernels and not in others).
__device__ __forceinline__ _Float16 scaled(int sum, float sx, float sw)
{
    float y = (float)sum * sx * sw;
    asm("" : "+v"(y));
    return (_Float16)y;
}

// A wavefront takes 16 rows by 64 outputs, its operands straight from memory.
__global__ __launch_bounds__(256) void linear_simple(const LinearArgs a)
{
    const int wv = threadIdx.x >> 6, lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
    const int m0 = blockIdx.y * 16, n0 = (blockIdx.x * 4 + wv) * 64;
    if (n0 >= a.n_out) return;
    const int8_t *xr = a.x + (size_t)min(m0 + c, a.rows - 1) * a.n_in;
    const int8_t *wr[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) wr[j] = a.w + (size_t)min(n0 + 16 * j + c, a.n_out - 1) * a.n_in;
    i32x4 sum[4] = {};
    for (int k0 = 0; k0 < a.n_in; k0 += 64) {
        const int k = k0 + 16 * g, at = min(k, a.n_in - 16);
        const i32x4 none = {0, 0, 0, 0};
        const i32x4 xv = k < a.n_in ? *reinterpret_cast<const i32x4 *>(xr + at) : none;
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(*reinterpret_cast<const i32x4 *>(wr[j] + at), xv, sum[j], 0, 0, 0);
    }
    const int m = m0 + c;
    if (m >= a.rows) return;
    const float sx = a.x_scale[m];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int n = n0 + 16 * j + 4 * g + r;
            if (n < a.n_out) a.out[(size_t)m * a.n_out + n] = __builtin_bit_cast(uint16_t, scaled(sum[j][r], sx, a.w_scale[n]));
        }
}

constexpr int kMostRows = 1 << 23;         // workgroups of a launch
constexpr int kMostIn = 131056;            // 128^2 times as many is below 2^31

int check_linear(const cf_linear_config &c)
{
    if (c.n_in < 16 || c.n_in % 16 || c.n_out < 8 || c.n_out % 8 || c.max_rows < 1) return CF_EINVAL;
    if (c.n_in > kMostIn || c.max_rows > kMostRows || (unsigned long long)c.n_in * c.n_out >= 1ull << 31) return CF_EUNSUPPORTED;
    return CF_OK;
}

}  // namespace

struct cf_linear_s {
    cf_linear_config cfg;
    int device = 0, cus = 0;
};

extern "C" {

int cf_linear_quantize(int32_t rows, int32_t n, const void *x, int8_t *codes, float *scale, void *stream)
{
    if (rows < 0 || n < 16 || n % 16) return CF_EINVAL;
    if (rows > kMostRows) return CF_EUNSUPPORTED;
    if (!x || !codes || !scale || !aligned(x, 16) || !aligned(codes, 16) || !aligned(scale, 4)) return CF_EINVAL;
    const size_t values = (size_t)rows * n;
    if (rows == 0) return CF_OK;
    if (overlap(x, 2 * values, codes, values) || overlap(x, 2 * values, scale, 4 * (size_t)rows) || overlap(codes, values, scale, 4 * (size_t)rows)) return CF_EINVAL;
    const auto *src = static_cast<const uint16_t *>(x);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (n <= 64 * 8 * kPieces)
        hipLaunchKernelGGL(quantize_rows<64>, dim3(rows), dim3(64), 0, s, src, codes, scale, n);
    else
        hipLaunchKernelGGL(quantize_rows<256>, dim3(rows), dim3(256), 0, s, src, codes, scale, n);
    return hipGetLastError() == hipSuccess ? CF_OK : CF_EHIP;
}

int cf_linear_create(const cf_linear_config *cfg, cf_linear *out)
{
    if (!cfg || !out) return CF_EINVAL;
    *out = nullptr;
    const int rc = check_linear(*cfg);
    if (rc != CF_OK) return rc;
    int dev = 0, cus = 0;
    if (hipGetDevice(&dev) != hipSuccess || hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cus < 1)
        return CF_EHIP;
    cf_linear t = new (std::nothrow) cf_linear_s();
    if (!t) return CF_ENOMEM;
    t->cfg = *cfg;
    t->device = dev, t->cus = cus;
    *out = t;
    return CF_OK;
}

int cf_linear_destroy(cf_linear t)
{
    if (!t) return CF_EINVAL;
    delete t;
    return CF_OK;
}

int cf_linear_forward(cf_linear t, int32_t rows, const int8_t *x, const float *x_scale, const int8_t *W, const float *w_scale, void *out,
                      void *stream)
{
    if (!t) return CF_EINVAL;
    const cf_linear_config &c = t->cfg;
    if (rows < 1 || rows > c.max_rows) return CF_EINVAL;
    if (!x || !x_scale || !W || !w_scale || !out || !aligned(x, 16) || !aligned(W, 16) || !aligned(out, 16) || !aligned(x_scale, 4) || !aligned(w_scale, 4)) return CF_EINVAL;
    const size_t out_bytes = 2 * (size_t)rows * c.n_out;
    if (overlap(out, out_bytes, x, (size_t)rows * c.n_in) || overlap(out, out_bytes, W, (size_t)c.n_out * c.n_in) || overlap(out, out_bytes, x_scale, 4 * (size_t)rows) ||
        overlap(out, out_bytes, w_scale, 4 * (size_t)c.n_out))
        return CF_EINVAL;
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess) return CF_EHIP;
    if (dev != t->device) return CF_EINVAL;
    LinearArgs a = {x, W, x_scale, w_scale, static_cast<uint16_t *>(out), rows, c.n_in, c.n_out};
    hipLaunchKernelGGL(linear_simple, dim3((c.n_out + 255) / 256, (rows + 15) / 16), dim3(256), 0, static_cast<hipStream_t>(stream), a);
    return hipGetLastError() == hipSuccess ? CF_OK : CF_EHIP;
}

int64_t cf_linear_algorithmic_bytes(const cf_linear_config *cfg, int32_t rows)
{
    if (!cfg) return 0;
    const int64_t m = rows, k = cfg->n_in, n = cfg->n_out;
    return m * k + n * k + 4 * (m + n) + 2 * m * n;
}

}  // extern "C"
