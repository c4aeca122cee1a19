// Rows quantised to 8-bit integers, and the product of such rows with weights quantised by output channel (cf_linear_* in include/cfdecode.h).
#include "../../include/cfdecode.h"
#include "cf_cache_device.h"
#include "cf_lanes_device.h"
#include "cf_linear_plan.h"
#include "cf_stream_device.h"

#include <cstring>
#include <new>

namespace {

using cf::cache::aligned;
using cf::cache::overlap;
using cf::cache::h8;
using cf::cache::u32x2;
using cf::cache::u32x4;
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 h4 __attribute__((ext_vector_type(4)));

// ---- rows to codes -----------------------------------------------------------------------------------------------------------
//
// The row in registers, 8 values to a piece: its largest magnitude, then the codes (cf::cache::Encoder: the correctly rounded quotients).  Rows of up
// to 4096 values have a wavefront each and no barrier, longer ones four.  Bound: memory; 8192 rows of 8192, 201 MB in 36.7 us, 5.5 TB/s (a copy
// reaches 5.15); one row of 4096 takes 2.8 us, the launch.
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
// 16 x 16 x 64 steps of the matrix units, 32-bit sums (exact below 2^31 / 128^2 = 131072 codes: kMostIn).  Operands, lane = 16 g + c: row c, codes 16 g .. 16 g + 15.
struct LinearArgs {
    const int8_t *x, *w;
    const float *x_scale, *w_scale;
    uint16_t *out;
    int rows, n_in, n_out;
    int row_blocks, col_blocks;    // workgroups of the rows, of the outputs
};

// A sum times its scales, as fp16.  The fp32 product is made first (the compiler would put it and the conversion into one instruction, which rounds
// once, in some kernels and not in others).
__device__ __forceinline__ _Float16 scaled(int sum, float sx, float sw)
{
    float y = (float)sum * sx * sw;
    asm("" : "+v"(y));
    return (_Float16)y;
}

// What this wavefront requested is in LDS but for its last LEFT requests, and so it is with all others.
template <int LEFT>
__device__ __forceinline__ void landed_barrier()
{
    static_assert(LEFT < 64, "counted in six bits");
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LEFT) : "memory");
}
__device__ __forceinline__ void cf_lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Few rows: reading the weights is the work.  A workgroup takes 16 MT rows by 16 NT outputs; its wavefronts divide the sum, in pieces of 128 codes,
// and their results are added at the end through LDS.  A wavefront's pieces go from memory into its own ring of DEPTH places in LDS, so that no
// barrier holds up its loads.  (A lane of the matrix product holds a row, so that loads into registers would ask for 16 rows with every 16 lanes,
// which passes 4.3 TB/s; into LDS eight adjacent lanes load 128 bytes of a row.)
// Bound: memory where there are enough workgroups (1 x 4096 -> 12288: 50 MB in 11.4 us, of which some 2.5 are the launch; 4.9 TB/s while it streams),
// else the requests that a compute unit has under way (1 x 28672 -> 1024, 64 workgroups: 16.4 us; 64 x 4096 -> 6144, 192 workgroups: 10.5 us; all in
// captured graphs, weights from memory).  Eight wavefronts a workgroup were faster at long sums of few outputs (the first of these 14.8 us) and slower at
// ordinary ones (1 x 4096 -> 4096 5.1 -> 6.0): they are not among the ways, which do not know the length of the sum.  Without gain: sixteen
// wavefronts, rings in registers.
template <int MT, int NT, int WAVES, int DEPTH>
__global__ __launch_bounds__(64 * WAVES) void linear_stream(const LinearArgs a)
{
    constexpr int ROWS = 16 * MT, COLS = 16 * NT, PITCH = COLS + 4, T = 64 * WAVES, QUADS = ROWS * COLS / 4, PER = (QUADS + T - 1) / T;
    constexpr int PLACE = (ROWS + COLS) * 128, LOADS = (ROWS + COLS) / 8;
    constexpr int RING = DEPTH * PLACE, SUMS = ROWS * PITCH * 4, SPACE = WAVES * (RING > SUMS ? RING : SUMS);
    __shared__ alignas(16) char lds[SPACE];
    const int tid = threadIdx.x, wv = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, c = lane & 15, g = lane >> 4;
    const cf::linear::Block mine = cf::linear::stream_block(blockIdx.x, a.row_blocks, a.col_blocks);
    const int m0 = mine.m * ROWS, n_block = mine.n, n0 = n_block * COLS;
    if (n0 >= a.n_out) return;
    const int rows = min(ROWS, a.rows - m0), cols = min(COLS, a.n_out - n0);
    const __amdgpu_buffer_rsrc_t xr = cf::buffer_of(a.x + (size_t)m0 * a.n_in, (uint32_t)rows * a.n_in), wr = cf::buffer_of(a.w + (size_t)n0 * a.n_in, (uint32_t)cols * a.n_in);
    // four adjacent outputs of a row to a thread at the end: their scales are requested now
    float sx[PER], sw[PER][4];
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        const int quad = tid + T * p, m = min(quad / (COLS / 4), rows - 1), n = min(4 * (quad % (COLS / 4)), cols - 4);
        sx[p] = a.x_scale[m0 + m];
#pragma unroll
        for (int r = 0; r < 4; ++r) sw[p][r] = a.w_scale[n0 + n + r];
    }

    // A wavefront's pieces follow each other in a row; workgroups start at different ones.
    const int pieces = (a.n_in + 127) / 128, per = (pieces + WAVES - 1) / WAVES, first = wv * per, from = n_block % per;
    auto piece_of = [&](int i) { return i < per ? first + (i + from < per ? i + from : i + from - per) : pieces; };
    char *ring = lds + wv * RING;
    const int chunk = (lane & 7) ^ (lane >> 3);                     // of a row, at place lane & 7
    const uint32_t row_at = (uint32_t)(lane >> 3) * a.n_in + 16 * chunk;
    auto request = [&](int d, int i) {
        const int k0 = 128 * piece_of(i);
        const uint32_t at = row_at + (k0 + 16 * chunk < a.n_in ? (uint32_t)k0 : 0x80000000u);      // (behind the end, and rows that are not there: no access)
#pragma unroll
        for (int r = 0; r < COLS / 8; ++r) cf::to_lds(wr, ring + d * PLACE + 1024 * r, at + (uint32_t)(8 * r) * a.n_in, 0);
#pragma unroll
        for (int r = 0; r < ROWS / 8; ++r) cf::to_lds(xr, ring + d * PLACE + COLS * 128 + 1024 * r, at + (uint32_t)(8 * r) * a.n_in, 0);
    };
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) request(d, d);
    i32x4 sum[MT][NT] = {};
    for (int i0 = 0; i0 < per; i0 += DEPTH)
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            static_assert((DEPTH - 1) * LOADS < 64, "counted in six bits");
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"((DEPTH - 1) * LOADS) : "memory");
            const int end = a.n_in - 128 * piece_of(i0 + d);
            if (end > 0) {
                const char *w_at = ring + d * PLACE + 128 * c, *x_at = w_at + COLS * 128;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int place = 16 * ((4 * h + g) ^ (c & 7));
                    i32x4 w[NT], x[MT];
#pragma unroll
                    for (int j = 0; j < NT; ++j) {
                        w[j] = *reinterpret_cast<const i32x4 *>(w_at + 2048 * j + place);
                        if (64 * h + 16 * g >= end) w[j] = i32x4{0, 0, 0, 0};
                    }
#pragma unroll
                    for (int m = 0; m < MT; ++m) x[m] = *reinterpret_cast<const i32x4 *>(x_at + 2048 * m + place);
#pragma unroll
                    for (int j = 0; j < NT; ++j)
#pragma unroll
                        for (int m = 0; m < MT; ++m) sum[m][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[j], x[m], sum[m][j], 0, 0, 0);
                }
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // the place has been read
            request(d, i0 + d + DEPTH);
        }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    int *sums = reinterpret_cast<int *>(lds);
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) *reinterpret_cast<i32x4 *>(sums + (wv * ROWS + 16 * i + c) * PITCH + 16 * j + 4 * g) = sum[i][j];
    __syncthreads();
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        const int quad = tid + T * p, m = quad / (COLS / 4), n = 4 * (quad % (COLS / 4));
        if (m >= rows || n >= cols) continue;
        i32x4 t = {0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) t += *reinterpret_cast<const i32x4 *>(sums + (w * ROWS + m) * PITCH + n);
        *reinterpret_cast<h4 *>(a.out + (size_t)(m0 + m) * a.n_out + n0 + n) =
            h4{scaled(t[0], sx[p], sw[p][0]), scaled(t[1], sx[p], sw[p][1]), scaled(t[2], sx[p], sw[p][2]), scaled(t[3], sx[p], sw[p][3])};
    }
}

// Many rows: WM x WN wavefronts share a tile of BM rows by BN outputs.  Steps of 128 codes go from memory straight into LDS, one step ahead of the
// one that is used.  A row's eight 16-byte chunks lie there at places chunk ^ (row / 2 & 7), so that the rows of an operand are read from different banks
// (chunk ^ (row & 7): every read from twice as many cycles); the loads fill LDS in the order of the lanes, so it is their addresses in memory that
// are permuted.
// Bound: the matrix units, and behind them the power that the card has for them: 8192 x 8192 -> 10240 in 604 to 618 us in a captured graph, 2.2 to 2.3 Pop/s,
// the units busy for 64 % of the cycles at 1.7 GHz (called one by one 572 to 597 us, by card; in the graph a library's product of these sizes 647 us, the
// products alone, of operands that are not loaded, 475, the loads and the reading of operands alone 396).  256 x 4096 -> 6144 takes 17.1 us, 512 x 4096 -> 4096 17.2: start, steps
// and end of one tile on a compute unit.  Without gain: 128 x 128 to a wavefront, four on a compute unit (649 us); operands read where the compiler puts
// them (618); the barrier and the next step's first operands before the last product of a step (609); through registers in place of direct loads (slower at all sizes).
// Operands of a 32 x 32 x 32 step, lane = 32 g + c: row c, codes 16 g .. 16 g + 15; the result: output 8 (r / 4) + 4 g + r % 4 of row c.
constexpr int kTileStep = 128;
template <int BM, int BN, int WM, int WN, int STAGES>
__global__ __launch_bounds__(64 * WM * WN) void linear_tiles(const LinearArgs a)
{
    constexpr int WAVES = WM * WN, T = 64 * WAVES, TM = BM / WM / 32, TN = BN / WN / 32, XL = BM / 8 / WAVES, WL = BN / 8 / WAVES, PITCH = 2 * BN + 16;
    constexpr int STAGE = (BM + BN) * kTileStep, SPACE = STAGES * STAGE > BM * PITCH ? STAGES * STAGE : BM * PITCH;
    static_assert(BM % (8 * WAVES) == 0 && BN % (8 * WAVES) == 0 && WAVES % 2 == 0, "whole loads, of row blocks of 8 whose number is odd where the wavefront's is");
    __shared__ alignas(16) char lds[SPACE];
    const int tid = threadIdx.x, wv = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, c = lane & 31, g = lane >> 5;
    // each die takes a part of the tiles, eight row blocks by as many output blocks as it has room for at a time
    int m_block, n_block;
    {
        const int per = gridDim.x >> 3, t = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
        if (t >= a.row_blocks * a.col_blocks) return;
        const int group = t / (8 * a.col_blocks), in = t - group * 8 * a.col_blocks, tall = min(8, a.row_blocks - 8 * group);
        n_block = in / tall, m_block = 8 * group + in - n_block * tall;
    }
    const int m0 = m_block * BM, n0 = n_block * BN, rows = min(BM, a.rows - m0), cols = min(BN, a.n_out - n0);
    const __amdgpu_buffer_rsrc_t xr = cf::buffer_of(a.x + (size_t)m0 * a.n_in, (uint32_t)rows * a.n_in), wr = cf::buffer_of(a.w + (size_t)n0 * a.n_in, (uint32_t)cols * a.n_in);
    const int chunk = (lane & 7) ^ (4 * (wv & 1) + (lane >> 4));
    uint32_t x_at[XL], w_at[WL];                                    // rows that are not there repeat the last one
#pragma unroll
    for (int i = 0; i < XL; ++i) x_at[i] = min(8 * (wv + WAVES * i) + (lane >> 3), rows - 1) * a.n_in + 16 * chunk;
#pragma unroll
    for (int i = 0; i < WL; ++i) w_at[i] = min(8 * (wv + WAVES * i) + (lane >> 3), cols - 1) * a.n_in + 16 * chunk;
    const int steps = (a.n_in + kTileStep - 1) / kTileStep, my_m = (wv / WN) * (32 * TM), my_n = (wv % WN) * (32 * TN);
    // the dies start at different steps, so that they do not all ask the same memory channels
    const int from = (blockIdx.x & 7) * steps / 8;
    auto turned = [&](int i) { return i + from < steps ? i + from : i + from - steps; };
    auto request = [&](int i, char *to) {
        const int k0 = turned(i) * kTileStep;
        const int back = max(k0 + 16 * chunk - (a.n_in - 16), 0);   // chunks behind the end: any other one
#pragma unroll
        for (int i = 0; i < XL; ++i) cf::to_lds(xr, to + 1024 * (wv + WAVES * i), x_at[i] - back, k0);
#pragma unroll
        for (int i = 0; i < WL; ++i) cf::to_lds(wr, to + BM * kTileStep + 1024 * (wv + WAVES * i), w_at[i] - back, k0);
    };
    i32x16 sum[TM][TN] = {};
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i)
        if (i < steps) request(i, lds + i * STAGE);
    char *now = lds, *next = lds + (STAGES - 1) * STAGE;
    for (int i = 0; i < steps; ++i) {
        // this step is there, and the buffer that is requested into has been read
        if (i + STAGES - 2 < steps)
            landed_barrier<(STAGES - 2) * (XL + WL)>();
        else
            landed_barrier<0>();
        if (i + STAGES - 1 < steps) request(i + STAGES - 1, next);
        const char *xs = now, *ws = now + BM * kTileStep;
        const int end = a.n_in - turned(i) * kTileStep;
        if (end < kTileStep) {                                      // what lies behind the end of the sums counts as zeros
            for (int e = tid; e < BN * 8; e += T)
                if (16 * (e & 7) >= end) *reinterpret_cast<i32x4 *>(now + BM * kTileStep + (e >> 3) * kTileStep + 16 * ((e ^ e >> 4) & 7)) = i32x4{0, 0, 0, 0};
            cf_lds_barrier();
        }
        next = now;
        now = now + STAGE == lds + STAGES * STAGE ? lds : now + STAGE;
        // operands are read a product ahead
        i32x4 x[2][TM], w[2][TN];
        auto read = [&](int kk) {
            const int place = 16 * ((2 * kk + g) ^ (c >> 1 & 7));
#pragma unroll
            for (int j = 0; j < TN; ++j) w[kk & 1][j] = *reinterpret_cast<const i32x4 *>(ws + (my_n + 32 * j + c) * kTileStep + place);
#pragma unroll
            for (int i = 0; i < TM; ++i) x[kk & 1][i] = *reinterpret_cast<const i32x4 *>(xs + (my_m + 32 * i + c) * kTileStep + place);
        };
        read(0);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int kk = 0; kk < kTileStep / 32; ++kk) {
            if (kk + 1 < kTileStep / 32) read(kk + 1);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) sum[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(w[kk & 1][j], x[kk & 1][i], sum[i][j], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    __syncthreads();
    // ---- scaled, and stored in whole rows by way of LDS
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int m = my_m + 32 * i + c;
        const float sx = a.x_scale[m0 + min(m, rows - 1)];
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int n = my_n + 32 * j + 8 * q + 4 * g;
                const float *sw = a.w_scale + n0 + min(n, cols - 4);
                *reinterpret_cast<h4 *>(lds + m * PITCH + 2 * n) = h4{scaled(sum[i][j][4 * q], sx, sw[0]), scaled(sum[i][j][4 * q + 1], sx, sw[1]),
                                                                     scaled(sum[i][j][4 * q + 2], sx, sw[2]), scaled(sum[i][j][4 * q + 3], sx, sw[3])};
            }
    }
    __syncthreads();
    for (int e = tid; e < BM * (BN / 8); e += T) {
        const int m = e / (BN / 8), n = 8 * (e % (BN / 8));
        if (m < rows && n < cols) *reinterpret_cast<u32x4 *>(a.out + (size_t)(m0 + m) * a.n_out + n0 + n) = *reinterpret_cast<const u32x4 *>(lds + m * PITCH + 2 * n);
    }
}

using Kernel = void (*)(const LinearArgs);
constexpr Kernel kKernels[] = {            // of cf::linear::kWays
    linear_stream<1, 1, 4, 3>, linear_stream<1, 2, 4, 4>, linear_stream<2, 2, 4, 2>, linear_stream<4, 2, 4, 2>, linear_stream<4, 4, 4, 2>,
    linear_tiles<64, 64, 2, 2, 4>, linear_tiles<128, 64, 2, 2, 4>, linear_tiles<256, 128, 4, 2, 3>, linear_tiles<256, 256, 2, 4, 2>,
};
static_assert(sizeof kKernels / sizeof *kKernels == cf::linear::kNumWays, "a kernel for each way");

constexpr int kMostRows = 1 << 23;         // workgroups of a launch
constexpr int kMostIn = 131056;            // the last multiple of 16 that 128^2 times of is below 2^31: codes of -128 are allowed

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
    LinearArgs a = {x, W, x_scale, w_scale, static_cast<uint16_t *>(out), rows, c.n_in, c.n_out, 0, 0};
    const int way = cf::linear::way_of(c.n_out, rows, t->cus);
    const cf::linear::Way &p = cf::linear::kWays[way];
    a.row_blocks = cf::linear::blocks_of(rows, p.rows), a.col_blocks = cf::linear::blocks_of(c.n_out, p.cols);
    const unsigned grid = p.tiles ? (unsigned)(a.row_blocks * a.col_blocks + 7) / 8 * 8 : cf::linear::stream_grid(a.row_blocks, a.col_blocks);
    hipLaunchKernelGGL(kKernels[way], dim3(grid), dim3(p.threads), 0, static_cast<hipStream_t>(stream), a);
    return hipGetLastError() == hipSuccess ? CF_OK : CF_EHIP;
}

int64_t cf_linear_algorithmic_bytes(const cf_linear_config *cfg, int32_t rows)
{
    if (!cfg) return 0;
    const int64_t m = rows, k = cfg->n_in, n = cfg->n_out;
    return m * k + n * k + 4 * (m + n) + 2 * m * n;
}

}  // extern "C"
