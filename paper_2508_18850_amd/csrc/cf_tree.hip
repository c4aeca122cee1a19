// Attention of drafted tokens over a key/value cache (cf_tree_* in include/cfdecode.h).
//
// The rows of one KV head's queries (token t, query head hh of the group: row t * group + hh) are cut into blocks of 16 NR, the keys of a
// sequence into parts; a workgroup takes one block over one part.  Its four wavefronts take steps of 32 keys in turn, each with all rows
// of the block: scores and weighted values are matrix products (cf_tree_device.h), keys and values go from memory into registers as the
// operands want them, and nothing passes through LDS until the wavefronts' results are joined.
//
// Softmax in one pass.  Every row keeps a reference mm, the sum l of 2^(x_j - mm) and the sums of w_j v_j with
// w_j = 2^(x_j - mm) * scale_j (x_j: score in units of log2 e, scale_j: scale of an 8-bit value row, else 1), so that values enter the
// product as codes.  mm is moved, and what has been summed brought to the new one, only when some w_j exceeds 2^15: to where the
// largest w_j that the row has seen is 2^7.  w_j is rounded to fp16 for the product (half a step, 2^-11 of each weight: about as much as
// the rounding of the result; below 2^-14, that is 2^-21 of the largest, half of 2^-24); all else is fp32.  Each row's own scores alone decide when its mm moves, so
// that what it does not see leaves its bits alone.
#include "../../include/cfdecode.h"
#include "cf_cache_device.h"
#include "cf_lanes_device.h"
#include "cf_tree_device.h"

#include <cmath>
#include <cstring>
#include <new>

namespace {

using namespace cf::cache;
using cf::tree::f32x4;
using cf::tree::Keys;
using cf::tree::mfma16;
using cf::tree::Values;

constexpr int kMaxTokens = 256;
constexpr int NT = 256, NW = NT / 64;
constexpr int kStep = 32;                  // keys of a step
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNone = -1e30f;            // mm of a row that has seen nothing
constexpr float kSmallScale = 0x1p-60f;    // stands for smaller scales: no fp16 result shows values of 448 times that
constexpr float kMostWeight = 32768.f, kTopExponent = 7.f;

struct TreeArgs {
    const uint16_t *q;
    const char *k, *v;
    const float *k_scale, *v_scale, *slopes;
    uint16_t *out;
    float *part;                   // [batch, KV head][split][row] : HD sums, for more than one split
    float2 *part_ml;               // the same rows' mm and l
    Lengths rows;
    const int32_t *depth;
    const uint64_t *tree;
    int depth_stride;              // depths of a batch row: 0 where all share them
    int tree_stride, words;        // words of a batch row's masks (0: shared), of a token's mask
    int nq, nkv, group, max_seq, window;
    int splits, blocks, units;     // parts of a sequence; row blocks; batch * nkv * splits
    float cap;
};

__device__ __forceinline__ uint32_t low_bits(int n) { return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u; }

// Which of the keys j0 .. j0 + 31 token t sees: bit i for key j0 + i (without the window).
__device__ __forceinline__ uint32_t seen_bits(const TreeArgs &a, const uint64_t *tree, int t, int j0, int len, int n)
{
    const int u0 = j0 - len;                                       // the new token at j0
    uint32_t mine;
    if (tree) {
        const uint64_t *w = tree + (size_t)t * a.words;
        if (u0 < 0) {
            mine = u0 <= -32 ? 0u : (uint32_t)w[0] << -u0;
        } else {
            const int i = u0 >> 6, sh = u0 & 63;
            uint64_t x = i < a.words ? w[i] >> sh : 0;
            if (sh > 32 && i + 1 < a.words) x |= w[i + 1] << (64 - sh);
            mine = (uint32_t)x;
        }
    } else {
        mine = low_bits(t - u0 + 1);
    }
    return (low_bits(len - j0) | (mine & ~low_bits(-u0))) & low_bits(len + n - j0);
}

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

template <int HD, int NR>
constexpr int kWaveFloats = 16 * (HD + 4) > NR * 16 * kStep ? 16 * (HD + 4) : NR * 16 * kStep;

// FORMS: the scores may be capped, biased or windowed.
template <int HD, int FMT, int NR, bool FORMS>
__global__ __launch_bounds__(NT, NR == 4 ? 1 : 2) void tree_tiles(const TreeArgs a)
{
    constexpr int KS = HD / 32, NJ = HD / 16, ROW = HD * kValueBytes<FMT>;
    constexpr bool SCALED = FMT != CF_CACHE_F16;
    __shared__ float smem[NW * kWaveFloats<HD, NR>];
    __shared__ float2 ml[NW][16 * NR];
    __shared__ float scales[NW][2][kStep];
    const int tid = threadIdx.x, wv = tid >> 6, lane = tid & 63, c = lane & 15, g = lane >> 4;
    // Workgroup i runs on die i mod 8: the row blocks of a unit, which read the same keys and values, follow each other on one die.
    const int turn = blockIdx.x >> 3, unit = turn / a.blocks * 8 + (blockIdx.x & 7), block = turn % a.blocks;
    if (unit >= a.units) return;
    const int bh = unit / a.splits, split = unit - bh * a.splits, b = bh / a.nkv, head = bh - b * a.nkv;
    const int n = a.rows.fresh(b), len = a.rows.cached(b), end = len + n;
    const int first_row = block * (16 * NR), live = min(n * a.group - first_row, 16 * NR);
    if (live <= 0) return;
    const int32_t *depth = a.depth ? a.depth + (size_t)b * a.depth_stride : nullptr;
    const uint64_t *tree = a.tree ? a.tree + (size_t)b * a.tree_stride : nullptr;

    // ---- the rows of this lane: queries as B operands, positions
    h8 q[NR][KS];
    int tok[NR];
    [[maybe_unused]] int at[NR];
    [[maybe_unused]] float slope[NR];
    int nearest = 0x3fffffff, farthest = -0x3fffffff;               // of the positions of the block's tokens
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        const int row = first_row + 16 * r + c, t = row / a.group, hh = row - t * a.group;
        tok[r] = t < n ? t : -1;
        if (t < n) {
            const uint16_t *src = a.q + (((size_t)b * a.rows.tokens + t) * a.nq + head * a.group + hh) * HD;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) q[r][ks] = *reinterpret_cast<const h8 *>(src + Keys<HD, FMT>::dim(ks, g));
        } else {
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) q[r][ks] = h8{};
        }
        if constexpr (FORMS) {
            at[r] = 0, slope[r] = 0.f;
            if (t < n) {
                const long long p = (long long)len + (depth ? depth[t] : t);
                at[r] = (int)min(max(p, -0x3fffffffLL), 0x3fffffffLL);
                nearest = min(nearest, at[r]), farthest = max(farthest, at[r]);
                slope[r] = a.slopes ? a.slopes[head * a.group + hh] * kLog2e : 0.f;
            }
        }
    }

    // ---- the keys of this part: steps of 32, counted from key 0
    int lo = 0, all_from = 0;                                       // the first key that some row sees, that all rows see
    if constexpr (FORMS) {
        if (a.window > 0) {
#pragma unroll
            for (int s = 1; s < 64; s <<= 1) nearest = min(nearest, __shfl_xor(nearest, s)), farthest = max(farthest, __shfl_xor(farthest, s));
            lo = min(max(nearest - a.window + 1, 0), len);
            all_from = max(farthest - a.window + 1, 0);
        }
    }
    const int step0 = lo / kStep, steps = (end + kStep - 1) / kStep - step0, per = (steps + a.splits - 1) / a.splits;
    const int s_begin = step0 + split * per, s_end = min(step0 + steps, s_begin + per);

    const size_t slice = (size_t)bh * a.max_seq;
    const __amdgpu_buffer_rsrc_t kr = cf::buffer_of(a.k + slice * ROW, (uint32_t)end * ROW), vr = cf::buffer_of(a.v + slice * ROW, (uint32_t)end * ROW);
    const float *scale_src = SCALED ? (lane < 32 ? a.k_scale : a.v_scale) + slice : nullptr;
    const float unit_k = (FMT == CF_CACHE_INT8 ? cf::tree::kInt8Unit : 1.f) * (HD == 64 ? 0.125f : 0.08838834764831845f);
    // what a score is multiplied with: to units of log2 e, or, with a cap, to twice its share of the cap in the same units
    const float to_score = FORMS && a.cap > 0.f ? unit_k * 2.f * kLog2e / a.cap : unit_k * kLog2e;

    Keys<HD, FMT> keys;
    Values<HD, FMT> vals;
    float scale = 0.f;
    f32x4 acc[NR][NJ];
    float mm[NR], l[NR];
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        mm[r] = kNone, l[r] = 0.f;
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[r][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const uint32_t koff = Keys<HD, FMT>::offset(c, g), voff = Values<HD, FMT>::offset(c, g);
    auto load_scale = [&](int step) {
        if constexpr (SCALED) scale = scale_src[min(step * kStep + (lane & 31), end - 1)];
    };
    int step = s_begin + wv;
    if (step < s_end) {
        load_scale(step);
        keys.load(kr, koff + (uint32_t)step * (kStep * ROW));
        vals.load(vr, voff + (uint32_t)step * (kStep * ROW));
    }
    for (; step < s_end; step += NW) {
        const int j0 = step * kStep;
        const bool masked = j0 + kStep > len || j0 < all_from;      // (the same for the whole wavefront)
        const uint32_t next = (uint32_t)min(step + NW, s_end - 1) * (kStep * ROW);
        if constexpr (SCALED) {
            const float x = lane < 32 ? scale * to_score : fabsf(scale) < kSmallScale ? kSmallScale : scale;
            scales[wv][lane >> 5][lane & 31] = x;
        }
        // ---- scores
        f32x4 s[NR][2];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const h8 k = keys.operand(t, ks);
#pragma unroll
                for (int r = 0; r < NR; ++r) s[r][t] = mfma16(k, q[r][ks], ks ? s[r][t] : f32x4{0.f, 0.f, 0.f, 0.f});
            }
        keys.load(kr, koff + next);
        f32x4 kscale[2], vscale[2];
        if constexpr (SCALED) {
            wave_sync();
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                kscale[t] = *reinterpret_cast<const f32x4 *>(&scales[wv][0][16 * t + 4 * g]);
                vscale[t] = *reinterpret_cast<const f32x4 *>(&scales[wv][1][16 * t + 4 * g]);
            }
            wave_sync();
            load_scale(min(step + NW, s_end - 1));
        }
        // ---- weights
        h8 w[NR];
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            float x[8], p[8], wt[8];
            if (FORMS || masked) {
                const uint32_t bits = !masked ? ~0u : tok[r] < 0 ? 0u : seen_bits(a, tree, tok[r], j0, len, n);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int i = 16 * (e >> 2) + 4 * g + (e & 3), j = j0 + i;
                    x[e] = s[r][e >> 2][e & 3] * (SCALED ? kscale[e >> 2][e & 3] : to_score);
                    bool seen = bits >> i & 1;
                    if constexpr (FORMS) {
                        int key_at = j;
                        if (masked && j >= len && depth) key_at = j < end ? (int)min(max((long long)len + depth[j - len], -0x3fffffffLL), 0x3fffffffLL) : 0;
                        const int distance = at[r] - key_at;
                        if (a.cap > 0.f) x[e] = a.cap * kLog2e * (1.f - 2.f * __builtin_amdgcn_rcpf(exp2_(x[e]) + 1.f));      // tanh
                        x[e] -= slope[r] * (float)distance;
                        if (masked && a.window > 0) seen = seen && distance < a.window;
                    }
                    if (masked && !seen) x[e] = -INFINITY;
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = s[r][e >> 2][e & 3] * (SCALED ? kscale[e >> 2][e & 3] : to_score);
            }
            auto weigh = [&]() {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    p[e] = exp2_(x[e] - mm[r]);
                    wt[e] = SCALED ? p[e] * vscale[e >> 2][e & 3] : p[e];
                    if (SCALED && masked && x[e] == -INFINITY) wt[e] = 0.f;             // (the scale of an unseen row may be anything)
                }
            };
            weigh();
            float most = fmaxf(fmaxf(fmaxf(wt[0], wt[1]), fmaxf(wt[2], wt[3])), fmaxf(fmaxf(wt[4], wt[5]), fmaxf(wt[6], wt[7])));
            if (__any(most > kMostWeight)) {
                float top = kNone;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float y = SCALED ? x[e] + __builtin_amdgcn_logf(vscale[e >> 2][e & 3]) : x[e];
                    top = fmaxf(top, masked && x[e] == -INFINITY ? kNone : y);
                }
                top = cf::lanes::max_groups<16>(top);
                most = cf::lanes::max_groups<16>(most);
                const float to = most > kMostWeight ? top - kTopExponent : mm[r], by = exp2_(mm[r] - to);
                mm[r] = to;
                l[r] *= by;
#pragma unroll
                for (int j = 0; j < NJ; ++j) acc[r][j] *= by;
                weigh();
            }
            l[r] += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
#pragma unroll
            for (int e = 0; e < 8; ++e) w[r][e] = (_Float16)wt[e];
        }
        // ---- values
        h8 v[NJ];
        vals.operands(v);
        if (FMT != CF_CACHE_INT8 && masked) {
            // 0 times an infinity or a NaN of an unseen value row would be NaN: where the step holds one, such values are left out of the
            // product and added, token by token, to the rows that see them.
            uint32_t odd = 0;
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int d = 0; d < 4; ++d) odd |= (__builtin_bit_cast(cf::tree::u32x4, v[j])[d] & 0x7c007c00u) + 0x04000400u;
            if (__any(odd & 0x80008000u)) {
#pragma unroll
                for (int j = 0; j < NJ; ++j)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if ((__builtin_bit_cast(uint16_t, (_Float16)v[j][e]) & 0x7c00u) == 0x7c00u) v[j][e] = (_Float16)0.f;
                float *tmp = smem + wv * kWaveFloats<HD, NR>;                          // [r][key][row]
                wave_sync();
#pragma unroll
                for (int r = 0; r < NR; ++r)
#pragma unroll
                    for (int e = 0; e < 8; ++e) tmp[(r * kStep + 16 * (e >> 2) + 4 * g + (e & 3)) * 16 + c] = (float)w[r][e];
                wave_sync();
#pragma unroll 1
                for (int i = 0; i < kStep; ++i)
#pragma unroll
                    for (int rr = 0; rr < 4; ++rr)
#pragma unroll
                        for (int j = 0; j < NJ; ++j) {
                            const uint32_t d = (uint32_t)(j0 + i) * ROW + (NJ * (4 * g + rr) + j) * kValueBytes<FMT>;
                            float x;
                            if constexpr (FMT == CF_CACHE_F16) {
                                x = (float)__builtin_bit_cast(_Float16, (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(vr, d, 0, 0));
                            } else {
                                float f[4];
                                decode4<FMT>((uint32_t)(uint8_t)__builtin_amdgcn_raw_buffer_load_b8(vr, d, 0, 0), f);
                                x = f[0];
                            }
                            if (!(fabsf(x) <= 65504.f))
#pragma unroll
                                for (int r = 0; r < NR; ++r) {
                                    const float wt = tmp[(r * kStep + i) * 16 + c];
                                    if (wt != 0.f) acc[r][j][rr] += wt * x;
                                }
                        }
            }
        }
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int r = 0; r < NR; ++r) acc[r][j] = mfma16(v[j], w[r], acc[r][j]);
        vals.load(vr, voff + next);
    }

    // ---- the wavefronts' results joined, 16 rows at a time
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        l[r] = cf::lanes::sum_groups<16>(l[r]);
        if (g == 0) ml[wv][16 * r + c] = make_float2(mm[r], l[r]);
    }
    constexpr int CH = HD / 8;                                      // a thread has eight dimensions of a row
    const int row16 = tid / CH, d0 = 8 * (tid % CH);
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        __syncthreads();
#pragma unroll
        for (int rr = 0; rr < 4; ++rr)
#pragma unroll
            for (int j = 0; j < NJ; j += 4)
                *reinterpret_cast<float4 *>(smem + (wv * 16 + c) * (HD + 4) + NJ * (4 * g + rr) + j) =
                    make_float4(acc[r][j][rr], acc[r][j + 1][rr], acc[r][j + 2][rr], acc[r][j + 3][rr]);
        __syncthreads();
        const int row = 16 * r + row16;
        if (row16 < 16 && row < live) {
            float m = kNone, total = 0.f, o[8] = {};
#pragma unroll
            for (int k = 0; k < NW; ++k) m = fmaxf(m, ml[k][row].x);
#pragma unroll
            for (int k = 0; k < NW; ++k) {
                const float f = exp2_(ml[k][row].x - m);
                const float *src = smem + (k * 16 + row16) * (HD + 4) + d0;
                total += f * ml[k][row].y;
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] += f * src[e];
            }
            if (a.splits > 1) {
                const size_t at_row = (size_t)unit * (a.blocks * 16 * NR) + first_row + row;
                float4 *dst = reinterpret_cast<float4 *>(a.part + at_row * HD + d0);
                dst[0] = make_float4(o[0], o[1], o[2], o[3]);
                dst[1] = make_float4(o[4], o[5], o[6], o[7]);
                if (d0 == 0) a.part_ml[at_row] = make_float2(m, total);
            } else {
                const int t = (first_row + row) / a.group, hh = first_row + row - t * a.group;
                const float inv = total == 0.f ? 0.f : (FMT == CF_CACHE_INT8 ? cf::tree::kInt8Unit : 1.f) / total;
                h8 res;
#pragma unroll
                for (int e = 0; e < 8; ++e) res[e] = (_Float16)(o[e] * inv);
                *reinterpret_cast<h8 *>(a.out + (((size_t)b * a.rows.tokens + t) * a.nq + head * a.group + hh) * HD + d0) = res;
            }
        }
    }
}

// The parts of a sequence joined, in their order: eight dimensions of a row to a thread.
template <int HD>
__global__ __launch_bounds__(NT) void tree_join(const TreeArgs a, int padded, float unit_v)
{
    constexpr int CH = HD / 8;
    const int bh = blockIdx.y, b = bh / a.nkv, head = bh - b * a.nkv;
    const int row = blockIdx.x * (NT / CH) + threadIdx.x / CH, d0 = 8 * (threadIdx.x % CH);
    if (row >= a.rows.fresh(b) * a.group) return;
    const size_t first = (size_t)bh * a.splits * padded + row;
    float m = kNone, total = 0.f, o[8] = {};
    for (int s = 0; s < a.splits; ++s) m = fmaxf(m, a.part_ml[first + (size_t)s * padded].x);
    for (int s = 0; s < a.splits; ++s) {
        const float2 x = a.part_ml[first + (size_t)s * padded];
        const float f = exp2_(x.x - m);
        const float4 *src = reinterpret_cast<const float4 *>(a.part + (first + (size_t)s * padded) * HD + d0);
        const float4 u = src[0], w = src[1];
        total += f * x.y;
        o[0] += f * u.x, o[1] += f * u.y, o[2] += f * u.z, o[3] += f * u.w;
        o[4] += f * w.x, o[5] += f * w.y, o[6] += f * w.z, o[7] += f * w.w;
    }
    const float inv = total == 0.f ? 0.f : unit_v / total;
    h8 res;
#pragma unroll
    for (int e = 0; e < 8; ++e) res[e] = (_Float16)(o[e] * inv);
    const int t = row / a.group, hh = row - t * a.group;
    *reinterpret_cast<h8 *>(a.out + (((size_t)b * a.rows.tokens + t) * a.nq + head * a.group + hh) * HD + d0) = res;
}

using KernelFn = void (*)(const TreeArgs);
template <int HD, int FMT>
KernelFn pick_rows(int nr, bool forms)
{
    if (forms) return nr == 1 ? tree_tiles<HD, FMT, 1, true> : nr == 2 ? tree_tiles<HD, FMT, 2, true> : tree_tiles<HD, FMT, 4, true>;
    return nr == 1 ? tree_tiles<HD, FMT, 1, false> : nr == 2 ? tree_tiles<HD, FMT, 2, false> : tree_tiles<HD, FMT, 4, false>;
}
KernelFn pick(int hd, int fmt, int nr, bool forms)
{
    if (hd == 64) return fmt == CF_CACHE_F16 ? pick_rows<64, CF_CACHE_F16>(nr, forms) : fmt == CF_CACHE_E4M3 ? pick_rows<64, CF_CACHE_E4M3>(nr, forms) : pick_rows<64, CF_CACHE_INT8>(nr, forms);
    return fmt == CF_CACHE_F16 ? pick_rows<128, CF_CACHE_F16>(nr, forms) : fmt == CF_CACHE_E4M3 ? pick_rows<128, CF_CACHE_E4M3>(nr, forms) : pick_rows<128, CF_CACHE_INT8>(nr, forms);
}

// How a call is divided.
struct Plan {
    int nr, blocks, splits;
};
constexpr int kMaxSplits = 64;
// keys: the most that a row sees.  As many parts as bring two workgroups to a compute unit, with a step or more for every wavefront.
Plan plan_of(int batch, int nkv, int group, int tokens, int keys, int cus, int limit)
{
    const int rows = tokens * group;
    Plan p;
    p.nr = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
    p.blocks = (rows + 16 * p.nr - 1) / (16 * p.nr);
    const long long items = (long long)batch * nkv * p.blocks;
    const int wanted = (int)((2ll * cus + items - 1) / items), most = (keys + NW * kStep - 1) / (NW * kStep);
    p.splits = wanted < most ? wanted : most;
    if (p.splits > kMaxSplits) p.splits = kMaxSplits;
    if (limit > 0 && p.splits > limit) p.splits = limit;
    if (p.splits < 1) p.splits = 1;
    return p;
}

}  // namespace

struct cf_tree_s {
    cf_tree_config cfg;
    int device = 0, cus = 0;
    int max_splits = 0;
    char *ws = nullptr;
    size_t ws_rows = 0;            // rows of partial results that the workspace holds
};

extern "C" {

int cf_tree_create(const cf_tree_config *cfg, cf_tree *out)
{
    if (!cfg || !out) return CF_EINVAL;
    *out = nullptr;
    const int rc = check_config(cfg->cache);
    if (rc != CF_OK) return rc;
    if (cfg->max_tokens < 1 || cfg->max_tokens > kMaxTokens || cfg->window < 0 || !(cfg->score_cap >= 0.f) || !(cfg->score_cap <= 3.402823466e38f)) return CF_EINVAL;
    int dev = 0, cus = 0;
    if (hipGetDevice(&dev) != hipSuccess ||
        hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cus < 1)
        return CF_EHIP;
    // Rows of partial results: a call with more than one part has fewer than 2 * cus + items workgroups of at most 64 rows, and items
    // (batch rows, KV heads and row blocks) below 2 * cus.
    const size_t rows = 4 * (size_t)cus * 64;
    cf_tree t = new (std::nothrow) cf_tree_s();
    if (!t) return CF_ENOMEM;
    t->cfg = *cfg;
    t->device = dev, t->cus = cus, t->ws_rows = rows;
    const hipError_t e = hipMalloc(reinterpret_cast<void **>(&t->ws), rows * (cfg->cache.head_dim * sizeof(float) + sizeof(float2)));
    if (e != hipSuccess) {
        delete t;
        return e == hipErrorOutOfMemory ? CF_ENOMEM : CF_EHIP;
    }
    *out = t;
    return CF_OK;
}

int cf_tree_destroy(cf_tree t)
{
    if (!t) return CF_EINVAL;
    const hipError_t e = hipFree(t->ws);
    delete t;
    return e == hipSuccess ? CF_OK : CF_EHIP;
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
    a.nq = c.n_q_heads, a.nkv = c.n_kv_heads, a.group = c.n_q_heads / c.n_kv_heads, a.max_seq = c.max_seq;
    a.window = t->cfg.window, a.cap = t->cfg.score_cap;
    const int keys = (a.window > 0 && a.window < draft->max_len ? a.window : draft->max_len) + draft->tokens;
    Plan p = plan_of(batch, a.nkv, a.group, draft->tokens, keys, t->cus, t->max_splits);
    const size_t rows = (size_t)batch * a.nkv * p.blocks * 16 * p.nr;
    if (p.splits > 1 && rows * p.splits > t->ws_rows) p.splits = (int)(t->ws_rows / rows) > 1 ? (int)(t->ws_rows / rows) : 1;
    a.splits = p.splits, a.blocks = p.blocks, a.units = batch * a.nkv * p.splits;
    a.part = reinterpret_cast<float *>(t->ws);
    a.part_ml = reinterpret_cast<float2 *>(t->ws + t->ws_rows * c.head_dim * sizeof(float));
    const hipStream_t s = static_cast<hipStream_t>(stream);
    hipLaunchKernelGGL(pick(c.head_dim, c.format, p.nr, a.cap > 0.f || a.window > 0 || a.slopes), dim3((a.units + 7) / 8 * 8 * p.blocks), dim3(NT), 0, s, a);
    if (hipGetLastError() != hipSuccess) return CF_EHIP;
    if (p.splits > 1) {
        const int per = NT / (c.head_dim / 8), live = draft->tokens * a.group;
        const float unit_v = c.format == CF_CACHE_INT8 ? cf::tree::kInt8Unit : 1.f;
        hipLaunchKernelGGL((c.head_dim == 64 ? tree_join<64> : tree_join<128>), dim3((live + per - 1) / per, batch * a.nkv), dim3(NT), 0, s, a,
                           p.blocks * 16 * p.nr, unit_v);
        if (hipGetLastError() != hipSuccess) return CF_EHIP;
    }
    return CF_OK;
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
