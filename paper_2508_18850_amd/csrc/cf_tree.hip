// Attention of drafted tokens over a key/value cache (cf_tree_* in include/cfdecode.h).
//
// The rows of one KV head's queries (token t, query head hh of the group: row t * group + hh) are cut into blocks, the keys of a sequence
// into parts; a workgroup takes one block over one part.  Scores and weighted values are matrix products (cf_tree_device.h).  Three
// kernels: with blocks of up to 32 rows the four wavefronts of a workgroup take steps of 32 keys in turn, each with all rows, and keys and
// values go from memory into registers as the operands want them (tree_tiles); with larger ones the wavefronts divide the rows and share
// steps of 64 keys, which are staged in LDS as fp16 (tree_blocks), so that 8-bit codes are converted once for all rows.  A 4-bit cache has
// blocks of up to 32 rows alone, whose values go through LDS that each wavefront has for itself (tree_fours).
//
// Softmax in one pass.  Every row keeps a reference mm, the sum l of 2^(x_j - mm) and the sums of w_j v_j with
// w_j = 2^(x_j - mm) * scale_j (x_j: score in units of log2 e, scale_j: scale of an 8-bit value row, else 1), so that values enter the
// product as codes.  mm is moved, and what has been summed brought to the new one, only when some w_j exceeds 2^15: to where the
// largest w_j that the row has seen is 2^7.  w_j is rounded to fp16 for the product (half a step, 2^-11 of each weight: about as much as
// the rounding of the result; below 2^-14, that is 2^-21 of the largest, half of 2^-24); all else is fp32.  Each row's own scores alone
// decide when its mm moves, so that what it does not see leaves its bits alone.
#include "../../include/cfdecode.h"
#include "cf_cache_device.h"
#include "cf_lanes_device.h"
#include "cf_tree_device.h"

#include <algorithm>
#include <cmath>
#include <cstring>
#include <initializer_list>
#include <new>
#include <type_traits>

namespace {

using namespace cf::cache;
using cf::tree::f32x4;
using cf::tree::Keys;
using cf::tree::Keys4;
using cf::tree::mfma16;
using cf::tree::Values;
using cf::tree::Values4;

constexpr int kMaxTokens = 256, kMaskWords = kMaxTokens / 64;
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
    // for more than one part
    float *part;                   // [batch, KV head][part][row]: HD sums, and behind all rows, from part_ml on, their mm and l
    uint32_t part_ml, part_bytes;  // bytes
    uint32_t *arrived;             // [batch, KV head][row block]: parts that are done, if the last one joins them; else NULL
    Lengths rows;
    const int32_t *depth;
    const uint64_t *tree;
    int depth_stride;              // depths of a batch row: 0 where all share them
    int tree_stride, words;        // words of a batch row's masks (0: shared), of a token's mask
    int nq, nkv, group, max_seq, window;
    int splits, blocks, units;     // parts of a sequence; row blocks; batch * nkv * splits
    int padded;                    // rows of all row blocks
    float cap;
};

__device__ __forceinline__ uint32_t low_bits(int n) { return (uint32_t)(((1ull << min(max(n, 0), 32)) - 1)); }

// Which of the keys j0 .. j0 + 31 token t sees: bit i for key j0 + i (without the window).  j0 is the same in all lanes; mask: the token's
// words (t < 0: of any other token; it sees nothing).
__device__ __forceinline__ uint32_t seen_bits(bool tree, int words, const uint64_t *mask, int t, int j0, int len, int n)
{
    const int u0 = j0 - len;                                       // the new token at j0
    uint32_t mine = 0;
    if (!tree) {
        mine = low_bits(t - u0 + 1);
    } else if (u0 > -32) {
        const int i = max(u0, 0) >> 6, sh = max(u0, 0) & 63;
        if (i < words) {
            uint64_t x = mask[i] >> sh;
            if (sh > 32 && i + 1 < words) x |= mask[i + 1] << (64 - sh);
            mine = (uint32_t)x << max(-u0, 0);
        }
    }
    const uint32_t seen = (low_bits(len - j0) | (mine & ~low_bits(-u0))) & low_bits(len + n - j0);
    return t < 0 ? 0u : seen;
}

// the scale of a row of values, not below kSmallScale (a NaN stays one; scales are not negative)
__device__ __forceinline__ float at_least_small(float x) { return x != x ? x : fmaxf(x, kSmallScale); }

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}
__device__ __forceinline__ void lds_barrier()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// whether a cached row has one scale that scores and weights are multiplied with (8 bits)
template <int FMT>
constexpr bool kRowScale = FMT == CF_CACHE_E4M3 || FMT == CF_CACHE_INT8;

constexpr int kFar = 0x3fffffff;

// In the kernels below no branch inside the loops over the keys depends on the lane: conditions of lanes are selections, and addresses of
// lanes without a value are taken to one that is there.  (The register allocator of this compiler, when it runs out of registers, has put
// copies for all lanes into the end of a branch that only some lanes take, and the others then had stale values.)

// What a workgroup knows of its batch row.
struct Sequence {
    int n, len, end;               // new tokens, cached rows, their sum
    const int32_t *depth;
    const uint64_t *tree;
    __device__ __forceinline__ Sequence(const TreeArgs &a, int b)
        : n(__builtin_amdgcn_readfirstlane(a.rows.fresh(b))), len(__builtin_amdgcn_readfirstlane(a.rows.cached(b))), end(len + n), depth(a.depth ? a.depth + (size_t)b * a.depth_stride : nullptr),
          tree(a.tree ? a.tree + (size_t)b * a.tree_stride : nullptr)
    {
    }
    // of new token u; kept where differences do not overflow
    __device__ __forceinline__ int position(int u) const
    {
        const int p = __builtin_elementwise_add_sat(len, depth ? depth[u] : u);
        return min(max(p, -kFar), kFar);
    }
};

// What the workgroups that have new tokens among their keys look up in LDS: the masks of their rows, the positions of the new tokens.
template <int ROWS>
struct Lookup {
    uint64_t mask[ROWS][kMaskWords];
    int at[kMaxTokens];
};
// One row of queries of a lane.
struct Row {
    int tok;                       // its token, -1: padding
    const uint64_t *mask;          // its words, in LDS
    int at;                        // position and slope (times log2 e): with FORMS
    float slope;
};

// Scores as they come out of the product: factors to units of log2 e (without a cap), and the forms of the score.
template <int HD, int FMT>
__device__ __forceinline__ float score_factor(float cap)
{
    const float unit = (FMT == CF_CACHE_INT8 ? cf::tree::kInt8Unit : 1.f) * (HD == 64 ? 0.125f : 0.08838834764831845f) * kLog2e;
    return cap > 0.f ? unit * 2.f / cap : unit;                    // with a cap: twice its share of the cap, for the tanh
}

// tanh(y) for x = 2 y log2(e): 1 - 2 / (2^x + 1), which is off by 2^-23 of one, and for |x| < 1/2, where that would be much of the result,
// the odd series of tanh up to the seventh power (the ninth is less than 2^-25 of it).
__device__ __forceinline__ float tanh_(float x)
{
    constexpr float h = 0.34657359027997265f, h2 = h * h;           // y = h x
    const float far = 1.f - 2.f * __builtin_amdgcn_rcpf(exp2_(x) + 1.f), z = x * x * h2;
    const float near = x * h * fmaf(fmaf(fmaf(-17.f / 315.f, z, 2.f / 15.f), z, -1.f / 3.f), z, 1.f);
    return fabsf(x) < 0.5f ? near : far;
}

// Arguments x_j of a row for two tiles of 16 keys from j0 on; minus infinity for a key that it does not see.
template <int FMT, bool FORMS>
__device__ __forceinline__ void arguments(const TreeArgs &a, const Sequence &sq, const int *new_at, const Row &row, int g, int j0, bool masked, float to_score,
                                          const f32x4 (&s)[2], const f32x4 (&kscale)[2], float (&x)[8], bool (&sees)[8])
{
    const uint32_t bits = masked ? seen_bits(sq.tree != nullptr, a.words, row.mask, row.tok, j0, sq.len, sq.n) : ~0u;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int i = 16 * (e >> 2) + 4 * g + (e & 3), j = j0 + i;
        x[e] = s[e >> 2][e & 3] * (kRowScale<FMT> ? kscale[e >> 2][e & 3] : to_score);
        bool seen = bits >> i & 1;
        if constexpr (FORMS) {
            int key_at = j;
            if (masked) {
                int theirs = new_at[min(max(j - sq.len, 0), sq.n - 1)];
                asm volatile("" : "+v"(theirs));                    // (no branch around the load)
                key_at = j >= sq.len ? theirs : j;
            }
            const int distance = row.at - key_at;
            if (a.cap > 0.f) x[e] = a.cap * kLog2e * tanh_(x[e]);
            x[e] -= row.slope * (float)distance;
            if (masked && a.window > 0) seen = seen && distance < a.window;
        }
        x[e] = seen ? x[e] : -INFINITY;
        sees[e] = seen;
    }
}

// What a row has summed so far.
template <int HD>
struct Sums {
    float mm, l;
    f32x4 acc[HD / 16];
    __device__ __forceinline__ Sums() : mm(kNone), l(0.f)
    {
#pragma unroll
        for (int j = 0; j < HD / 16; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
};

// The weights of NR rows for two tiles of 16 keys from j0 on, as B operands of the second product.  masked: some row of the workgroup does
// not see all of these keys.  Where a row's reference is large, x_j - mm has to be the difference of rounded numbers (the fused multiply-add
// keeps bits of x_j that mm, which was taken from a rounded one, lacks: above 2^24 that is whole powers of two); careful: some row of the
// wavefront has such a reference, and each row looks at its own.  Whether a row moves its reference, and to where, is its own matter as well:
// the other rows of the wavefront go through the second pass with the weights that they had.
constexpr float kCareful = 0x1p20f;
template <int HD, int FMT, bool FORMS, int NR>
__device__ __forceinline__ void weigh(const TreeArgs &a, const Sequence &sq, const int *new_at, const Row (&row)[NR], int g, int j0, bool masked, bool &careful,
                                      float to_score, const f32x4 (&s)[NR][2], const f32x4 (&kscale)[2], const f32x4 (&vscale)[2], Sums<HD> (&sum)[NR],
                                      h8 (&w)[NR])
{
    constexpr bool SCALED = kRowScale<FMT>;
    float add[NR], most[NR];
    for (int pass = 0;; ++pass) {
        float highest = 0.f;
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            float p[8], wt[8];
            bool sees[8];
            if (FORMS || masked || careful) {
                const bool large = fabsf(sum[r].mm) > kCareful;
                arguments<FMT, FORMS>(a, sq, new_at, row[r], g, j0, masked, to_score, s[r], kscale, p, sees);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float rounded = p[e] - sum[r].mm;
                    float y = rounded;
                    if (!FORMS && !masked) {
                        const float fused = fmaf(s[r][e >> 2][e & 3], SCALED ? kscale[e >> 2][e & 3] : to_score, -sum[r].mm);
                        y = large ? rounded : fused;
                    }
                    p[e] = exp2_(y);
                    wt[e] = SCALED ? (sees[e] ? p[e] * vscale[e >> 2][e & 3] : 0.f) : p[e];       // (the scale of an unseen row may be anything)
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    p[e] = exp2_(fmaf(s[r][e >> 2][e & 3], SCALED ? kscale[e >> 2][e & 3] : to_score, -sum[r].mm));
                    wt[e] = SCALED ? p[e] * vscale[e >> 2][e & 3] : p[e];
                }
            }
            add[r] = ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
            most[r] = 0.f;
#pragma unroll
            for (int e = 0; e < 8; e += 2) most[r] = fmaxf(fmaxf(most[r], wt[e]), wt[e + 1]);
            highest = r ? fmaxf(highest, most[r]) : most[r];
#pragma unroll
            for (int e = 0; e < 8; ++e) w[r][e] = (_Float16)wt[e];
        }
        if (pass || !__any(highest > kMostWeight)) break;
        // some weight is too large: rows with such a one get a new reference, and all weights are taken again
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            float x[8], top = kNone;
            bool sees[8];
            arguments<FMT, FORMS>(a, sq, new_at, row[r], g, j0, masked, to_score, s[r], kscale, x, sees);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float y = x[e] == -INFINITY ? kNone : SCALED ? x[e] + __builtin_amdgcn_logf(vscale[e >> 2][e & 3]) : x[e];
                top = fmaxf(top, y);
            }
            top = cf::lanes::max_groups<16>(top);
            const bool moves = cf::lanes::max_groups<16>(most[r]) > kMostWeight;
            const float to = moves ? top - kTopExponent : sum[r].mm, by = moves ? exp2_(sum[r].mm - to) : 1.f;
            sum[r].mm = to;
            sum[r].l *= by;
#pragma unroll
            for (int j = 0; j < HD / 16; ++j) sum[r].acc[j] *= by;
            careful = careful || __any(moves && fabsf(to) > kCareful);
        }
    }
#pragma unroll
    for (int r = 0; r < NR; ++r) sum[r].l += add[r];
}

// The same for tree_fours, without scales of rows, and with the ordinary way of all rows apart: 16 registers fewer there and, without a branch for
// every row, 9 % less time at 32 rows a wavefront.  (The other kernels, whose scales are in the way, would need more registers.)  The sums l are
// those of the rounded weights, by a product with ones (total): a rounding then moves a result towards or away from a value by the difference to
// it alone, and the additions cost nothing.  (Root mean square error of the results of one token over 256 rows against fp64, 12 inputs, at most:
// 2.8e-4 of them, 3.4e-4 with sums of what was not rounded, 2.1e-4 is their own rounding to fp16; times alike.)
//
// Exponentials, which are the weights, as an operand, and the largest one.
__device__ __forceinline__ void take(const float (&p)[8], h8 &w, float &most)
{
    most = 0.f;
#pragma unroll
    for (int e = 0; e < 8; e += 2) most = fmaxf(fmaxf(most, p[e]), p[e + 1]);
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = (_Float16)p[e];
}
template <int HD, int FMT, bool FORMS, int NR>
__device__ __forceinline__ void weigh_apart(const TreeArgs &a, const Sequence &sq, const int *new_at, const Row (&row)[NR], int g, int j0, bool masked, bool &careful,
                                            float to_score, const f32x4 (&s)[NR][2], Sums<HD> (&sum)[NR], f32x4 (&total)[NR], h8 (&w)[NR])
{
    static_assert(!kRowScale<FMT>, "no scales");
    const f32x4 none[2] = {};
    float most[NR], highest = 0.f;
    const bool ordinary = !(FORMS || masked || careful);
    if (ordinary)
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            float p[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) p[e] = exp2_(fmaf(s[r][e >> 2][e & 3], to_score, -sum[r].mm));
            take(p, w[r], most[r]);
            highest = r ? fmaxf(highest, most[r]) : most[r];
        }
    if (!ordinary || __any(highest > kMostWeight))
        for (int pass = ordinary;; ++pass) {
            if (pass)
                // some weight is too large: rows with such a one get a new reference
#pragma unroll
                for (int r = 0; r < NR; ++r) {
                    float x[8], top = kNone;
                    bool sees[8];
                    arguments<FMT, FORMS>(a, sq, new_at, row[r], g, j0, masked, to_score, s[r], none, x, sees);
#pragma unroll
                    for (int e = 0; e < 8; ++e) top = fmaxf(top, x[e] == -INFINITY ? kNone : x[e]);
                    top = cf::lanes::max_groups<16>(top);
                    const bool moves = cf::lanes::max_groups<16>(most[r]) > kMostWeight;
                    const float to = moves ? top - kTopExponent : sum[r].mm, by = moves ? exp2_(sum[r].mm - to) : 1.f;
                    sum[r].mm = to;
                    total[r] *= by;
#pragma unroll
                    for (int j = 0; j < HD / 16; ++j) sum[r].acc[j] *= by;
                    careful = careful || __any(moves && fabsf(to) > kCareful);
                }
            highest = 0.f;
#pragma unroll
            for (int r = 0; r < NR; ++r) {
                float p[8];
                bool sees[8];
                const bool large = fabsf(sum[r].mm) > kCareful;
                arguments<FMT, FORMS>(a, sq, new_at, row[r], g, j0, masked, to_score, s[r], none, p, sees);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float rounded = p[e] - sum[r].mm;
                    float y = rounded;
                    if (!FORMS && !masked) {
                        const float fused = fmaf(s[r][e >> 2][e & 3], to_score, -sum[r].mm);
                        y = large ? rounded : fused;
                    }
                    p[e] = exp2_(y);
                }
                take(p, w[r], most[r]);
                highest = fmaxf(highest, most[r]);
            }
            if (pass || !__any(highest > kMostWeight)) break;
        }
}

// A value that is infinite or NaN, and that a row sees, makes that dimension of its result infinite or NaN, however small the weight: the
// weight of a key that a row sees is more than 0, though fp16 and fp32 may not hold it.  Products would give 0 times infinity there, and also
// to the rows that do not see the key.  So steps in which some row does not see all keys leave such values out of the product, and where some
// were left out, or results are not finite, the threads that wrote results look over the keys once more and write the infinities and NaN that
// their rows see.  (Behind their stores: between the loop and the join the jump across this code cost a call of 7.3 us, one token over 512 e4m3
// rows, up to 0.3.)
//
// The sums of those among P pieces of W adjacent values, from dimension d0 + 16 p on, of the 32 keys from j0 on, for one row of queries.
// (vr: the rows, in 4 bits their scales.)
template <int HD, int FMT, bool FORMS, int P, int W>
__device__ __forceinline__ void add_unfit(const TreeArgs &a, const Sequence &sq, const int *new_at, const Row &row, __amdgpu_buffer_rsrc_t vr, int j0, int c, int g,
                                          int d0, float (&special)[P][W])
{
    constexpr int VB = kValueBytes<FMT>, ROW = HD * VB, DW = W * VB / 4, SROW = HD / kBlock;
    uint32_t some = 0;                                              // is there one at all
    if constexpr (FMT == CF_CACHE_MXFP4) {
#pragma unroll
        for (int i = 0; i < SROW / 2; ++i) some |= __builtin_amdgcn_raw_buffer_load_b8(vr, (uint32_t)j0 * SROW + 64 * i + 16 * g + c, 0, 0) == 255;
    } else {
        Values<HD, FMT> vals;
        vals.load(vr, Values<HD, FMT>::offset(c, g) + (uint32_t)j0 * ROW);
        some = vals.take_out_unfit();
    }
    if (!__any(some)) return;
    const uint32_t bits = seen_bits(sq.tree != nullptr, a.words, row.mask, row.tok, j0, sq.len, sq.n);
#pragma unroll 1
    for (int i = 0; i < 32; ++i) {
        bool seen = bits >> i & 1;
        if (FORMS && a.window > 0) {
            const int key_at = j0 + i < sq.len ? j0 + i : new_at[min(j0 + i - sq.len, sq.n - 1)];
            seen = seen && row.at - key_at < a.window;
        }
        if constexpr (FMT == CF_CACHE_MXFP4) {
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const bool bad = __builtin_amdgcn_raw_buffer_load_b8(vr, (uint32_t)(j0 + i) * SROW + (d0 + 16 * p) / kBlock, 0, 0) == 255;
#pragma unroll
                for (int e = 0; e < W; ++e) special[p][e] += seen && bad ? __builtin_nanf("") : 0.f;
            }
            continue;
        }
        uint32_t x[P][DW];
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int d = 0; d < DW; ++d) x[p][d] = __builtin_amdgcn_raw_buffer_load_b32(vr, (uint32_t)(j0 + i) * ROW + (d0 + 16 * p) * VB + 4 * d, 0, 0);
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int e = 0; e < W; ++e) {
                float v;
                if constexpr (FMT == CF_CACHE_F16)
                    v = (float)__builtin_bit_cast(_Float16, (uint16_t)(x[p][e / 2] >> 16 * (e & 1)));
                else
                    v = (x[p][e / 4] >> 8 * (e & 3) & 0x7f) == 0x7f ? __builtin_nanf("") : 0.f;
                special[p][e] += seen && !(fabsf(v) <= 65504.f) ? v : 0.f;
            }
    }
}

// Where a workgroup works: workgroup i runs on die i mod 8, and the row blocks of a unit (a sequence's head and part), which read the same
// keys and values, follow each other on one die.
struct Place {
    int unit, block, bh, split, b, head;                           // bh: batch row and KV head
    __device__ __forceinline__ explicit Place(const TreeArgs &a)
    {
        const int turn = blockIdx.x >> 3;
        unit = turn / a.blocks * 8 + (blockIdx.x & 7), block = turn % a.blocks;
        bh = unit / a.splits, split = unit - bh * a.splits;
        b = bh / a.nkv, head = bh - b * a.nkv;
    }
    __device__ __forceinline__ Place(const TreeArgs &a, int bh) : unit(0), block(0), bh(bh), split(0), b(bh / a.nkv), head(bh % a.nkv) {}
};

// Keys of a part in steps of STEP, counted from key 0, and from which key on all rows of the workgroup see all cached rows.
template <bool FORMS, int STEP>
struct Part {
    int begin, end, all_from;
    __device__ __forceinline__ Part(const TreeArgs &a, const Sequence &sq, const Place &at, int nearest, int farthest)
    {
        int lo = 0;
        all_from = 0;
        if (FORMS && a.window > 0) {
            lo = min(max(__builtin_elementwise_sub_sat(__builtin_amdgcn_readfirstlane(nearest), a.window) + 1, 0), sq.len);
            all_from = max(__builtin_elementwise_sub_sat(__builtin_amdgcn_readfirstlane(farthest), a.window) + 1, 0);
        }
        const int first = lo / STEP, steps = (sq.end + STEP - 1) / STEP - first, per = (steps + a.splits - 1) / a.splits;
        begin = first + at.split * per, end = min(first + steps, begin + per);
    }
    // Step i of the part, or the last one if there is none.  With forms from the last key to the first: under a bias that falls with the
    // distance the last keys have the largest scores, and references then move once and not in every step (one token over 2048 fp16 rows, one part
    // 35 -> 23 us).  Without forms from the first to the last: the step with the masks, which wait for LDS, does not come first (7 % over 256 rows).
    __device__ __forceinline__ bool has(int i) const { return i < end - begin; }
    __device__ __forceinline__ int at(int i) const { return FORMS ? max(end - 1 - i, begin) : min(begin + i, end - 1); }
};

// Queries of a row as B operands (dims(ks): first dimension of this lane's eight in contraction step ks) and what else a row has.
template <int HD, bool FORMS, typename Dims>
__device__ __forceinline__ Row load_row(const TreeArgs &a, const Sequence &sq, const Place &at, int index, const uint64_t *mask, h8 (&q)[HD / 32], int &nearest, int &farthest, Dims dims)
{
    const bool there = index / a.group < sq.n;
    const int from = min(index, sq.n * a.group - 1), t = from / a.group, hh = from - t * a.group;
    Row row = {there ? t : -1, mask, 0, 0.f};
    const uint16_t *src = a.q + (((size_t)at.b * a.rows.tokens + t) * a.nq + at.head * a.group + hh) * HD;
#pragma unroll
    for (int ks = 0; ks < HD / 32; ++ks) {
        const u32x4 x = *reinterpret_cast<const u32x4 *>(src + dims(ks));
        q[ks] = __builtin_bit_cast(h8, there ? x : u32x4{0u, 0u, 0u, 0u});
    }
    if constexpr (FORMS) {
        row.at = sq.position(t);
        row.slope = a.slopes ? a.slopes[at.head * a.group + hh] * kLog2e : 0.f;
        nearest = min(nearest, row.at), farthest = max(farthest, row.at);      // (a row of padding repeats the last one)
    }
    return row;
}
// Fills the rows first .. first + live - 1 of a Lookup; a barrier has to follow.
template <bool FORMS, int T, int ROWS>
__device__ __forceinline__ void fill(const TreeArgs &a, const Sequence &sq, int first, int live, Lookup<ROWS> &look_up)
{
    if (sq.tree)
        for (int i = threadIdx.x; i < live * a.words; i += T) {
            const int r = i / a.words, w = i - r * a.words;
            look_up.mask[r][w] = sq.tree[(size_t)((first + r) / a.group) * a.words + w];
        }
    if (FORMS)
        for (int u = threadIdx.x; u < sq.n; u += T) look_up.at[u] = sq.position(u);
}
__device__ __forceinline__ uint16_t *out_row(const TreeArgs &a, const Place &at, int index, int hd)
{
    const int t = index / a.group, hh = index - t * a.group;
    return a.out + (((size_t)at.b * a.rows.tokens + t) * a.nq + at.head * a.group + hh) * hd;
}
template <int FMT>
constexpr float kValueUnit = FMT == CF_CACHE_INT8 ? cf::tree::kInt8Unit : 1.f;

// ---- parts joined
//
// Partial results go through memory.  Either a second kernel joins them, or, where there is little to read, the workgroup whose part is done
// last: the parts are then written through to memory (the dies' L2 caches are not coherent), a counter tells which workgroup is the last,
// and that one reads past the caches.  Nobody waits for anybody.  (Written through, larger parts are slow: the 16-byte pieces do not meet in a
// cache any more; 64 tokens over 4096 e4m3 rows in 16 parts 35 us, 23 with cached writes.)
constexpr int kThrough = 16;       // cache policy: through to memory, from memory

struct Partials {
    __amdgpu_buffer_rsrc_t r;
    uint32_t ml;
    int hd;
    __device__ __forceinline__ Partials(const TreeArgs &a, int hd) : r(cf::buffer_of(a.part, a.part_bytes)), ml(a.part_ml), hd(hd) {}
    template <int AUX>
    __device__ __forceinline__ void put(uint32_t row, int dim, const f32x4 &v) const
    {
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), r, (row * hd + dim) * 4, 0, AUX);
    }
    template <int AUX>
    __device__ __forceinline__ void put_one(uint32_t row, int dim, float v) const
    {
        __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, v), r, (row * hd + dim) * 4, 0, AUX);
    }
    template <int AUX>
    __device__ __forceinline__ void put_ml(uint32_t row, float m, float l) const
    {
        __builtin_amdgcn_raw_buffer_store_b64(u32x2{__builtin_bit_cast(uint32_t, m), __builtin_bit_cast(uint32_t, l)}, r, ml + row * 8, 0, AUX);
    }
    template <int AUX>
    __device__ __forceinline__ f32x4 get(uint32_t row, int dim) const
    {
        return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(r, (row * hd + dim) * 4, 0, AUX));
    }
    template <int AUX>
    __device__ __forceinline__ float2 get_ml(uint32_t row) const
    {
        return __builtin_bit_cast(float2, __builtin_amdgcn_raw_buffer_load_b64(r, ml + row * 8, 0, AUX));
    }
};

// A factor of a part's sums that an infinity among them outlives.  (The sums are below 2^55, and 2^-126 of one is below 2^-70: no result shows
// it, with scales of values that fp16 holds.)
__device__ __forceinline__ float for_sums(float f) { return fmaxf(f, 0x1p-126f); }

// What T threads need to join rows.
template <int HD, int T>
struct JoinSpace {
    float sums[T / (HD / 8)][HD + 4];
    float2 ml[T / (HD / 8)];
};
// Rows first .. first + count - 1 of a sequence's head: eight dimensions of a row to a thread, its parts dealt to `lanes` (a power of two)
// threads, whose sums are added in their order.
template <int HD, int T, int AUX>
__device__ __forceinline__ void join_rows(const TreeArgs &a, const Place &at, int first, int count, int lanes, float unit_v, JoinSpace<HD, T> &space)
{
    constexpr int CH = HD / 8, SLOTS = T / CH;
    const Partials part(a, HD);
    const int slot = threadIdx.x / CH, d0 = 8 * (threadIdx.x % CH), lane = slot & (lanes - 1), per_pass = SLOTS / lanes;
    for (int r0 = 0; r0 < count; r0 += per_pass) {
        const int row = first + min(r0 + slot / lanes, count - 1);
        const uint32_t base = (uint32_t)at.bh * a.splits * a.padded + row;
        float m = kNone, total = 0.f;
        f32x4 o[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
        auto fold = [&](auto deep) {                                // parts that are requested together
            constexpr int DEEP = decltype(deep)::value;
            for (int s = lane; s < a.splits; s += DEEP * lanes) {
                float2 x[DEEP];
                f32x4 u[DEEP][2];
#pragma unroll
                for (int i = 0; i < DEEP; ++i) {
                    const uint32_t from = base + (uint32_t)min(s + i * lanes, a.splits - 1) * a.padded;
                    x[i] = part.get_ml<AUX>(from);
                    u[i][0] = part.get<AUX>(from, d0), u[i][1] = part.get<AUX>(from, d0 + 4);
                }
#pragma unroll
                for (int i = 0; i < DEEP; ++i) {
                    const bool there = s + i * lanes < a.splits;
                    const float to = there ? fmaxf(m, x[i].x) : m, old = exp2_(m - to), f = there ? exp2_(x[i].x - to) : 0.f;
                    m = to;
                    total = total * old + (there ? f * x[i].y : 0.f);
#pragma unroll
                    for (int h = 0; h < 2; ++h) o[h] = o[h] * for_sums(old) + (there ? u[i][h] * for_sums(f) : f32x4{0.f, 0.f, 0.f, 0.f});
                }
            }
        };
        if (a.splits <= lanes)
            fold(std::integral_constant<int, 1>());
        else if (a.splits <= 2 * lanes)
            fold(std::integral_constant<int, 2>());
        else
            fold(std::integral_constant<int, 4>());
        if (lanes == 1) {
            if (r0 + slot < count) {
                const float inv = total == 0.f ? 0.f : unit_v / total;
                h8 res;
#pragma unroll
                for (int e = 0; e < 8; ++e) res[e] = (_Float16)(o[e >> 2][e & 3] * inv);
                *reinterpret_cast<h8 *>(out_row(a, at, row, HD) + d0) = res;
            }
            continue;
        }
        if (r0) __syncthreads();
        *reinterpret_cast<f32x4 *>(&space.sums[slot][d0]) = o[0];
        *reinterpret_cast<f32x4 *>(&space.sums[slot][d0 + 4]) = o[1];
        if (d0 == 0) space.ml[slot] = make_float2(m, total);
        __syncthreads();
        for (int i = threadIdx.x; i < min(per_pass, count - r0) * (HD / 4); i += T) {      // four dimensions of a row to a thread
            const int mine = i / (HD / 4), d = 4 * (i % (HD / 4));
            float top = kNone, sum = 0.f;
            f32x4 x = {0.f, 0.f, 0.f, 0.f};
            for (int s = 0; s < lanes; ++s) top = fmaxf(top, space.ml[mine * lanes + s].x);
#pragma unroll 4
            for (int s = 0; s < lanes; ++s) {
                const float2 y = space.ml[mine * lanes + s];
                const float f = exp2_(y.x - top);
                sum += f * y.y;
                x += *reinterpret_cast<const f32x4 *>(&space.sums[mine * lanes + s][d]) * for_sums(f);
            }
            const float inv = sum == 0.f ? 0.f : unit_v / sum;
            typedef _Float16 h4 __attribute__((ext_vector_type(4)));
            *reinterpret_cast<h4 *>(out_row(a, at, first + r0 + mine, HD) + d) =
                h4{(_Float16)(x[0] * inv), (_Float16)(x[1] * inv), (_Float16)(x[2] * inv), (_Float16)(x[3] * inv)};
        }
    }
}
// Over what W dimensions of row i of the workgroup's block have: the infinities and NaN that the row sees.  (A row with a NaN among its scores
// stays NaN.)
template <int HD, int W>
__device__ __forceinline__ void put_special(const TreeArgs &a, const Place &at, int i, int d0, float total, const float (&special)[W])
{
    if (a.splits == 1) {
        uint16_t *dst = out_row(a, at, i, HD) + d0;
#pragma unroll
        for (int e = 0; e < W; ++e)
            if (special[e] != 0.f) dst[e] = __builtin_bit_cast(uint16_t, (_Float16)(special[e] + (total - total)));
        return;
    }
    const Partials to(a, HD);
    const uint32_t row = (uint32_t)at.unit * a.padded + i;
    const auto put = [&](auto aux) {
#pragma unroll
        for (int e = 0; e < W; ++e)
            if (special[e] != 0.f) to.put_one<decltype(aux)::value>(row, d0 + e, special[e]);
    };
    if (a.arrived)
        put(std::integral_constant<int, kThrough>());
    else
        put(std::integral_constant<int, 0>());
}

// Whether this workgroup, whose partial results are on their way, is the last one of its row block; it clears the counter for the next launch.
__device__ __forceinline__ bool last_to_arrive(const TreeArgs &a, const Place &at, int &shared)
{
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");                // this wavefront's results are in memory
    __syncthreads();
    if (threadIdx.x == 0) {
        uint32_t *counter = a.arrived + at.bh * a.blocks + at.block;
        const int before = (int)__hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (before == a.splits - 1) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        shared = before;
    }
    __syncthreads();
    return __builtin_amdgcn_readfirstlane(shared) == a.splits - 1;
}
// threads that share a row's parts
__device__ __forceinline__ int join_lanes(int splits, int rows, int slots)
{
    int lanes = 1;
    while (lanes < splits && 2 * lanes * rows <= slots) lanes *= 2;
    return lanes;
}

// What the wavefronts of tree_tiles and tree_fours share at their end, and the Lookup before it.
template <int HD>
struct alignas(16) TilesSums {
    float of[NW * 16 * (HD + 4)];
};
template <int HD, int NR>
struct TilesSpace {
    float2 ml[NW][16 * NR];
    Lookup<16 * NR> look_up;
    int left_out[NW];
    int before;
};
// Their sums joined, and the results stored or handed to the join of the parts.  vr: as for add_unfit.
template <int HD, int FMT, int NR, bool FORMS>
__device__ __forceinline__ void finish_tiles(const TreeArgs &a, const Sequence &sq, const Place &place, const Part<FORMS, kStep> &part, int first_row, int live,
                                             __amdgpu_buffer_rsrc_t vr, bool unfit, Sums<HD> (&sum)[NR], TilesSums<HD> &sums, TilesSpace<HD, NR> &space)
{
    constexpr int NJ = HD / 16;
    const int tid = threadIdx.x, wv = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, c = lane & 15, g = lane >> 4;
    float *smem = sums.of;
    auto &ml = space.ml;
    auto &look_up = space.look_up;
    auto &left_out = space.left_out;
    // 16 rows at a time
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        sum[r].l = cf::lanes::sum_groups<16>(sum[r].l);
        if (g == 0) ml[wv][16 * r + c] = make_float2(sum[r].mm, sum[r].l);
    }
    if (FMT != CF_CACHE_INT8 && lane == 0) left_out[wv] = unfit;
    float odd = 0.f;                                                // NaN where a result is not finite
    constexpr int CH = HD / 8;                                      // a thread has eight dimensions of a row
    const int row16 = tid / CH, d0 = 8 * (tid % CH);
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        __syncthreads();
#pragma unroll
        for (int rr = 0; rr < 4; ++rr)
#pragma unroll
            for (int j = 0; j < NJ; j += 4)
                if constexpr (FMT == CF_CACHE_MXFP4)                // (its sums are those of dimensions 16 j + 4 g .. 16 j + 4 g + 3)
                    *reinterpret_cast<f32x4 *>(smem + (wv * 16 + c) * (HD + 4) + 4 * NJ * rr + 4 * j + 4 * g) = sum[r].acc[(NJ * rr + j) / 4];
                else
                    *reinterpret_cast<float4 *>(smem + (wv * 16 + c) * (HD + 4) + NJ * (4 * g + rr) + j) =
                        make_float4(sum[r].acc[j][rr], sum[r].acc[j + 1][rr], sum[r].acc[j + 2][rr], sum[r].acc[j + 3][rr]);
        __syncthreads();
        const int i = 16 * r + row16;
        if (row16 < 16 && i < live) {
            float m = kNone, total = 0.f, o[8] = {};
#pragma unroll
            for (int k = 0; k < NW; ++k) m = fmaxf(m, ml[k][i].x);
#pragma unroll
            for (int k = 0; k < NW; ++k) {
                const float f = exp2_(ml[k][i].x - m);
                const float *src = smem + (k * 16 + row16) * (HD + 4) + d0;
                total += f * ml[k][i].y;
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] += f * src[e];
            }
            if (FMT != CF_CACHE_INT8) odd += ((o[0] + o[1]) + (o[2] + o[3])) * 0.f + ((o[4] + o[5]) + (o[6] + o[7])) * 0.f;
            if (a.splits > 1) {
                const Partials to(a, HD);
                const uint32_t at = (uint32_t)place.unit * a.padded + first_row + i;
                const f32x4 lo = {o[0], o[1], o[2], o[3]}, hi = {o[4], o[5], o[6], o[7]};
                if (a.arrived) {
                    to.put<kThrough>(at, d0, lo), to.put<kThrough>(at, d0 + 4, hi);
                    if (d0 == 0) to.put_ml<kThrough>(at, m, total);
                } else {
                    to.put<0>(at, d0, lo), to.put<0>(at, d0 + 4, hi);
                    if (d0 == 0) to.put_ml<0>(at, m, total);
                }
            } else {
                const float inv = total == 0.f ? 0.f : kValueUnit<FMT> / total;
                h8 res;
#pragma unroll
                for (int e = 0; e < 8; ++e) res[e] = (_Float16)(o[e] * inv);
                *reinterpret_cast<h8 *>(out_row(a, place, first_row + i, HD) + d0) = res;
            }
        }
    }
    if constexpr (FMT != CF_CACHE_INT8) {
        const bool all = __any(odd != 0.f);
        if (all || __builtin_amdgcn_readfirstlane(left_out[0] | left_out[1] | left_out[2] | left_out[3])) {
#pragma unroll 1
            for (int r = 0; r < NR; ++r) {
                const int i = min(16 * r + row16, live - 1);
                const int tok = (first_row + i) / a.group;
                const Row mine = {tok, look_up.mask[i], FORMS ? sq.position(tok) : 0, 0.f};
                float special[1][8] = {}, total = 0.f;
                for (int k = 0; k < NW; ++k) total += ml[k][i].y;
                for (int s = part.begin; s < part.end; ++s)
                    if (all || (s + 1) * kStep > sq.len || s * kStep < part.all_from)
                        add_unfit<HD, FMT, FORMS, 1, 8>(a, sq, look_up.at, mine, vr, s * kStep, c, g, d0, special);
                if (row16 < 16 && 16 * r + row16 < live) put_special<HD, 8>(a, place, first_row + i, d0, total, special[0]);
            }
        }
    }
    if (a.splits > 1 && a.arrived) {
        if (last_to_arrive(a, place, space.before))
            join_rows<HD, NT, kThrough>(a, place, first_row, live, join_lanes(a.splits, live, NT / CH), kValueUnit<FMT>, *reinterpret_cast<JoinSpace<HD, NT> *>(smem));
    }
}

// Few rows: reading the keys and values is the work.  Every wavefront has its own steps, so that no barrier holds up its loads: the next step's
// keys are requested as soon as this one's are used, and its values.  The four wavefronts' sums are joined once, through LDS.
// Bound: memory where the cache is long (one token over 32768 e4m3 rows, 64 heads: 69 MB in 14.0 us, 4.9 TB/s, then the join; a copy
// reaches 4.8), the chain launch - lengths - queries - keys - values - sums where it is short (256 rows 5.9 us from launch to launch).  In
// between a wavefront waits for its one step of loads: 64 tokens over 4096 e4m3 rows 41 % of its time, the matrix units busy 13 %.
// Eight wavefronts to a workgroup were 5 % slower over 117 shapes: they start later and have more to join.
// FORMS: the scores may be capped, biased or windowed.
template <int HD, int FMT, int NR, bool FORMS>
__global__ __launch_bounds__(NT, 2) void tree_tiles(const TreeArgs a)
{
    constexpr int KS = HD / 32, NJ = HD / 16, ROW = HD * kValueBytes<FMT>;
    constexpr bool SCALED = kRowScale<FMT>;
    __shared__ TilesSums<HD> sums;
    __shared__ TilesSpace<HD, NR> space;
    __shared__ alignas(16) float scales[NW][2][kStep];
    Lookup<16 * NR> &look_up = space.look_up;
    const int tid = threadIdx.x, wv = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, c = lane & 15, g = lane >> 4;
    const Place place(a);
    if (place.unit >= a.units) return;
    const Sequence sq(a, place.b);
    const int first_row = place.block * (16 * NR), live = min(sq.n * a.group - first_row, 16 * NR);
    if (live <= 0) return;

    h8 q[NR][KS];
    Row row[NR];
    int nearest = kFar, farthest = -kFar;                           // of the positions of the block's tokens
#pragma unroll
    for (int r = 0; r < NR; ++r)
        row[r] = load_row<HD, FORMS>(a, sq, place, first_row + 16 * r + c, look_up.mask[16 * r + c], q[r], nearest, farthest, [&](int ks) { return Keys<HD, FMT>::dim(ks, g); });
    if (FORMS && a.window > 0)
#pragma unroll
        for (int s = 1; s < 16; s <<= 1) nearest = min(nearest, __shfl_xor(nearest, s)), farthest = max(farthest, __shfl_xor(farthest, s));
    const Part<FORMS, kStep> part(a, sq, place, nearest, farthest);

    const size_t slice = (size_t)place.bh * a.max_seq;
    const __amdgpu_buffer_rsrc_t kr = cf::buffer_of(a.k + slice * ROW, (uint32_t)sq.end * ROW), vr = cf::buffer_of(a.v + slice * ROW, (uint32_t)sq.end * ROW);
    const float *scale_src = SCALED ? (lane < 32 ? a.k_scale : a.v_scale) + slice : nullptr;
    const float to_score = score_factor<HD, FMT>(FORMS ? a.cap : 0.f);

    Keys<HD, FMT> keys;
    Values<HD, FMT> vals;
    float scale = 0.f;
    Sums<HD> sum[NR];
    bool careful = false, unfit = false;                            // unfit: infinities or NaN were left out of the product
    const uint32_t koff = Keys<HD, FMT>::offset(c, g), voff = Values<HD, FMT>::offset(c, g);
    auto load_scale = [&](int step) {
        if constexpr (SCALED) scale = scale_src[min(step * kStep + (lane & 31), sq.end - 1)];
    };
    int step = part.at(wv);
    if (part.has(wv)) {
        load_scale(step);
        keys.load(kr, koff + (uint32_t)step * (kStep * ROW));
        vals.load(vr, voff + (uint32_t)step * (kStep * ROW));
    }
    if (part.end * kStep > sq.len) {
        fill<FORMS, NT>(a, sq, first_row, live, look_up);
        lds_barrier();
    }
    for (int i = wv; part.has(i); i += NW) {
        const int j0 = step * kStep;
        const bool masked = j0 + kStep > sq.len || j0 < part.all_from;      // (the same for the whole wavefront)
        const int next = part.at(i + NW);
        if constexpr (SCALED) {
            const float x = lane < 32 ? scale * to_score : at_least_small(scale);
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
        keys.load(kr, koff + (uint32_t)next * (kStep * ROW));
        f32x4 kscale[2], vscale[2];
        if constexpr (SCALED) {
            wave_sync();
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                kscale[t] = *reinterpret_cast<const f32x4 *>(&scales[wv][0][16 * t + 4 * g]);
                vscale[t] = *reinterpret_cast<const f32x4 *>(&scales[wv][1][16 * t + 4 * g]);
            }
            wave_sync();
            load_scale(next);
        }
        h8 w[NR];
        weigh<HD, FMT, FORMS, NR>(a, sq, look_up.at, row, g, j0, masked, careful, to_score, s, kscale, vscale, sum, w);
        // ---- values
        if (FMT != CF_CACHE_INT8 && masked) unfit = __any(vals.take_out_unfit()) || unfit;
        vals.flip();
#pragma unroll
        for (int pair = 0; pair < NJ / 2; ++pair) {
            h8 v[2];
            vals.operands(pair, v);
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int r = 0; r < NR; ++r) sum[r].acc[2 * pair + j] = mfma16(v[j], w[r], sum[r].acc[2 * pair + j]);
        }
        vals.load(vr, voff + (uint32_t)next * (kStep * ROW));
        step = next;
    }

    finish_tiles<HD, FMT, NR, FORMS>(a, sq, place, part, first_row, live, vr, unfit, sum, sums, space);
}

// Staged steps: 64 rows of keys and of values as fp16 in LDS, two steps deep.  A row of keys is 16 bytes longer than its values, so that the
// sixteen rows of an operand start in different banks; a row of values 32 bytes, for the transposing reads of four rows by 16 dimensions.
constexpr int kBlockStep = 64;
template <int HD>
struct alignas(16) Stage {
    static constexpr int KROW = 2 * HD + 16, VROW = 2 * HD + 32;
    char k[2][kBlockStep * KROW], v[2][kBlockStep * VROW];
    float scale[2][2][kBlockStep];
};

// A row's 16-byte chunks (eight dimensions) in LDS: those of the second half of 128 dimensions change places in pairs.  The eight lanes that
// write a row of 8-bit values, two chunks each, then write to all 32 banks at a time and not twice to every other four.
__device__ __forceinline__ int chunk_at(int chunk) { return chunk ^ (chunk >> 3 & 1); }

typedef short s16x4 __attribute__((ext_vector_type(4)));
// A operand of 16 dimensions from dim on and the keys of one h8 of weights: of keys first + 4 g .. + 3 and first + 16 + 4 g .. + 3.
template <int VROW>
__device__ __forceinline__ h8 transposed(const char *v, int first, int dim, int c, int g)
{
    using Ptr = __attribute__((address_space(3))) s16x4 *;
    const int of_row = dim < 64 ? c & 3 : (c & 3) ^ 2;              // (dim is a constant, chunk_at of dim / 8 + (c & 3) / 2)
    const char *at = v + (first + 4 * g + (c >> 2)) * VROW + 2 * (dim + 4 * of_row);
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Ptr)at), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Ptr)(at + 16 * VROW));
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    return __builtin_bit_cast(h8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// RW wavefronts with 16 NR rows each share the steps of a part; with KG = 2 there are two such groups, one for each half of a step, whose
// sums are joined at the end.  (One group needs 1.15 us for a step of 128 dimensions when it has the compute unit for itself, most of it
// the time from one instruction to the next that needs its result.)
// Bound with many rows: no unit is full.  16 x 64 tokens over 8192 int8 rows, 32 heads: 138 GFLOP in 165 to 176 us, 0.78 to 0.84 PFLOP/s (a
// large fp16 product reaches 1.24); of the 337 thousand cycles that a compute unit is busy its matrix units are for 132 thousand, each SIMD
// issues vector instructions for 173 thousand, and a wavefront waits for 34 % of its time.  Products, weights and products of a wavefront
// follow each other (timed by phases, of 2190 cycles for half a step of 32 int8 keys by 32 rows, 128 dimensions, 590 were the scores'
// products, 1090 the weights, 510 the values' products), and the two wavefronts of a SIMD overlap in part only.
// Two groups in antiphase, steps of 128 keys and requests two steps ahead were 0 to 15 % slower.
template <int HD, int FMT, int RW, int KG, int NR, bool FORMS>
__global__ __launch_bounds__(64 * RW * KG, 2) void tree_blocks(const TreeArgs a)
{
    constexpr int WV = RW * KG, KS = HD / 32, NJ = HD / 16, ROW = HD * kValueBytes<FMT>, T = 64 * WV;
    constexpr bool SCALED = kRowScale<FMT>;
    // 16-byte pieces of a row; of the keys of a step, to a thread.  Where there are more threads than pieces the first ones have the keys,
    // the last ones the values.
    constexpr int PPR = ROW / 16, ALL = kBlockStep * PPR, PIECES = ALL < T ? 1 : ALL / T, APART = ALL < T ? T - ALL : 0;
    static_assert(ALL % T == 0 || 2 * ALL == T, "every thread stages as much");
    using S = Stage<HD>;
    __shared__ S lds;
    __shared__ Lookup<16 * NR * RW> look_up;
    __shared__ int left_out;                                        // infinities or NaN were left out of the product
    const int tid = threadIdx.x, wv = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, c = lane & 15, g = lane >> 4;
    const Place place(a);
    if (place.unit >= a.units) return;
    const Sequence sq(a, place.b);
    const int first_row = place.block * (16 * NR * RW), live = min(sq.n * a.group - first_row, 16 * NR * RW);
    if (live <= 0) return;
    const int my_rows = 16 * NR * (wv % RW), my_half = wv / RW;     // first of this wavefront's rows in the block, its half of a step

    h8 q[NR][KS];
    Row row[NR];
    int nearest = kFar, farthest = -kFar;
#pragma unroll
    for (int r = 0; r < NR; ++r)
        row[r] = load_row<HD, FORMS>(a, sq, place, first_row + my_rows + 16 * r + c, look_up.mask[my_rows + 16 * r + c], q[r], nearest, farthest, [&](int ks) { return 32 * ks + 8 * g; });
    if (FORMS && a.window > 0) {                                    // the part is the whole block's: its extremes by way of LDS
#pragma unroll
        for (int s = 1; s < 16; s <<= 1) nearest = min(nearest, __shfl_xor(nearest, s)), farthest = max(farthest, __shfl_xor(farthest, s));
        int *ends = reinterpret_cast<int *>(lds.k[0]);
        if (lane == 0) ends[2 * wv] = nearest, ends[2 * wv + 1] = farthest;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < WV; ++i) nearest = min(nearest, ends[2 * i]), farthest = max(farthest, ends[2 * i + 1]);
        __syncthreads();
    }
    const Part<FORMS, kBlockStep> part(a, sq, place, nearest, farthest);

    const size_t slice = (size_t)place.bh * a.max_seq;
    const __amdgpu_buffer_rsrc_t kr = cf::buffer_of(a.k + slice * ROW, (uint32_t)sq.end * ROW), vr = cf::buffer_of(a.v + slice * ROW, (uint32_t)sq.end * ROW);
    const float *scale_src = SCALED ? (wv == 1 ? a.v_scale : a.k_scale) + slice : nullptr;
    const float to_score = score_factor<HD, FMT>(FORMS ? a.cap : 0.f);

    Sums<HD> sum[NR];
    bool careful = false;

    // ---- staging: requested a step ahead of the one that is written, which is a step ahead of the one that is used
    u32x4 kraw[PIECES], vraw[PIECES];
    float scale = 0.f;
    auto request = [&](int step) {
        const uint32_t off = (uint32_t)step * (kBlockStep * ROW) + 16 * tid;
        if (!APART || 64 * wv < ALL)
#pragma unroll
            for (int i = 0; i < PIECES; ++i) kraw[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(kr, off + 16 * T * i, 0, 0));
        if (!APART || 64 * wv >= APART)
#pragma unroll
            for (int i = 0; i < PIECES; ++i) vraw[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(vr, off + 16 * (T * i - APART), 0, 0));
        if (SCALED && wv < 2) scale = scale_src[min(step * kBlockStep + lane, sq.end - 1)];
    };
    auto masked_step = [&](int step) { return (step + 1) * kBlockStep > sq.len || step * kBlockStep < part.all_from; };
    auto write = [&](int i) {
        const int buf = i & 1, step = part.at(i);
        const bool look = FMT != CF_CACHE_INT8 && masked_step(step);
        uint32_t odd = 0;
        auto put = [&](char *rows, int row_bytes, u32x4 raw, int piece, bool check) {
            if (check)
#pragma unroll
                for (int d = 0; d < 4; ++d) odd |= cf::tree::unfit_bits<FMT>(raw[d]), raw[d] = cf::tree::without_unfit<FMT>(raw[d]);
            char *dst = rows + piece / PPR * row_bytes;
            const int col = piece % PPR;
            if constexpr (FMT == CF_CACHE_F16) {
                *reinterpret_cast<u32x4 *>(dst + 16 * chunk_at(col)) = raw;
            } else {
                *reinterpret_cast<u32x4 *>(dst + 16 * chunk_at(2 * col)) = cf::tree::widen<FMT>(raw[0], raw[1]);
                *reinterpret_cast<u32x4 *>(dst + 16 * chunk_at(2 * col + 1)) = cf::tree::widen<FMT>(raw[2], raw[3]);
            }
        };
        if (!APART || 64 * wv < ALL)
#pragma unroll
            for (int i = 0; i < PIECES; ++i) put(lds.k[buf], S::KROW, kraw[i], tid + T * i, false);
        if (!APART || 64 * wv >= APART)
#pragma unroll
            for (int i = 0; i < PIECES; ++i) put(lds.v[buf], S::VROW, vraw[i], tid + T * i - APART, look);
        if (look && __any(odd)) left_out = 1;
        if (SCALED && wv < 2)
            lds.scale[buf][wv][lane] = wv == 0 ? scale * to_score : at_least_small(scale);
    };
    if (tid == 0) left_out = 0;
    if (part.begin < part.end) {
        request(part.at(0));
        if (part.end * kBlockStep > sq.len) fill<FORMS, T>(a, sq, first_row, live, look_up);
        lds_barrier();
        write(0);
        request(part.at(1));
    }
    for (int i = 0; part.has(i); ++i) {
        lds_barrier();                                              // this step is written, and the other buffer has been read
        if (part.has(i + 1)) {
            write(i + 1);
            request(part.at(i + 2));
        }
        if (my_rows >= live) continue;                              // a wavefront without rows only stages
        const int buf = i & 1, step = part.at(i), j0 = step * kBlockStep;
        const char *kb = lds.k[buf], *vb = lds.v[buf];
        const bool masked = masked_step(step);
#pragma unroll
        for (int h = 0; h < 2 / KG; ++h) {
            const int half = KG == 2 ? my_half : h;
            f32x4 s[NR][2];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    const h8 k = *reinterpret_cast<const h8 *>(kb + (32 * half + 16 * t + c) * S::KROW + 64 * ks + 16 * (ks < 2 ? g : g ^ 1));
#pragma unroll
                    for (int r = 0; r < NR; ++r) s[r][t] = mfma16(k, q[r][ks], ks ? s[r][t] : f32x4{0.f, 0.f, 0.f, 0.f});
                }
            f32x4 kscale[2], vscale[2];
            if constexpr (SCALED) {
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    kscale[t] = *reinterpret_cast<const f32x4 *>(&lds.scale[buf][0][32 * half + 16 * t + 4 * g]);
                    vscale[t] = *reinterpret_cast<const f32x4 *>(&lds.scale[buf][1][32 * half + 16 * t + 4 * g]);
                }
            }
            h8 w[NR];
            weigh<HD, FMT, FORMS, NR>(a, sq, look_up.at, row, g, j0 + 32 * half, masked, careful, to_score, s, kscale, vscale, sum, w);
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                const h8 v = transposed<S::VROW>(vb, 32 * half, 16 * j, c, g);
#pragma unroll
                for (int r = 0; r < NR; ++r) sum[r].acc[j] = mfma16(v, w[r], sum[r].acc[j]);
            }
        }
    }

#pragma unroll
    for (int r = 0; r < NR; ++r) sum[r].l = cf::lanes::sum_groups<16>(sum[r].l);
    if constexpr (KG == 2) {
        constexpr int STRIDE = HD + 4;                              // floats of a row in LDS
        float *other = reinterpret_cast<float *>(&lds);
        float2 *other_ml = reinterpret_cast<float2 *>(other + 16 * NR * RW * STRIDE);
        static_assert(16 * NR * RW * (STRIDE * sizeof(float) + sizeof(float2)) <= sizeof(S), "the second group's sums where the steps were");
        __syncthreads();
        if (my_half)
#pragma unroll
            for (int r = 0; r < NR; ++r) {
                const int i = my_rows + 16 * r + c;
#pragma unroll
                for (int j = 0; j < NJ; ++j) *reinterpret_cast<f32x4 *>(other + i * STRIDE + 16 * j + 4 * g) = sum[r].acc[j];
                other_ml[i] = make_float2(sum[r].mm, sum[r].l);     // (the same from all four lanes of a row)
            }
        __syncthreads();
        if (!my_half)
#pragma unroll
            for (int r = 0; r < NR; ++r) {
                const int i = my_rows + 16 * r + c;
                const float2 x = other_ml[i];
                const float to = fmaxf(sum[r].mm, x.x), mine = exp2_(sum[r].mm - to), theirs = exp2_(x.x - to);
                sum[r].mm = to;
                sum[r].l = sum[r].l * mine + x.y * theirs;
#pragma unroll
                for (int j = 0; j < NJ; ++j) sum[r].acc[j] = sum[r].acc[j] * mine + *reinterpret_cast<const f32x4 *>(other + i * STRIDE + 16 * j + 4 * g) * theirs;
            }
    }
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        const int i = my_half ? live : my_rows + 16 * r + c;
        const float total = sum[r].l;
        if (i < live && a.splits > 1) {
            const Partials to(a, HD);
            const uint32_t at = (uint32_t)place.unit * a.padded + first_row + i;
            if (a.arrived) {
#pragma unroll
                for (int j = 0; j < NJ; ++j) to.put<kThrough>(at, 16 * j + 4 * g, sum[r].acc[j]);
                if (g == 0) to.put_ml<kThrough>(at, sum[r].mm, total);
            } else {
#pragma unroll
                for (int j = 0; j < NJ; ++j) to.put<0>(at, 16 * j + 4 * g, sum[r].acc[j]);
                if (g == 0) to.put_ml<0>(at, sum[r].mm, total);
            }
        } else if (i < live) {
            const float inv = total == 0.f ? 0.f : kValueUnit<FMT> / total;
            uint16_t *dst = out_row(a, place, first_row + i, HD) + 4 * g;
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                typedef _Float16 h4 __attribute__((ext_vector_type(4)));
                h4 res;
#pragma unroll
                for (int rr = 0; rr < 4; ++rr) res[rr] = (_Float16)(sum[r].acc[j][rr] * inv);
                *reinterpret_cast<h4 *>(dst + 16 * j) = res;
            }
        }
    }
    if (FMT != CF_CACHE_INT8 && !my_half && my_rows < live) {
        f32x4 odd = {0.f, 0.f, 0.f, 0.f};                           // NaN where a result is not finite
#pragma unroll
        for (int r = 0; r < NR; ++r)
#pragma unroll
            for (int j = 0; j < NJ; ++j) odd += sum[r].acc[j] * 0.f;
        const bool all = __any((odd[0] + odd[1]) + (odd[2] + odd[3]) != 0.f);
        if (part.begin < part.end && (all || __builtin_amdgcn_readfirstlane(left_out)))
#pragma unroll
            for (int r = 0; r < NR; ++r) {
                const int i = my_rows + 16 * r + c;
                float special[NJ][4] = {};
                for (int s = 2 * part.begin; s < 2 * part.end; ++s)
                    if (all || masked_step(s / 2)) add_unfit<HD, FMT, FORMS, NJ, 4>(a, sq, look_up.at, row[r], vr, s * kStep, c, g, 4 * g, special);
#pragma unroll
                for (int j = 0; j < NJ; ++j)
                    if (i < live) put_special<HD, 4>(a, place, first_row + i, 16 * j + 4 * g, sum[r].l, special[j]);
            }
    }
    if (a.splits > 1 && a.arrived) {
        __shared__ int before;
        static_assert(sizeof(JoinSpace<HD, T>) <= sizeof(S), "joined where the steps were");
        if (last_to_arrive(a, place, before))
            join_rows<HD, T, kThrough>(a, place, first_row, live, join_lanes(a.splits, live, T / (HD / 8)), kValueUnit<FMT>, *reinterpret_cast<JoinSpace<HD, T> *>(&lds));
    }
}

// The same over a cache held in 4 bits.  A code and its block's power of two make an fp16 number, so that the conversion to fp16 (one instruction for
// two values, the scale taken in) is all that the format costs, and the rest is as for fp16 rows.  A lane has a quarter of a key's row, which is its share
// of all of an operand's columns.  Values would need a transposition by codes of half a byte: a lane takes a block of 32 instead, with one scale, and
// puts it as fp16 where the transposing reads of LDS find it, in its wavefront's own rows, so that no barrier is needed.
// Bound: few rows as tree_tiles, by the chain of a step's loads (one token over 4096 rows, 32 heads, 10.7 us, 8.9 MB; over 32768 rows, 64 / 8 heads,
// 15.5 us, 36 MB); many rows by the instructions of a step, 0.76 us of 32 rows x 32 keys x 128 dimensions on a SIMD: conversions, weights and products
// take their turns there (64 tokens over 8192 rows, 32 / 8 heads, batch 16: 171 to 176 us, 0.8 PFLOP/s; tree_blocks with 4-bit staging the same; all
// in captured graphs: called one by one that batch takes 161 to 167 us, by card).
// Without gain: two or three steps of loads ahead in registers (1.4 us more in short calls: the code is larger) or in LDS, steps of 64 keys (long calls
// -6 %, short ones +1 us), the next step's scores among this one's weights, 64 rows a wavefront (206 us), three wavefronts a SIMD (176), products of
// 32 x 32 in place of 16 x 16 (184 against 171).
template <int HD, int NR, bool FORMS>
__global__ __launch_bounds__(NT, 2) void tree_fours(const TreeArgs a)
{
    constexpr int FMT = CF_CACHE_MXFP4, KS = HD / 32, NJ = HD / 16, ROW = HD / 2, SROW = HD / kBlock, VROW = 2 * HD + 32;
    __shared__ union alignas(16) {
        char values[NW][kStep * VROW];                              // of a wavefront's step
        TilesSums<HD> sums;
    } u;
    __shared__ TilesSpace<HD, NR> space;
    Lookup<16 * NR> &look_up = space.look_up;
    const int tid = threadIdx.x, wv = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, c = lane & 15, g = lane >> 4;
    const Place place(a);
    if (place.unit >= a.units) return;
    const Sequence sq(a, place.b);
    const int first_row = place.block * (16 * NR), live = min(sq.n * a.group - first_row, 16 * NR);
    if (live <= 0) return;

    h8 q[NR][KS];
    Row row[NR];
    int nearest = kFar, farthest = -kFar;                           // of the positions of the block's tokens
#pragma unroll
    for (int r = 0; r < NR; ++r)
        row[r] = load_row<HD, FORMS>(a, sq, place, first_row + 16 * r + c, look_up.mask[16 * r + c], q[r], nearest, farthest, [&](int ks) { return Keys4<HD>::dim(ks, g); });
    if (FORMS && a.window > 0)
#pragma unroll
        for (int s = 1; s < 16; s <<= 1) nearest = min(nearest, __shfl_xor(nearest, s)), farthest = max(farthest, __shfl_xor(farthest, s));
    const Part<FORMS, kStep> part(a, sq, place, nearest, farthest);

    const size_t slice = (size_t)place.bh * a.max_seq;
    const __amdgpu_buffer_rsrc_t kr = cf::buffer_of(a.k + slice * ROW, (uint32_t)sq.end * ROW), vr = cf::buffer_of(a.v + slice * ROW, (uint32_t)sq.end * ROW);
    const __amdgpu_buffer_rsrc_t ksr = cf::buffer_of(reinterpret_cast<const char *>(a.k_scale) + slice * SROW, (uint32_t)sq.end * SROW);
    const __amdgpu_buffer_rsrc_t vsr = cf::buffer_of(reinterpret_cast<const char *>(a.v_scale) + slice * SROW, (uint32_t)sq.end * SROW);
    const float to_score = score_factor<HD, FMT>(FORMS ? a.cap : 0.f);

    Keys4<HD> keys;
    Values4<HD, VROW> vals;
    Sums<HD> sum[NR];
    f32x4 total[NR] = {};
    h8 ones;                                                        // in the operand's first row: total[r][0] of the first 16 lanes
#pragma unroll
    for (int e = 0; e < 8; ++e) ones[e] = (_Float16)(c == 0 ? 1.f : 0.f);
    bool careful = false, unfit = false;                            // unfit: NaN were left out of the product
    int j0 = part.at(wv) * kStep;
    if (part.has(wv)) {
        keys.load(kr, ksr, j0, c, g);
        vals.load(vr, vsr, j0, lane);
    }
    if (part.end * kStep > sq.len) {
        fill<FORMS, NT>(a, sq, first_row, live, look_up);
        lds_barrier();
    }
    for (int i = wv; part.has(i); i += NW) {
        const bool masked = j0 + kStep > sq.len || j0 < part.all_from;      // (the same for the whole wavefront)
        const int next = part.at(i + NW) * kStep;
        // ---- scores
        f32x4 s[NR][2];
        keys.settle();
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const h8 k = keys.operand(t, ks);
#pragma unroll
                for (int r = 0; r < NR; ++r) s[r][t] = mfma16(k, q[r][ks], ks ? s[r][t] : f32x4{0.f, 0.f, 0.f, 0.f});
            }
        keys.load(kr, ksr, next, c, g);
        // ---- values, and weights: before the products of the unit's other wavefront (2 to 3 %)
        __builtin_amdgcn_s_setprio(1);
        vals.settle();
        if (masked) unfit = __any(vals.take_out_unfit()) || unfit;
        vals.store(u.values[wv], lane);
        vals.load(vr, vsr, next, lane);
        h8 w[NR];
        weigh_apart<HD, FMT, FORMS, NR>(a, sq, look_up.at, row, g, j0, masked, careful, to_score, s, sum, total, w);
        __builtin_amdgcn_s_setprio(0);
        wave_sync();
#pragma unroll
        for (int r = 0; r < NR; ++r) total[r] = mfma16(ones, w[r], total[r]);
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            const h8 v = transposed<VROW>(u.values[wv], 0, 16 * j, c, g);
#pragma unroll
            for (int r = 0; r < NR; ++r) sum[r].acc[j] = mfma16(v, w[r], sum[r].acc[j]);
        }
        wave_sync();
        j0 = next;
    }
#pragma unroll
    for (int r = 0; r < NR; ++r) sum[r].l = total[r][0];
    __syncthreads();                                                // the sums go where the values were
    finish_tiles<HD, FMT, NR, FORMS>(a, sq, place, part, first_row, live, vsr, unfit, sum, u.sums, space);
}

// The parts of a sequence joined by a kernel of its own: as many rows to a workgroup as its threads have.  Bound: memory, behind a launch
// (64 rows of 32 heads in 8 parts, 8 MB, 4.8 us; 256 rows of 128 heads in 2 parts, 34 MB, 9.4 us, 3.6 TB/s).
template <int HD>
__global__ __launch_bounds__(NT) void tree_join(const TreeArgs a, int lanes, float unit_v)
{
    __shared__ JoinSpace<HD, NT> space;
    const Place at(a, blockIdx.y);
    const int per = NT / (HD / 8) / lanes, first = blockIdx.x * per, count = min(per, a.rows.fresh(at.b) * a.group - first);
    if (count > 0) join_rows<HD, NT, 0>(a, at, first, count, lanes, unit_v, space);
}

using KernelFn = void (*)(const TreeArgs);
// How a call is divided.
struct Plan {
    int shape;                     // index into kShapes
    int blocks, splits;
    bool in_place;                 // the last workgroup of a row block joins its parts
};
// Rows of a workgroup: tree_tiles with one or two tiles of 16, tree_blocks with two groups of four wavefronts of one tile, four of two, or
// eight of two.  (fp16, 33 to 64 rows in two groups against one: 16 tokens over 8192 rows, batch 4 30.1 / 33.6 us.)  8-bit caches up to
// 128 rows take blocks of 32 rows, which read the codes several times, out of the die's L2 but for the first: 64 tokens over 4096 e4m3
// rows 20.3 / 22.1 us, 32 tokens over 8192 int8 rows, batch 4 32.8 / 37.0.  With forms of the score one tile to a wavefront (more do not
// fit the registers).
constexpr int kShapes = 5;
struct Shape {
    int rows, waves;
};
constexpr Shape kPlain[kShapes] = {{16, 4}, {32, 4}, {64, 8}, {128, 4}, {256, 8}};
constexpr Shape kPlain8[kShapes] = {{16, 4}, {32, 4}, {32, 4}, {32, 4}, {256, 8}};
constexpr Shape kForms[kShapes] = {{16, 4}, {16, 4}, {64, 8}, {128, 8}, {128, 8}};
// 4-bit caches take blocks of 32 rows, with forms of 16, for any number of rows.  (256 rows in eight such blocks against one of tree_blocks: 64 tokens,
// 8 KV heads, over 4096 rows, batch 1 / 4: 18.9 / 34.3 us against 31.7 / 44.8, over 8192 rows, batch 16: 172 both; with forms, 160 rows over 4096,
// batch 2: 31.3 us in blocks of 16, 40.3 of 32, 45.9 by tree_blocks.)
constexpr Shape kPlain4[kShapes] = {{16, 4}, {32, 4}, {32, 4}, {32, 4}, {32, 4}};
constexpr Shape kForms4[kShapes] = {{16, 4}, {16, 4}, {16, 4}, {16, 4}, {16, 4}};

const Shape (&shapes_of(const cf_cache_config &c, bool forms))[kShapes]
{
    if (c.format == CF_CACHE_MXFP4) return forms ? kForms4 : kPlain4;
    return forms ? kForms : c.format == CF_CACHE_F16 ? kPlain : kPlain8;
}

template <int HD, int FMT, bool FORMS>
KernelFn pick_shape(int shape)
{
    if constexpr (FORMS) {
        return shape < 2 ? tree_tiles<HD, FMT, 1, true> : shape == 2 ? tree_blocks<HD, FMT, 4, 2, 1, true> : tree_blocks<HD, FMT, 8, 1, 1, true>;
    } else if constexpr (FMT != CF_CACHE_F16) {
        return shape == 0 ? tree_tiles<HD, FMT, 1, false> : shape < 4 ? tree_tiles<HD, FMT, 2, false> : tree_blocks<HD, FMT, 8, 1, 2, false>;
    } else {
        static const KernelFn fn[kShapes] = {tree_tiles<HD, FMT, 1, false>, tree_tiles<HD, FMT, 2, false>, tree_blocks<HD, FMT, 4, 2, 1, false>,
                                             tree_blocks<HD, FMT, 4, 1, 2, false>, tree_blocks<HD, FMT, 8, 1, 2, false>};
        return fn[shape];
    }
}
template <int HD, bool FORMS>
KernelFn pick_four(int shape)
{
    if constexpr (FORMS) return tree_fours<HD, 1, true>;
    else return shape == 0 ? tree_fours<HD, 1, false> : tree_fours<HD, 2, false>;
}
template <int HD, bool FORMS>
KernelFn pick_format(int fmt, int shape)
{
    if (fmt == CF_CACHE_MXFP4) return pick_four<HD, FORMS>(shape);
    return fmt == CF_CACHE_F16 ? pick_shape<HD, CF_CACHE_F16, FORMS>(shape) : fmt == CF_CACHE_E4M3 ? pick_shape<HD, CF_CACHE_E4M3, FORMS>(shape) : pick_shape<HD, CF_CACHE_INT8, FORMS>(shape);
}
KernelFn pick(int hd, int fmt, int shape, bool forms)
{
    if (hd == 64) return forms ? pick_format<64, true>(fmt, shape) : pick_format<64, false>(fmt, shape);
    return forms ? pick_format<128, true>(fmt, shape) : pick_format<128, false>(fmt, shape);
}

// shape for `live` rows of a KV head, and the rows of its row blocks
int shape_of(int live)
{
    int i = 0;
    while (i < kShapes - 1 && live > 16 << i) ++i;
    return i;
}
int block_rows(const Shape (&shapes)[kShapes], int live)
{
    const int rows = shapes[shape_of(live)].rows;
    return (live + rows - 1) / rows * rows;
}

constexpr int kMaxSplits = 64;
// Parts that the last workgroup of a row block joins by itself have at most this many values (fp32) together, where there are many row
// blocks, whose join kernel would read as much again, the second number.  (Against the join kernel: up to 4096 values -0.7 us, 8192 to 10240
// -0.3, 12288 to 16384 +0.3 with 8 row blocks, 0 with 32, -0.5 with 48, -0.7 with 64; 32768 +12.)
constexpr int kJoinedInPlace = 10240, kManyInPlace = 16384, kManyBlocks = 32;

// keys: the most that a row sees.  A part costs time in proportion to its keys and, where they are joined in place, to its being one more,
// so that the best number of parts grows with the root of the keys: sqrt(keys / 24) for plain scores.  (One token, 8 KV heads, int8, 8 / 16 / 32
// parts: 2048 rows 8.7 / 8.9 / 9.7 us, 8192 rows 13.1 / 11.3 / 12.3.)  The join kernel costs about the same for any number: three times as
// many keys under the root.  (One token, 64 heads, fp16, 4096 rows: 12 / 16 / 24 / 32 parts 11.7 / 11.5 / 10.6 / 10.5.)  Scores with forms take
// twice the time per key.  No more parts than leave every workgroup a compute unit (280 workgroups on 256 units 16.0 us, 252 13.7: 16 tokens over
// 4096 rows with forms, 14 / 7 heads, batch 2), or, where parts then still have 1024 keys (512 in 4 bits and blocks of 16 rows: one token over 32768
// rows, 8 KV heads, 32 / 64 parts 16.8 / 15.6 us; 64 tokens over 4096, blocks of 32, 4 / 8 parts 18.9 / 21.7), than fill the eight wavefronts that a
// unit holds (32 tokens over 8192 int8 rows, batch 4, 2 / 4 parts 37.6 / 32.5 us; 64 tokens over 4096 e4m3 rows, 32 heads, 4 / 8 parts
// 17.7 / 20.6).  Never fewer than 128 keys, and one part up to 384 keys (192 with forms) where a workgroup has at most 64 rows: nothing to
// join saves 0.7 to 1.7 us.  Parts are whole multiples of 128 keys, so that all wavefronts have as many steps.
Plan plan_of(const cf_cache_config &c, bool forms, int batch, int tokens, int keys, int cus, int limit)
{
    const auto &shapes = shapes_of(c, forms);
    const int live = tokens * (c.n_q_heads / c.n_kv_heads);
    Plan p;
    p.shape = shape_of(live);
    const Shape &shape = shapes[p.shape];
    p.blocks = block_rows(shapes, live) / shape.rows;
    const long long items = (long long)batch * c.n_kv_heads * p.blocks;
    const auto fill = [&](long long places) { return (int)std::max(places / items, 1ll); };
    const auto in_place = [&](int parts) {
        const long long values = (long long)parts * (live < shape.rows ? live : shape.rows) * c.head_dim;
        return values <= kJoinedInPlace || (values <= kManyInPlace && items >= kManyBlocks);
    };
    const int one = fill(cus), full = fill((long long)cus * 8 / shape.waves), most = (keys + 4 * kStep - 1) / (4 * kStep);
    // parts of as many times 128 keys
    const auto in_rounds = [&](double rounds) { return std::min((int)std::ceil(most / std::max(std::floor(rounds), 1.0)), one); };
    const double work = forms ? 2.0 * keys : keys;
    int few = in_rounds(most / std::sqrt(work / 24) + 0.5);
    if (!in_place(few)) few = in_rounds(most / std::sqrt(work / 8));
    const int long_parts = keys / (c.format == CF_CACHE_MXFP4 && shape.rows == 16 ? 512 : 1024);
    const int wanted = long_parts < few ? few : long_parts < full ? long_parts : full;
    p.splits = work <= 384 && shape.rows <= 64 ? 1 : std::min(wanted, most);
    if (p.splits > kMaxSplits) p.splits = kMaxSplits;
    if (limit > 0) p.splits = p.splits > limit ? limit : p.splits;
    if (p.splits < 1) p.splits = 1;
    p.in_place = in_place(p.splits);
    return p;
}

// Rows of partial results that no call of this configuration exceeds.  A call with more than one part has no more workgroups than there are
// places for them (plan_of), two to a compute unit up to 128 rows a workgroup, one with 256, and set_splits only takes some away.  And none
// has more rows than the largest batch with the most tokens (the rows of all row blocks grow with the tokens), nor more parts than 128 keys
// each leave.
size_t partial_rows(const cf_tree_config &t, int cus)
{
    const cf_cache_config &c = t.cache;
    const int live = t.max_tokens * (c.n_q_heads / c.n_kv_heads);
    size_t padded = 0;
    for (const bool forms : {false, true}) padded = std::max(padded, (size_t)block_rows(shapes_of(c, forms), live));
    const size_t parts = std::min((c.max_seq + 4 * kStep - 1) / (4 * kStep), kMaxSplits);
    return std::min(2 * (size_t)cus * 128, (size_t)c.max_batch * c.n_kv_heads * padded * parts);
}

}  // namespace

struct cf_tree_s {
    cf_tree_config cfg;
    int device = 0, cus = 0;
    int max_splits = 0;
    char *ws = nullptr;            // counters (zero between calls), then partial results
    size_t ws_rows = 0;            // rows of partial results that it holds
    uint32_t counters = 0;
};

extern "C" {

int cf_tree_create(const cf_tree_config *cfg, cf_tree *out)
{
    if (!cfg || !out) return CF_EINVAL;
    *out = nullptr;
    const int rc = check_config(cfg->cache);
    if (rc != CF_OK) return rc;
    if (cfg->max_tokens < 1 || cfg->max_tokens > kMaxTokens || cfg->window < 0 || !(cfg->score_cap >= 0.f) || !(cfg->score_cap <= 3.402823466e38f)) return CF_EINVAL;
    if (cfg->score_cap > 0.f && (cfg->score_cap < 0x1p-60f || cfg->score_cap > 0x1p60f)) return CF_EUNSUPPORTED;   // 2 / cap and cap log2 e in fp32
    int dev = 0, cus = 0;
    if (hipGetDevice(&dev) != hipSuccess ||
        hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cus < 1)
        return CF_EHIP;
    const size_t rows = partial_rows(*cfg, cus);
    const uint32_t counters = ((uint32_t)cus + 63) / 64 * 64;       // a call with more than one part has half as many row blocks as workgroups, at most
    cf_tree t = new (std::nothrow) cf_tree_s();
    if (!t) return CF_ENOMEM;
    t->cfg = *cfg;
    t->device = dev, t->cus = cus, t->ws_rows = rows, t->counters = counters;
    const size_t head = counters * sizeof(uint32_t);
    hipError_t e = hipMalloc(reinterpret_cast<void **>(&t->ws), head + rows * (cfg->cache.head_dim * sizeof(float) + sizeof(float2)));
    if (e == hipSuccess) e = hipMemset(t->ws, 0, head);
    if (e == hipSuccess) e = hipDeviceSynchronize();
    if (e != hipSuccess) {
        if (t->ws) (void)hipFree(t->ws);
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
    if (overlap(q, q_bytes, out, q_bytes) || in_cache(c, *cache, batch, out, q_bytes)) return CF_EINVAL;
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
    const bool forms = a.cap > 0.f || a.window > 0 || a.slopes;
    Plan p = plan_of(c, forms, batch, draft->tokens, keys, t->cus, t->max_splits);
    const Shape shape = shapes_of(c, forms)[p.shape];
    a.padded = p.blocks * shape.rows;
    const size_t rows = (size_t)batch * a.nkv * a.padded;
    if (rows * p.splits > t->ws_rows) p.splits = rows < t->ws_rows ? (int)(t->ws_rows / rows) : 1;
    a.splits = p.splits, a.blocks = p.blocks, a.units = batch * a.nkv * p.splits;
    const size_t sums = t->ws_rows * c.head_dim * sizeof(float);
    a.part = reinterpret_cast<float *>(t->ws + t->counters * sizeof(uint32_t));
    a.part_ml = (uint32_t)sums, a.part_bytes = (uint32_t)(sums + t->ws_rows * sizeof(float2));
    if (p.in_place && (uint32_t)batch * a.nkv * p.blocks <= t->counters) a.arrived = reinterpret_cast<uint32_t *>(t->ws);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    hipLaunchKernelGGL(pick(c.head_dim, c.format, p.shape, forms), dim3((a.units + 7) / 8 * 8 * p.blocks),
                       dim3(64 * shape.waves), 0, s, a);
    if (hipGetLastError() != hipSuccess) return CF_EHIP;
    if (p.splits > 1 && !a.arrived) {
        const int slots = NT / (c.head_dim / 8);
        int lanes = 1;
        while (lanes < p.splits && lanes < slots) lanes *= 2;
        hipLaunchKernelGGL((c.head_dim == 64 ? tree_join<64> : tree_join<128>), dim3((draft->tokens * a.group * lanes + slots - 1) / slots, batch * a.nkv), dim3(NT), 0, s, a,
                           lanes, c.format == CF_CACHE_INT8 ? cf::tree::kInt8Unit : 1.f);
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
    const int64_t row = row_bytes(c) + row_scale_bytes(c);
    const int64_t read = cfg->window > 0 && cfg->window < len ? cfg->window : len;      // cached rows that some token may see
    return (int64_t)batch * (2 * c.n_kv_heads * row * (read + tokens) + 4 * (int64_t)tokens * c.n_q_heads * c.head_dim);
}

}  // extern "C"
