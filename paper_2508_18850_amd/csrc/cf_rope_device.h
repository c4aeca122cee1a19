// RoPE angle arithmetic shared by the decode kernels.
#ifndef CF_ROPE_DEVICE_H
#define CF_ROPE_DEVICE_H

#include <hip/hip_runtime.h>

namespace cf {

// Frequency of RoPE pair i: base^(-2i/head_dim), from log2(base), in fp64.
__device__ __forceinline__ double rope_inv_freq(int i, int head_dim, double log2_base)
{
    return exp2(-(2.0 * (double)i / (double)head_dim) * log2_base);
}

// cos and sin of pos * inv_freq, angle and range reduction in fp64.
__device__ __forceinline__ void rope_cos_sin(int pos, double inv_freq, float &cos_out, float &sin_out)
{
    const double ang = (double)pos * inv_freq;
    const double k = rint(ang * 0.63661977236758134308);              // 2/pi
    double r = fma(-k, 1.57079632679489655800e+00, ang);              // pi/2, high part
    r = fma(-k, 6.12323399573676603587e-17, r);                       // pi/2, low part
    const double r2 = r * r;                                          // |r| <= pi/4: Taylor series
    double s = -1.0 / 1307674368000.0;
    s = fma(s, r2, 1.0 / 6227020800.0);
    s = fma(s, r2, -1.0 / 39916800.0);
    s = fma(s, r2, 1.0 / 362880.0);
    s = fma(s, r2, -1.0 / 5040.0);
    s = fma(s, r2, 1.0 / 120.0);
    s = fma(s, r2, -1.0 / 6.0);
    s = fma(s * r2, r, r);
    double c = 1.0 / 20922789888000.0;
    c = fma(c, r2, -1.0 / 87178291200.0);
    c = fma(c, r2, 1.0 / 479001600.0);
    c = fma(c, r2, -1.0 / 3628800.0);
    c = fma(c, r2, 1.0 / 40320.0);
    c = fma(c, r2, -1.0 / 720.0);
    c = fma(c, r2, 1.0 / 24.0);
    c = fma(c, r2, -0.5);
    c = fma(c, r2, 1.0);
    const int q = (int)((long long)k & 3);
    const double sv = (q == 0) ? s : (q == 1) ? c : (q == 2) ? -s : -c;
    const double cv = (q == 0) ? c : (q == 1) ? -s : (q == 2) ? -c : s;
    cos_out = (float)cv;
    sin_out = (float)sv;
}

// cos and sin of the fp64 product pos * inv_freq, errors below 2^-51 for that angle (the product's own rounding comes on top, half a step:
// 2^-39 where it is 2^14 to 2^15): the angle less the nearest multiple of pi / 2 (taken off in two parts), the Taylor series of both up to a remainder
// of 2^-54 at pi / 4, and the quadrant.
__device__ __forceinline__ void rope_cos_sin64(double pos, double inv_freq, double &cos_out, double &sin_out)
{
    const double ang = pos * inv_freq;
    const double k = rint(ang * 0.63661977236758134308);              // 2/pi
    const double r = fma(-k, 6.12323399573676603587e-17, fma(-k, 1.57079632679489655800e+00, ang)), r2 = r * r;
    double s = 0.0, c = 0.0;
#pragma unroll
    for (int n = 16; n >= 2; n -= 2) {                                // s = 1 - r2 / 2 3 (1 - r2 / 4 5 (...)), c = 1 - r2 / 1 2 (...)
        s = fma(-(1.0 / (n * (n + 1))) * r2, s, -(1.0 / (n * (n + 1))) * r2);
        c = fma(-(1.0 / (n * (n - 1))) * r2, c, -(1.0 / (n * (n - 1))) * r2);
    }
    const double sr = fma(s, r, r), cr = 1.0 + c;
    const int q = (int)((long long)k & 3);
    const double sv = q & 1 ? cr : sr, cv = q & 1 ? sr : cr;
    sin_out = q & 2 ? -sv : sv;
    cos_out = (q + 1) & 2 ? -cv : cv;
}

}  // namespace cf
#endif
