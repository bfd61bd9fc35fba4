// A double-precision exponential of non-positive arguments for kernels that need one per element.
#pragma once
#include <cuda_runtime.h>

namespace accerl {

// exp(x) for x <= 0 by table and a short polynomial (Tang, "Table-driven implementation of the exponential
// function", 1989): x = (64 m + j) ln2 / 64 + r, |r| <= ln2 / 128, exp(x) = 2^m 2^(j/64) (1 + r + ... + r^5 / 120);
// the truncation is below 3e-17, the result within about one ulp.  `table` holds 2^(j/64).  It has half the
// instructions of exp(), of which the rows kernel needs two per action (16 x 8192 rollouts of 18 actions,
// V-trace and both launches of the KL, rows copied element by element as they were then: 27 us with exp(), 24.6 with this).
__device__ __forceinline__ double exp_nonpositive(double x, const double *table)
{
    const double shift = 6755399441055744.0;  // 1.5 * 2^52: adding it rounds to an integer
    const double t = fma(x, 92.332482616893656, shift), nf = t - shift;
    const int n = __double2loint(t);
    const double r = fma(nf, -3.623510646634843e-19, fma(nf, -0.010830424696249145, x));
    const double p = fma(r * r, fma(r, fma(r, fma(r, 1.0 / 120.0, 1.0 / 24.0), 1.0 / 6.0), 0.5), r);
    const double v = fma(table[n & 63], p, table[n & 63]);
    const double y = __hiloint2double(__double2hiint(v) + ((n >> 6) << 20), __double2loint(v));
    // What underflows is nothing beside the row's largest term; the last case is a NaN.
    return x >= -708.0 ? y : x < 0.0 ? 0.0 : x;
}

// Fills the 64-entry table of exp_nonpositive (shared memory); a barrier has to follow.
__device__ __forceinline__ void fill_exp_table(double *table)
{
    if (threadIdx.x < 64) table[threadIdx.x] = exp2((double)threadIdx.x * (1.0 / 64.0));
}

}  // namespace accerl
