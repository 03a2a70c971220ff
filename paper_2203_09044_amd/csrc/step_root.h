// The square root of the 8-bit step.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

// Correctly rounded square root of 0 <= v < 2^40 (the tests compare it with the root in 64 bits for every such number): an estimate by
// the reciprocal root, off by a few units, and one correction by the exactly known rest v - s^2.  The scaling keeps the rest of
// a small v above the smallest number; the summand gives 0 a finite reciprocal and changes nothing else.  (The
// compiler's root is right everywhere and takes twice the operations.)
__device__ __forceinline__ float root_below_2_40(float v)
{
    const float x = v * 0x1p80f, y = __builtin_amdgcn_rsqf(x + 0x1p-120f), s = x * y;
    return __builtin_fmaf(__builtin_fmaf(-s, s, x), 0.5f * y, s) * 0x1p-40f;
}
