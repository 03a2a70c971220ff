// The short square root of the 8-bit step, number by number against the root in 64 bits rounded once (which is the correctly
// rounded one: 53 bits are more than twice 24 and two).
#include "../../paper_2203_09044_amd/csrc/step_root.h"

// out[0]: how many of the numbers with the bits first .. first + count - 1 have another root; out[1]: the lowest of them
__global__ void k_root_check(uint32_t first, uint32_t count, uint32_t *out)
{
    for (uint64_t i = (uint64_t)blockIdx.x * blockDim.x + threadIdx.x; i < count; i += (uint64_t)gridDim.x * blockDim.x) {
        const uint32_t bits = first + (uint32_t)i;
        const float v = __uint_as_float(bits);
        if (__float_as_uint(root_below_2_40(v)) != __float_as_uint((float)__builtin_sqrt((double)v))) {
            atomicAdd(out, 1u);
            atomicMin(out + 1, bits);
        }
    }
}

extern "C" int32_t root_check(uint32_t first, uint32_t count, uint32_t *out, void *stream)
{
    if (!out || (uint64_t)first + count > (uint64_t)1 << 32) return -1;
    k_root_check<<<2048, 256, 0, static_cast<hipStream_t>(stream)>>>(first, count, out);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}
