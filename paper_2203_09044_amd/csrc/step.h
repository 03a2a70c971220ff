// What the host and the kernels of the server's update share: the table of chunks, the scalars of a step.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/co3.h"

// A norm: wavefronts of a workgroup, and the most workgroups (one to a compute unit).
#define ST_NORM_WAVES 16
#define ST_NORM_GROUPS_MAX 256

// One piece of a tensor, at most co3_step_layout.chunk elements: what a workgroup has to know, in one entry.
struct Co3StepChunk {
    void *param;            // first element of the piece
    const void *grad;
    int64_t state;          // its place in the state arrays
    int32_t count;
    float lr_scale, weight_decay;
    int32_t reserved;
};
static_assert(sizeof(Co3StepChunk) == CO3_STEP_CHUNK_BYTES, "entry of the plan");

struct Co3StepFix {         // scalars that do not change from step to step
    float b1, c1, b2, c2, eps;
};
struct Co3StepVar {         // scalars of step t
    float lr, step, rbc2;   // learning rate, learning rate / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
    uint32_t key;           // of the rounding of the 8-bit states
};
// co3_step_state as the kernels see it
struct Co3StepDev {
    int64_t t, skipped;
    float norm, factor;
    Co3StepVar var;
};
static_assert(sizeof(Co3StepDev) <= sizeof(co3_step_state), "state of a step");

// Random bits are a hash of (seed, step, place): multiplications by odd constants (the fractions of the golden ratio and
// of the square roots of 2 and 3) and xors with the upper bits, two rounds of them.
#define CO3_STEP_H0 0x9E3779B9u
__host__ __device__ static inline uint32_t co3_step_fin(uint32_t x)
{
    x ^= x >> 15;
    x *= 0x6A09E667u;
    x ^= x >> 13;
    x *= 0xBB67AE85u;
    return x ^ (x >> 16);
}
__host__ __device__ static inline uint32_t co3_step_key(uint64_t seed, int64_t t)
{
    uint32_t k = co3_step_fin((uint32_t)t * CO3_STEP_H0 + 0x3C6EF372u);
    k = co3_step_fin((uint32_t)(seed >> 32) * CO3_STEP_H0 + k);
    return co3_step_fin((uint32_t)seed * CO3_STEP_H0 + k);
}
__host__ __device__ static inline double co3_step_pow(double b, int64_t t)
{
    double r = 1.0;
    for (; t > 0; t >>= 1) {
        if (t & 1) r *= b;
        b *= b;
    }
    return r;
}
__host__ __device__ static inline Co3StepVar co3_step_var(const co3_adamw_args &a)
{
    Co3StepVar v;
    v.lr = (float)a.lr;
    v.step = (float)(a.lr / (1.0 - co3_step_pow(a.beta1, a.t)));
    v.rbc2 = (float)(1.0 / __builtin_sqrt(1.0 - co3_step_pow(a.beta2, a.t)));
    v.key = co3_step_key(a.seed, a.t);
    return v;
}

// What is to be made of the partial sums of a norm: {norm, factor} at out, the beginning of a step at dev, or nothing.
struct Co3StepFinish {
    float *out;
    Co3StepDev *dev;
    const float *lr_dev;
    co3_adamw_args args;
};

struct Co3StepLaunch {
    const co3_step_layout *layout;
    const void *plan;
    float *master;
    void *m, *v;            // 32-bit moments, or 8-bit elements with their scales
    uint8_t *m_scale, *v_scale;
    Co3StepFix fix;
    Co3StepVar var;
    float factor;
    const void *state;      // co3_step_state, or NULL: var and factor count
};

hipError_t co3_launch_grad_sumsq(const co3_step_layout *L, const void *plan, double *partials, const Co3StepFinish &f, hipStream_t st);
hipError_t co3_launch_step_begin(const double *partials, int64_t count, const Co3StepFinish &f, hipStream_t st);
hipError_t co3_launch_adamw(const Co3StepLaunch &s, hipStream_t st);
