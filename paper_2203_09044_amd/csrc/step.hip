// The server's update of the model with the averaged gradient: global gradient norm and AdamW over many tensors
// at once, with states in 32 bits or in 8.  Everything here streams: an element is read once, a few dozen
// operations are done on it, and it is written once.  The tensors are cut into pieces on the host; one table entry
// holds all a workgroup has to know of its piece (addresses, place in the state arrays, length, the tensor's factors).
#include "co3_dev.h"
#include "kernels.h"
#include "step.h"
#include "step_root.h"

#define ST_BLOCK 256
#define ST_NORM_BLOCK (CO3_WAVE * ST_NORM_WAVES)

// Addresses that come out of the table are global memory: said so, or every access would be a flat one.
#define ST_GLOBAL __attribute__((address_space(1)))

// Vectors of consecutive elements, aligned as a single element is: a tensor of a packed vector starts anywhere, and the vector
// memory unit takes any address of that alignment.
typedef float st_f32x4 __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned short st_u16x4 __attribute__((ext_vector_type(4), aligned(2)));
typedef unsigned short st_u16x8 __attribute__((ext_vector_type(8), aligned(2)));
typedef uint32_t st_u32x2 __attribute__((ext_vector_type(2), aligned(4)));

// Streaming (non-temporal) accesses: nothing here is touched twice by a kernel.  Against plain ones, us for the step of 100 M fp32
// elements and for that of 62 tensors of 11.2 M with the norm before it: both streaming 484 and 61.4, plain loads 528 and
// 69.4, plain stores 517 and 70.9.
template <bool NT, typename V> __device__ __forceinline__ V ld(ST_GLOBAL V *p)
{
    return NT ? __builtin_nontemporal_load(p) : *p;
}
template <typename V> __device__ __forceinline__ void st(ST_GLOBAL V *p, V x) { __builtin_nontemporal_store(x, p); }

// N consecutive elements of a type as floats, and one.
template <int T> struct Elems;
template <> struct Elems<CO3_F32> {
    typedef ST_GLOBAL float *ptr;
    static constexpr int WIDE = 4;
    template <int N, bool NT = true> static __device__ __forceinline__ void load(ptr p, float *x)
    {
#pragma unroll
        for (int k = 0; k < N; k += 4) {
            const st_f32x4 t = ld<NT>(reinterpret_cast<ST_GLOBAL st_f32x4 *>(p + k));
#pragma unroll
            for (int e = 0; e < 4; ++e) x[k + e] = t[e];
        }
    }
    template <int N> static __device__ __forceinline__ void store(ptr p, const float *x)
    {
#pragma unroll
        for (int k = 0; k < N; k += 4) {
            const st_f32x4 t = {x[k], x[k + 1], x[k + 2], x[k + 3]};
            st(reinterpret_cast<ST_GLOBAL st_f32x4 *>(p + k), t);
        }
    }
    static __device__ __forceinline__ float load1(ptr p) { return *p; }
    static __device__ __forceinline__ void store1(ptr p, float x) { *p = x; }
};
struct Bf16 {
    static __device__ __forceinline__ float up(unsigned short b) { return __uint_as_float((uint32_t)b << 16); }
    static __device__ __forceinline__ unsigned short down(float x) { return __builtin_bit_cast(unsigned short, (__bf16)x); }
};
struct Fp16 {
    static __device__ __forceinline__ float up(unsigned short b) { return (float)__builtin_bit_cast(_Float16, b); }
    static __device__ __forceinline__ unsigned short down(float x) { return __builtin_bit_cast(unsigned short, (_Float16)x); }
};
template <typename H> struct Elems16 {       // rounded to nearest, ties to even
    typedef ST_GLOBAL unsigned short *ptr;
    static constexpr int WIDE = 8;
    template <int N, bool NT = true> static __device__ __forceinline__ void load(ptr p, float *x)
    {
        static_assert(N == 4 || N == 8, "vectors of 8 or 16 bytes");
        if constexpr (N == 4) {
            const st_u16x4 t = ld<NT>(reinterpret_cast<ST_GLOBAL st_u16x4 *>(p));
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = H::up(t[e]);
        } else {
            const st_u16x8 t = ld<NT>(reinterpret_cast<ST_GLOBAL st_u16x8 *>(p));
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = H::up(t[e]);
        }
    }
    template <int N> static __device__ __forceinline__ void store(ptr p, const float *x)
    {
        if constexpr (N == 4) {
            st_u16x4 t;
#pragma unroll
            for (int e = 0; e < 4; ++e) t[e] = H::down(x[e]);
            st(reinterpret_cast<ST_GLOBAL st_u16x4 *>(p), t);
        } else {
            st_u16x8 t;
#pragma unroll
            for (int e = 0; e < 8; ++e) t[e] = H::down(x[e]);
            st(reinterpret_cast<ST_GLOBAL st_u16x8 *>(p), t);
        }
    }
    static __device__ __forceinline__ float load1(ptr p) { return H::up(*p); }
    static __device__ __forceinline__ void store1(ptr p, float x) { *p = H::down(x); }
};
template <> struct Elems<CO3_BF16> : Elems16<Bf16> {};
template <> struct Elems<CO3_F16> : Elems16<Fp16> {};

template <int T> __device__ __forceinline__ typename Elems<T>::ptr at(const void *p)
{
    return (typename Elems<T>::ptr)const_cast<void *>(p);
}
// N elements of which the first `here` exist; the others read 0 and are not written.
template <int T, int N, bool NT = true> __device__ __forceinline__ void load_some(typename Elems<T>::ptr p, int here, float *x)
{
    if (here >= N) Elems<T>::template load<N, NT>(p, x);
    else
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = e < here ? Elems<T>::load1(p + e) : 0.0f;
}
template <int T, int N> __device__ __forceinline__ void store_some(typename Elems<T>::ptr p, int here, const float *x)
{
    if (here >= N) Elems<T>::template store<N>(p, x);
    else
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (e < here) Elems<T>::store1(p + e, x[e]);
}

// ---- norm ---------------------------------------------------------------------------------------------------
// Sum over the workgroup in a fixed order, in every lane.
__device__ __forceinline__ double block_sum_f64(double s, double *red)
{
#pragma unroll
    for (int d = CO3_WAVE / 2; d >= 1; d >>= 1) s += __shfl_xor(s, d, CO3_WAVE);
    if ((threadIdx.x & (CO3_WAVE - 1)) == 0) red[threadIdx.x / CO3_WAVE] = s;
    __syncthreads();
    double t = 0.0;
    for (int w = 0; w < ST_NORM_WAVES; ++w) t += red[w];
    return t;
}

// What is made of the partial sums of a norm, by one workgroup: {norm, factor} at `out`, or the beginning of a step that the
// device counts (a captured step has no other way to).  The factor is negative where the norm is not finite.  What follows from the
// number of the step alone (two powers, quotients and a root in 64 bits) is made by a wavefront that has nothing else to do
// while the sums arrive.
struct StepNext {
    int64_t t;
    Co3StepVar var;
};
__device__ __forceinline__ void prepare_next(const Co3StepFinish &f, StepNext *next)      // before the sum's barrier
{
    if (!f.dev || threadIdx.x != CO3_WAVE) return;
    co3_adamw_args a = f.args;
    a.t = f.dev->t + 1;
    if (f.lr_dev) a.lr = (double)*f.lr_dev;
    next->t = a.t;
    next->var = co3_step_var(a);
}
__device__ __forceinline__ void finish_norm(double s, bool norm, const Co3StepFinish &f, const StepNext *next)     // one lane
{
    float factor = (float)f.args.grad_scale, total32 = 0.0f;
    if (norm) {
        const double total = f.args.grad_scale * __builtin_sqrt(s);
        const double c = f.args.max_norm / (total + 1e-6);
        total32 = (float)total;
        factor = s - s == 0.0 ? (float)(f.args.grad_scale * (c < 1.0 ? c : 1.0)) : -1.0f;
    }
    if (f.out) {
        f.out[0] = total32;
        f.out[1] = factor;
        return;
    }
    f.dev->norm = total32;
    f.dev->factor = factor;
    if (factor < 0.0f) {
        f.dev->skipped += 1;
        return;
    }
    f.dev->t = next->t;
    f.dev->var = next->var;
}

// partials[1 + workgroup] = sum of the squares of its pieces; a wavefront takes a piece, ROUNDS vectors of it in flight.  In 64 bits: the
// squares of 24-bit numbers are exact and none overflows, so the norm is right for any finite gradient; the sums are
// taken in a fixed order, so it is the same in every run.  Where something is to be made of the sums, the workgroup
// that is the last to have written its own does it: that saves a launch (65,536 elements: 5.5 us a call, with a second
// kernel 10.7); the ticket in front of the partial sums (zero between calls, so at the same place however many sums a table has: tables
// may take turns on a workspace) says which one it is.  Tickets are drawn one
// after another, some 8 ns each, so few large workgroups are better than many: one of 16 wavefronts to a compute unit reads 100 M
// bf16 elements in 33.2 us (6.0 TB/s, bound by the reading), 512 of them in 36.3, 2048 of four wavefronts in 52.3.
template <int G, bool NT>
__global__ __launch_bounds__(ST_NORM_BLOCK) void k_grad_sumsq(const Co3StepChunk *__restrict__ plan, int64_t chunks, double *partials,
                                                          Co3StepFinish f)
{
    constexpr int V = Elems<G>::WIDE, ROUNDS = 32 / V, STEP = CO3_WAVE * V;
    __shared__ double red[ST_NORM_WAVES];
    __shared__ uint32_t ticket;
    __shared__ StepNext next;
    const int lane = threadIdx.x & (CO3_WAVE - 1);
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    for (int64_t k = (int64_t)blockIdx.x * ST_NORM_WAVES + __builtin_amdgcn_readfirstlane((int)threadIdx.x / CO3_WAVE); k < chunks;
         k += (int64_t)gridDim.x * ST_NORM_WAVES) {
        const Co3StepChunk ch = plan[k];
        const auto g = at<G>(ch.grad);
        for (int b = 0; b < ch.count; b += STEP * ROUNDS) {
            float x[ROUNDS][V];
            const int i = b + lane * V;
            if (b + STEP * ROUNDS <= ch.count) {
#pragma unroll
                for (int r = 0; r < ROUNDS; ++r) Elems<G>::template load<V, NT>(g + i + r * STEP, x[r]);
            } else {
#pragma unroll
                for (int r = 0; r < ROUNDS; ++r) load_some<G, V, NT>(g + i + r * STEP, ch.count - (i + r * STEP), x[r]);
            }
#pragma unroll
            for (int r = 0; r < ROUNDS; ++r)
#pragma unroll
                for (int e = 0; e < V; ++e) s[e & 3] = __builtin_fma((double)x[r][e], (double)x[r][e], s[e & 3]);
        }
    }
    const double t = block_sum_f64((s[0] + s[1]) + (s[2] + s[3]), red);
    if (!f.out && !f.dev) {
        if (threadIdx.x == 0) {
            partials[1 + blockIdx.x] = t;
            if (blockIdx.x == 0) partials[0] = 0.0;      // no ticket here, and nothing to the sum
        }
        return;
    }
    if (threadIdx.x == 0) {
        // The sum is written through to where every compute unit sees it, and has arrived there before the ticket is drawn; a
        // release would write back the whole of the L2 first (2048 of them: 78 us).  The last ticket sets the counter back.
        __hip_atomic_store(partials + 1 + blockIdx.x, t, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        ticket = atomicInc(reinterpret_cast<uint32_t *>(partials), gridDim.x - 1);
    }
    __syncthreads();
    if (ticket != gridDim.x - 1) return;
    prepare_next(f, &next);
    double all = 0.0;
    for (uint32_t i = threadIdx.x; i < gridDim.x; i += ST_NORM_BLOCK)
        all += __hip_atomic_load(partials + 1 + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    all = block_sum_f64(all, red);
    if (threadIdx.x == 0) finish_norm(all, true, f, &next);
}

// The same from partial sums that are there already (several tables under one norm), or without a norm.
__global__ __launch_bounds__(ST_NORM_BLOCK) void k_step_begin(const double *__restrict__ partials, int64_t count, Co3StepFinish f)
{
    __shared__ double red[ST_NORM_WAVES];
    __shared__ StepNext next;
    prepare_next(f, &next);
    double s = 0.0;
    if (partials)
        for (int64_t i = threadIdx.x; i < count; i += ST_NORM_BLOCK) s += partials[i];
    s = block_sum_f64(s, red);
    if (threadIdx.x == 0) finish_norm(s, partials != nullptr, f, &next);
}

// ---- step ---------------------------------------------------------------------------------------------------
// One element, every operation rounded on its own (the build contracts nothing).
__device__ __forceinline__ void step_moments(const Co3StepFix &c, float factor, float g, float &m, float &v)
{
    g = g * factor;
    m = c.b1 * m + c.c1 * g;
    v = c.b2 * v + c.c2 * (g * g);
}
// The quotient by way of the reciprocal, which is one unit in the last place off at most: it goes into the weight alone,
// where a rounding of the step is far below one of the weight.  The divisor is no subnormal number (eps is not one).
__device__ __forceinline__ float step_weight(const Co3StepFix &c, float rbc2, float decay, float step, float w, float m, float root)
{
    const float u = m * __builtin_amdgcn_rcpf(root * rbc2 + c.eps);
    return w - (decay * w + step * u);
}

struct Co3StepNow {          // what a workgroup knows of its step
    float factor, rbc2, decay, step;
    uint32_t key;
};
__device__ __forceinline__ Co3StepNow step_now(const Co3StepChunk &ch, const Co3StepVar &host, float factor, const Co3StepDev *dev)
{
    const Co3StepVar var = dev ? dev->var : host;
    return {dev ? dev->factor : factor, var.rbc2, (var.lr * ch.lr_scale) * ch.weight_decay, var.step * ch.lr_scale, var.key};
}

// Bound by the memory: 28 bytes an element in fp32, 12 of them written.  Four elements to a lane, ST_GROUPS times, all loads in
// flight before the first is used: 100 M elements 484 us (5.8 TB/s; one group 513, four 490), 62 tensors of 11.2 M with
// their norm 61.4 us (71.5, 64.3).
#define ST_GROUPS 2
template <int P, int G, bool MASTER>
__global__ __launch_bounds__(ST_BLOCK) void k_adamw(const Co3StepChunk *__restrict__ plan, float *__restrict__ master_all,
                                                     float *__restrict__ m_all, float *__restrict__ v_all, Co3StepFix c,
                                                     Co3StepVar var, float factor, const Co3StepDev *__restrict__ dev)
{
    constexpr int V = 4;
    const Co3StepChunk ch = plan[blockIdx.x];
    const auto p = at<P>(ch.param);
    const auto g = at<G>(ch.grad);
    const auto w32 = at<CO3_F32>(MASTER ? master_all + ch.state : nullptr);
    const auto m = at<CO3_F32>(m_all + ch.state), v = at<CO3_F32>(v_all + ch.state);
    float gx[ST_GROUPS][V], mx[ST_GROUPS][V], vx[ST_GROUPS][V], wx[ST_GROUPS][V];
    const int i = threadIdx.x * V;
    auto step = [&](const Co3StepNow &now, int k) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            step_moments(c, now.factor, gx[k][e], mx[k][e], vx[k][e]);
            wx[k][e] = step_weight(c, now.rbc2, now.decay, now.step, wx[k][e], mx[k][e], __builtin_sqrtf(vx[k][e]));
        }
    };
    if (ch.count == ST_GROUPS * ST_BLOCK * V) {
#pragma unroll
        for (int k = 0; k < ST_GROUPS; ++k) {
            const int j = i + k * ST_BLOCK * V;
            Elems<G>::template load<V>(g + j, gx[k]);
            Elems<CO3_F32>::load<V>(m + j, mx[k]);
            Elems<CO3_F32>::load<V>(v + j, vx[k]);
            if (MASTER) Elems<CO3_F32>::load<V>(w32 + j, wx[k]);
            else Elems<P>::template load<V>(p + j, wx[k]);
        }
        const Co3StepNow now = step_now(ch, var, factor, dev);
        if (now.factor < 0.0f) return;
#pragma unroll
        for (int k = 0; k < ST_GROUPS; ++k) {
            const int j = i + k * ST_BLOCK * V;
            step(now, k);
            Elems<CO3_F32>::store<V>(m + j, mx[k]);
            Elems<CO3_F32>::store<V>(v + j, vx[k]);
            if (MASTER) Elems<CO3_F32>::store<V>(w32 + j, wx[k]);
            Elems<P>::template store<V>(p + j, wx[k]);
        }
    } else {
        const Co3StepNow now = step_now(ch, var, factor, dev);
        if (now.factor < 0.0f) return;
        for (int j = i; j < ch.count; j += ST_BLOCK * V) {
            const int here = ch.count - j;
            load_some<G, V>(g + j, here, gx[0]);
            load_some<CO3_F32, V>(m + j, here, mx[0]);
            load_some<CO3_F32, V>(v + j, here, vx[0]);
            if (MASTER) load_some<CO3_F32, V>(w32 + j, here, wx[0]);
            else load_some<P, V>(p + j, here, wx[0]);
            step(now, 0);
            store_some<CO3_F32, V>(m + j, here, mx[0]);
            store_some<CO3_F32, V>(v + j, here, vx[0]);
            if (MASTER) store_some<CO3_F32, V>(w32 + j, here, wx[0]);
            store_some<P, V>(p + j, here, wx[0]);
        }
    }
}

// ---- step with 8-bit states ---------------------------------------------------------------------------------
// The scale under which the largest magnitude of a block stays within 448 = 1.75 * 2^8 whichever way it is rounded.
__device__ __forceinline__ uint32_t e4m3_scale(uint32_t max_bits)
{
    const int s = (int)((max_bits + 0x200000u) >> 23) - 8;
    return s > 0 ? (uint32_t)s : 0u;
}
// The largest over the L lanes that share a block, in each of them: rotations within rows of 16 lanes, then across.
template <int L> __device__ __forceinline__ uint32_t block_max_u32(uint32_t v)
{
    if (L == CO3_WAVE) return wave_max_u32(v);
    auto step = [](uint32_t x, uint32_t y) { return x > y ? x : y; };
    v = step(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x121, 0xf, 0xf, false));   // row_ror:1
    v = step(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x122, 0xf, 0xf, false));   // row_ror:2
    v = step(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x124, 0xf, 0xf, false));   // row_ror:4
    v = step(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xf, 0xf, false));   // row_ror:8
    return step(v, (uint32_t)__builtin_amdgcn_ds_swizzle((int)v, 0x401f));                   // lane ^ 16
}

#define ST8_WAVE 512         // elements of a wavefront, two blocks

// With 16-bit weights an element is 10 bytes, and the arithmetic has to keep up with 600 G elements a second: some 55 issue slots
// of a SIMD each.  So codes are converted by the instructions for it, scale, random rounding, sign and place in the word included (20
// slots an element less than by shifts), the root is the short one (6 less), the quotient goes through a reciprocal (9 less),
// and the masks of a ragged end are in a second copy of the code.  100 M elements in bf16: 161 us (6.2 TB/s), with shifts,
// compiler's root and quotient 224.
template <int P, int G, bool MASTER> struct Step8 {
    // Elements to a lane in one place.  16-bit arrays alone: 8, so that the loads are of 16 bytes, and half a wavefront has a block.
    // With 32-bit ones among them 4, a wavefront to a block and two blocks after each other: 8 would take two 16-byte accesses
    // 32 bytes apart from lane to lane, each of which leaves half of every line to the other (62 tensors with masters:
    // 38.7 us against 31.3).
    static constexpr int V = P != CO3_F32 && G != CO3_F32 && !MASTER ? 8 : 4, GROUPS = 8 / V, LANES = CO3_STEP_BLOCK / V;
    typename Elems<P>::ptr p;
    typename Elems<G>::ptr g;
    typename Elems<CO3_F32>::ptr w32;
    ST_GLOBAL uint8_t *m, *r, *ms, *rs;
    uint32_t key;
    int count;
    Co3StepNow now;
    Co3StepFix c;

    // Elements b .. b + 511 of the piece, by one wavefront.  FULL: all of them exist.
    template <bool FULL> __device__ __forceinline__ void run(int b) const
    {
        typedef float f32x2 __attribute__((ext_vector_type(2)));
        const int lane = threadIdx.x & (CO3_WAVE - 1);
        float gx[8], wx[8], mx[8], vx[8], rx[8];
        uint32_t mc[2], rc[2];
        float mscale[GROUPS], rscale[GROUPS];
        int here[GROUPS];
#pragma unroll
        for (int k = 0; k < GROUPS; ++k) {
            const int i = b + k * CO3_STEP_BLOCK + lane * V;
            here[k] = FULL ? V : count - i;
            const bool block = FULL || (i & -CO3_STEP_BLOCK) < count;        // the state arrays go on to the end of a block
            if (V == 8) {
                const st_u32x2 z = {0, 0}, a = block ? ld<true>((ST_GLOBAL st_u32x2 *)(m + i)) : z,
                               q = block ? ld<true>((ST_GLOBAL st_u32x2 *)(r + i)) : z;
                mc[0] = a[0]; mc[1] = a[1]; rc[0] = q[0]; rc[1] = q[1];
            } else {
                mc[k] = block ? ld<true>((ST_GLOBAL uint32_t *)(m + i)) : 0u;
                rc[k] = block ? ld<true>((ST_GLOBAL uint32_t *)(r + i)) : 0u;
            }
            mscale[k] = __uint_as_float(block ? (uint32_t)ms[i / CO3_STEP_BLOCK] << 23 : 0u);
            rscale[k] = __uint_as_float(block ? (uint32_t)rs[i / CO3_STEP_BLOCK] << 23 : 0u);
            if (FULL) {
                Elems<G>::template load<V>(g + i, gx + k * V);
                if (MASTER) Elems<CO3_F32>::load<V>(w32 + i, wx + k * V);
                else Elems<P>::template load<V>(p + i, wx + k * V);
            } else {
                load_some<G, V>(g + i, here[k], gx + k * V);
                if (MASTER) load_some<CO3_F32, V>(w32 + i, here[k], wx + k * V);
                else load_some<P, V>(p + i, here[k], wx + k * V);
            }
        }
        float vtop = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            // the conversion takes a code's scale from the exponent field of its operand: the bits of an e8m0 number in their place
            const float sm = mscale[e / V], sr = rscale[e / V];
            const f32x2 a = e & 2 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(mc[e / 4], sm, true) : __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(mc[e / 4], sm, false);
            const f32x2 q = e & 2 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(rc[e / 4], sr, true) : __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(rc[e / 4], sr, false);
#pragma unroll
            for (int d = 0; d < 2; ++d) {
                mx[e + d] = a[d];
                vx[e + d] = q[d] * q[d];
                step_moments(c, now.factor, gx[e + d], mx[e + d], vx[e + d]);
                if (!FULL && (e + d) % V >= here[e / V]) mx[e + d] = vx[e + d] = 0.0f;
                vtop = fmaxf(vtop, vx[e + d]);
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) rx[e] = root_below_2_40(vx[e]);
        if (__any(vtop >= 0x1p40f)) {             // gradients of a million and more, or not finite
#pragma unroll
            for (int e = 0; e < 8; ++e) rx[e] = __builtin_sqrtf(vx[e]);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) wx[e] = step_weight(c, now.rbc2, now.decay, now.step, wx[e], mx[e], rx[e]);
#pragma unroll
        for (int k = 0; k < GROUPS; ++k) {
            const int i = b + k * CO3_STEP_BLOCK + lane * V;
            if (FULL) {
                if (MASTER) Elems<CO3_F32>::store<V>(w32 + i, wx + k * V);
                Elems<P>::template store<V>(p + i, wx + k * V);
            } else {
                if (MASTER) store_some<CO3_F32, V>(w32 + i, here[k], wx + k * V);
                store_some<P, V>(p + i, here[k], wx + k * V);
            }
        }
#pragma unroll
        for (int k = 0; k < GROUPS; ++k) {
            const int i = b + k * CO3_STEP_BLOCK + lane * V;
            float mtop = 0.0f, rtop = 0.0f;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                mtop = fmaxf(mtop, fabsf(mx[k * V + e]));
                rtop = fmaxf(rtop, rx[k * V + e]);
            }
            const uint32_t s1 = e4m3_scale(block_max_u32<LANES>(__float_as_uint(mtop)));
            const uint32_t s2 = e4m3_scale(block_max_u32<LANES>(__float_as_uint(rtop)));
            const float sm = __uint_as_float(s1 << 23), sr = __uint_as_float(s2 << 23);
            const uint32_t h0 = (uint32_t)(i >> 1) * CO3_STEP_H0 + key;
            uint32_t mw[V / 4], rw[V / 4];
#pragma unroll
            for (int q = 0; q < V / 4; ++q) {
                // The conversion adds the upper 20 bits of its random operand to the 20 that it cuts off: 16 of the hash and half of the
                // next place.  The halves of one hash serve two elements, their complements r.
                const uint32_t ha = co3_step_fin(h0 + (2 * q) * CO3_STEP_H0), hb = co3_step_fin(h0 + (2 * q + 1) * CO3_STEP_H0);
                const float *x = mx + k * V + 4 * q, *y = rx + k * V + 4 * q;
                const uint32_t h[4] = {ha << 16, ha & 0xffff0000u, hb << 16, hb & 0xffff0000u};
                const uint32_t n[4] = {~ha << 16, ~ha & 0xffff0000u, ~hb << 16, ~hb & 0xffff0000u};
                uint32_t a = 0, d = 0;
                a = __builtin_amdgcn_cvt_scalef32_sr_fp8_f32(a, x[0], h[0] | 0x8000u, sm, 0);
                a = __builtin_amdgcn_cvt_scalef32_sr_fp8_f32(a, x[1], h[1] | 0x8000u, sm, 1);
                a = __builtin_amdgcn_cvt_scalef32_sr_fp8_f32(a, x[2], h[2] | 0x8000u, sm, 2);
                a = __builtin_amdgcn_cvt_scalef32_sr_fp8_f32(a, x[3], h[3] | 0x8000u, sm, 3);
                d = __builtin_amdgcn_cvt_scalef32_sr_fp8_f32(d, y[0], n[0] | 0x8000u, sr, 0);
                d = __builtin_amdgcn_cvt_scalef32_sr_fp8_f32(d, y[1], n[1] | 0x8000u, sr, 1);
                d = __builtin_amdgcn_cvt_scalef32_sr_fp8_f32(d, y[2], n[2] | 0x8000u, sr, 2);
                d = __builtin_amdgcn_cvt_scalef32_sr_fp8_f32(d, y[3], n[3] | 0x8000u, sr, 3);
                if ((d - 0x01010101u) & ~d & 0x80808080u) {       // some code is 0: a divisor does not vanish
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (!(d >> (8 * e) & 0xffu) && y[e] != 0.0f) d |= 1u << (8 * e);
                }
                if (!FULL && here[k] < 4 * q + 4) {               // behind the tensor's last element: as it was
                    const uint32_t keep = here[k] <= 4 * q ? 0xffffffffu : 0xffffffffu << (8 * (here[k] - 4 * q));
                    a = (a & ~keep) | (mc[V == 8 ? q : k] & keep);
                    d = (d & ~keep) | (rc[V == 8 ? q : k] & keep);
                }
                mw[q] = a;
                rw[q] = d;
            }
            if (FULL || (i & -CO3_STEP_BLOCK) < count) {
                if constexpr (V == 8) {
                    const st_u32x2 a = {mw[0], mw[1]}, d = {rw[0], rw[1]};
                    st((ST_GLOBAL st_u32x2 *)(m + i), a);
                    st((ST_GLOBAL st_u32x2 *)(r + i), d);
                } else {
                    st((ST_GLOBAL uint32_t *)(m + i), mw[0]);
                    st((ST_GLOBAL uint32_t *)(r + i), rw[0]);
                }
                if (lane % LANES == 0) {
                    ms[i / CO3_STEP_BLOCK] = (uint8_t)s1;
                    rs[i / CO3_STEP_BLOCK] = (uint8_t)s2;
                }
            }
        }
    }
};

template <int P, int G, bool MASTER>
__global__ __launch_bounds__(ST_BLOCK) void k_adamw8(const Co3StepChunk *__restrict__ plan, float *__restrict__ master_all,
                                                      uint8_t *__restrict__ m_all, uint8_t *__restrict__ ms_all,
                                                      uint8_t *__restrict__ r_all, uint8_t *__restrict__ rs_all, Co3StepFix c,
                                                      Co3StepVar var, float factor, const Co3StepDev *__restrict__ dev)
{
    const Co3StepChunk ch = plan[blockIdx.x];
    const Co3StepNow now = step_now(ch, var, factor, dev);
    if (now.factor < 0.0f) return;
    typedef ST_GLOBAL uint8_t *bytes;
    const Step8<P, G, MASTER> s{at<P>(ch.param), at<G>(ch.grad), at<CO3_F32>(MASTER ? master_all + ch.state : nullptr),
                                (bytes)(m_all + ch.state), (bytes)(r_all + ch.state), (bytes)(ms_all + ch.state / CO3_STEP_BLOCK),
                                (bytes)(rs_all + ch.state / CO3_STEP_BLOCK),
                                (uint32_t)(ch.state / 2) * CO3_STEP_H0 + now.key, ch.count, now, c};
    const int b = __builtin_amdgcn_readfirstlane((int)threadIdx.x / CO3_WAVE) * ST8_WAVE;
    if (b + ST8_WAVE <= ch.count) s.template run<true>(b);
    else if (b < ch.count) s.template run<false>(b);
}

// ---- launches -------------------------------------------------------------------------------------------------
// A gradient of up to half of the memory-side cache (256 MB) is left there for the step that follows a norm: plain loads (62 tensors,
// 45 MB: norm and step 61.5 us, with streaming loads 66.1).  A longer one streams (100 M bf16: 34.3 us, with plain ones 36.4).
#define ST_NORM_CACHED ((int64_t)128 << 20)

namespace {
template <int G>
void launch_sumsq(const co3_step_layout *L, const void *plan, double *partials, const Co3StepFinish &f, hipStream_t st)
{
    const dim3 grid((uint32_t)L->partials - 1), block(ST_NORM_BLOCK);
    const auto *pl = static_cast<const Co3StepChunk *>(plan);
    if (L->elems > ST_NORM_CACHED / (G == CO3_F32 ? 4 : 2)) k_grad_sumsq<G, true><<<grid, block, 0, st>>>(pl, L->chunks, partials, f);
    else k_grad_sumsq<G, false><<<grid, block, 0, st>>>(pl, L->chunks, partials, f);
}
}  // namespace

hipError_t co3_launch_grad_sumsq(const co3_step_layout *L, const void *plan, double *partials, const Co3StepFinish &f, hipStream_t st)
{
    Co3LaunchTimer timer(CO3_K_GRAD_SUMSQ, st);
    switch (L->grad_type) {
    case CO3_F32: launch_sumsq<CO3_F32>(L, plan, partials, f, st); break;
    case CO3_BF16: launch_sumsq<CO3_BF16>(L, plan, partials, f, st); break;
    default: launch_sumsq<CO3_F16>(L, plan, partials, f, st); break;
    }
    return hipGetLastError();
}

hipError_t co3_launch_step_begin(const double *partials, int64_t count, const Co3StepFinish &f, hipStream_t st)
{
    Co3LaunchTimer timer(CO3_K_STEP_BEGIN, st);
    k_step_begin<<<1, ST_NORM_BLOCK, 0, st>>>(partials, count, f);
    return hipGetLastError();
}

namespace {
template <int P, int G, bool MASTER>
void launch_step(const Co3StepLaunch &s, hipStream_t st)
{
    const dim3 grid((uint32_t)s.layout->chunks), block(ST_BLOCK);
    const auto *pl = static_cast<const Co3StepChunk *>(s.plan);
    const auto *dev = static_cast<const Co3StepDev *>(s.state);
    if (s.layout->state_bits == 32)
        k_adamw<P, G, MASTER><<<grid, block, 0, st>>>(pl, s.master, static_cast<float *>(s.m), static_cast<float *>(s.v), s.fix,
                                                       s.var, s.factor, dev);
    else
        k_adamw8<P, G, MASTER><<<grid, block, 0, st>>>(pl, s.master, static_cast<uint8_t *>(s.m), s.m_scale,
                                                        static_cast<uint8_t *>(s.v), s.v_scale, s.fix, s.var, s.factor, dev);
}
template <int P, bool MASTER>
void launch_of_grad(const Co3StepLaunch &s, hipStream_t st)
{
    switch (s.layout->grad_type) {
    case CO3_F32: launch_step<P, CO3_F32, MASTER>(s, st); break;
    case CO3_BF16: launch_step<P, CO3_BF16, MASTER>(s, st); break;
    default: launch_step<P, CO3_F16, MASTER>(s, st); break;
    }
}
}  // namespace

hipError_t co3_launch_adamw(const Co3StepLaunch &s, hipStream_t st)
{
    if (s.layout->chunks == 0) return hipSuccess;
    Co3LaunchTimer timer(s.layout->state_bits == 32 ? CO3_K_ADAMW : CO3_K_ADAMW8, st);
    switch (s.layout->param_type) {
    case CO3_F32: launch_of_grad<CO3_F32, false>(s, st); break;
    case CO3_BF16: s.master ? launch_of_grad<CO3_BF16, true>(s, st) : launch_of_grad<CO3_BF16, false>(s, st); break;
    default: s.master ? launch_of_grad<CO3_F16, true>(s, st) : launch_of_grad<CO3_F16, false>(s, st); break;
    }
    return hipGetLastError();
}
