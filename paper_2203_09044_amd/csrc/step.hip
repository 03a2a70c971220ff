// The server's update of the model with the averaged gradient: global gradient norm and AdamW over many tensors
// at once, with states in 32 bits or in 8.  Everything here streams: an element is read once, a few dozen
// operations are done on it, and it is written once.  The tensors are cut into chunks on the host; one table entry
// holds all a workgroup has to know of its chunk (addresses, place in the state arrays, length, the tensor's factors).
#include "co3_dev.h"
#include "kernels.h"
#include "step.h"

#define ST_BLOCK 256
#define ST_VEC 4
#define ST_TILE (ST_BLOCK * ST_VEC)

// Addresses that come out of the table are global memory: said so, or every access would be a flat one.
#define ST_GLOBAL __attribute__((address_space(1)))

typedef float st_f32x4 __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned short st_u16x4 __attribute__((ext_vector_type(4), aligned(2)));

// Four consecutive elements of a type, aligned as its single elements are (a tensor of a packed vector starts
// anywhere; the vector memory unit takes any address of that alignment), and one.
template <int T> struct Elems;
template <> struct Elems<CO3_F32> {
    typedef ST_GLOBAL float *ptr;
    static __device__ __forceinline__ void load4(ptr p, float x[4])
    {
        const st_f32x4 t = *reinterpret_cast<ST_GLOBAL st_f32x4 *>(p);
        x[0] = t.x; x[1] = t.y; x[2] = t.z; x[3] = t.w;
    }
    static __device__ __forceinline__ void store4(ptr p, const float x[4])
    {
        const st_f32x4 t = {x[0], x[1], x[2], x[3]};
        *reinterpret_cast<ST_GLOBAL st_f32x4 *>(p) = t;
    }
    static __device__ __forceinline__ float load1(ptr p) { return *p; }
    static __device__ __forceinline__ void store1(ptr p, float x) { *p = x; }
};
template <> struct Elems<CO3_BF16> {
    typedef ST_GLOBAL unsigned short *ptr;
    static __device__ __forceinline__ float up(unsigned short b) { return __uint_as_float((uint32_t)b << 16); }
    static __device__ __forceinline__ unsigned short down(float x) { return __builtin_bit_cast(unsigned short, (__bf16)x); }   // ties to even
    static __device__ __forceinline__ void load4(ptr p, float x[4])
    {
        const st_u16x4 t = *reinterpret_cast<ST_GLOBAL st_u16x4 *>(p);
        x[0] = up(t.x); x[1] = up(t.y); x[2] = up(t.z); x[3] = up(t.w);
    }
    static __device__ __forceinline__ void store4(ptr p, const float x[4])
    {
        const st_u16x4 t = {down(x[0]), down(x[1]), down(x[2]), down(x[3])};
        *reinterpret_cast<ST_GLOBAL st_u16x4 *>(p) = t;
    }
    static __device__ __forceinline__ float load1(ptr p) { return up(*p); }
    static __device__ __forceinline__ void store1(ptr p, float x) { *p = down(x); }
};
template <> struct Elems<CO3_F16> {
    typedef ST_GLOBAL unsigned short *ptr;
    static __device__ __forceinline__ float up(unsigned short b) { return (float)__builtin_bit_cast(_Float16, b); }
    static __device__ __forceinline__ unsigned short down(float x) { return __builtin_bit_cast(unsigned short, (_Float16)x); }
    static __device__ __forceinline__ void load4(ptr p, float x[4])
    {
        const st_u16x4 t = *reinterpret_cast<ST_GLOBAL st_u16x4 *>(p);
        x[0] = up(t.x); x[1] = up(t.y); x[2] = up(t.z); x[3] = up(t.w);
    }
    static __device__ __forceinline__ void store4(ptr p, const float x[4])
    {
        const st_u16x4 t = {down(x[0]), down(x[1]), down(x[2]), down(x[3])};
        *reinterpret_cast<ST_GLOBAL st_u16x4 *>(p) = t;
    }
    static __device__ __forceinline__ float load1(ptr p) { return up(*p); }
    static __device__ __forceinline__ void store1(ptr p, float x) { *p = down(x); }
};
template <int T> __device__ __forceinline__ typename Elems<T>::ptr at(void *p)
{
    return (typename Elems<T>::ptr)p;
}

// ---- norm ---------------------------------------------------------------------------------------------------
// Sum over the workgroup in a fixed order, valid in thread 0.
__device__ __forceinline__ double block_sum_f64(double s, double *red)
{
#pragma unroll
    for (int d = CO3_WAVE / 2; d >= 1; d >>= 1) s += __shfl_xor(s, d, CO3_WAVE);
    if ((threadIdx.x & (CO3_WAVE - 1)) == 0) red[threadIdx.x / CO3_WAVE] = s;
    __syncthreads();
    double t = 0.0;
    for (int w = 0; w < ST_BLOCK / CO3_WAVE; ++w) t += red[w];
    return t;
}

// partials[workgroup] = sum of the squares of its chunks.  In 64 bits: the squares of 24-bit numbers are exact and
// none overflows, so the norm is right for any finite gradient; no atomics, so it is the same in every run.
template <int G>
__global__ __launch_bounds__(ST_BLOCK) void k_grad_sumsq(const Co3StepChunk *__restrict__ plan, int64_t chunks,
                                                          double *__restrict__ partials)
{
    __shared__ double red[ST_BLOCK / CO3_WAVE];
    double s[ST_VEC] = {0.0, 0.0, 0.0, 0.0};
    for (int64_t c = blockIdx.x; c < chunks; c += gridDim.x) {
        const Co3StepChunk ch = plan[c];
        const auto g = at<G>(const_cast<void *>(ch.grad));
        for (int i = threadIdx.x * ST_VEC; i < ch.count; i += ST_TILE) {
            float x[ST_VEC] = {0.f, 0.f, 0.f, 0.f};
            if (i + ST_VEC <= ch.count) Elems<G>::load4(g + i, x);
            else
                for (int e = 0; i + e < ch.count; ++e) x[e] = Elems<G>::load1(g + i + e);
#pragma unroll
            for (int e = 0; e < ST_VEC; ++e) s[e] = __builtin_fma((double)x[e], (double)x[e], s[e]);
        }
    }
    const double t = block_sum_f64((s[0] + s[1]) + (s[2] + s[3]), red);
    if (threadIdx.x == 0) partials[blockIdx.x] = t;
}

// The partial sums of a norm added in a fixed order; out = {norm, factor}, factor < 0 where the norm is not finite.
__device__ __forceinline__ void finish_norm(const double *partials, int64_t count, double grad_scale, double max_norm,
                                            double *red, float &norm, float &factor)
{
    double s = 0.0;
    for (int64_t i = threadIdx.x; i < count; i += ST_BLOCK) s += partials[i];
    s = block_sum_f64(s, red);
    const double total = grad_scale * __builtin_sqrt(s);
    const double c = max_norm / (total + 1e-6);
    norm = (float)total;
    factor = s - s == 0.0 ? (float)(grad_scale * (c < 1.0 ? c : 1.0)) : -1.0f;
}

__global__ __launch_bounds__(ST_BLOCK) void k_norm_finish(const double *__restrict__ partials, int64_t count,
                                                           double grad_scale, double max_norm, float *__restrict__ out)
{
    __shared__ double red[ST_BLOCK / CO3_WAVE];
    float norm, factor;
    finish_norm(partials, count, grad_scale, max_norm, red, norm, factor);
    if (threadIdx.x == 0) {
        out[0] = norm;
        out[1] = factor;
    }
}

// Begins a step whose number the device keeps (a captured step has no other way to count): norm and factor where
// partial sums are given, the number of the step, and what follows from it.
__global__ __launch_bounds__(ST_BLOCK) void k_step_begin(const double *__restrict__ partials, int64_t count, co3_adamw_args a,
                                                          const float *__restrict__ lr_dev, Co3StepDev *__restrict__ dev)
{
    __shared__ double red[ST_BLOCK / CO3_WAVE];
    float norm = 0.0f, factor = (float)a.grad_scale;
    if (partials) finish_norm(partials, count, a.grad_scale, a.max_norm, red, norm, factor);
    if (threadIdx.x != 0) return;
    dev->norm = norm;
    dev->factor = factor;
    if (factor < 0.0f) {
        dev->skipped += 1;
        return;
    }
    a.t = dev->t + 1;
    dev->t = a.t;
    if (lr_dev) a.lr = (double)*lr_dev;
    dev->var = co3_step_var(a);
}

// ---- step ---------------------------------------------------------------------------------------------------
// One element, every operation rounded on its own (the build contracts nothing).
__device__ __forceinline__ void step_moments(const Co3StepFix &c, float factor, float g, float &m, float &v)
{
    g = g * factor;
    m = c.b1 * m + c.c1 * g;
    v = c.b2 * v + c.c2 * (g * g);
}
__device__ __forceinline__ float step_weight(const Co3StepFix &c, float rbc2, float decay, float step, float w, float m, float root)
{
    const float u = m / (root * rbc2 + c.eps);
    return w - (decay * w + step * u);
}

template <int P, int G, bool MASTER>
__global__ __launch_bounds__(ST_BLOCK) void k_adamw(const Co3StepChunk *__restrict__ plan, float *__restrict__ master_all,
                                                     float *__restrict__ m_all, float *__restrict__ v_all, Co3StepFix c,
                                                     Co3StepVar var, float factor, const Co3StepDev *__restrict__ dev)
{
    const Co3StepChunk ch = plan[blockIdx.x];
    if (dev) {
        factor = dev->factor;
        var = dev->var;
        if (factor < 0.0f) return;
    }
    const float step = var.step * ch.lr_scale, decay = (var.lr * ch.lr_scale) * ch.weight_decay;
    const auto p = at<P>(ch.param);
    const auto g = at<G>(const_cast<void *>(ch.grad));
    const auto w32 = at<CO3_F32>(master_all + (MASTER ? ch.state : 0));
    const auto m = at<CO3_F32>(m_all + ch.state), v = at<CO3_F32>(v_all + ch.state);
    for (int i = threadIdx.x * ST_VEC; i < ch.count; i += ST_TILE) {
        if (i + ST_VEC <= ch.count) {
            float gx[ST_VEC], mx[ST_VEC], vx[ST_VEC], wx[ST_VEC];
            Elems<G>::load4(g + i, gx);
            Elems<CO3_F32>::load4(m + i, mx);
            Elems<CO3_F32>::load4(v + i, vx);
            if (MASTER) Elems<CO3_F32>::load4(w32 + i, wx);
            else Elems<P>::load4(p + i, wx);
#pragma unroll
            for (int e = 0; e < ST_VEC; ++e) {
                step_moments(c, factor, gx[e], mx[e], vx[e]);
                wx[e] = step_weight(c, var.rbc2, decay, step, wx[e], mx[e], __builtin_sqrtf(vx[e]));
            }
            Elems<CO3_F32>::store4(m + i, mx);
            Elems<CO3_F32>::store4(v + i, vx);
            if (MASTER) Elems<CO3_F32>::store4(w32 + i, wx);
            Elems<P>::store4(p + i, wx);
        } else {
            for (int j = i; j < ch.count; ++j) {
                float mx = m[j], vx = v[j];
                step_moments(c, factor, Elems<G>::load1(g + j), mx, vx);
                const float wx = step_weight(c, var.rbc2, decay, step, MASTER ? w32[j] : Elems<P>::load1(p + j), mx, __builtin_sqrtf(vx));
                m[j] = mx;
                v[j] = vx;
                if (MASTER) w32[j] = wx;
                Elems<P>::store1(p + j, wx);
            }
        }
    }
}

// ---- step with 8-bit states ---------------------------------------------------------------------------------
// An e4m3 magnitude (exponent bias 7, 3 mantissa bits, gradual underflow) under the scale 2^(s - 127): the bits of the
// code, 20 places up, are an fp32 number with the exponent bias 127, so a change of exponent is all the conversion is.
__device__ __forceinline__ float e4m3_value(uint32_t code, int s)
{
    const float a = ldexpf(__uint_as_float((code & 0x7fu) << 20), s - 7);
    return __uint_as_float(__float_as_uint(a) | ((code & 0x80u) << 24));
}
// The other way 20 bits are cut off; with a random number below 2^20 added before, the code goes up with the
// probability of the part cut off (within a binade, across its end and among the subnormal codes alike).
__device__ __forceinline__ uint32_t e4m3_code(float a, int s, uint32_t random20)
{
    const uint32_t c = (__float_as_uint(ldexpf(a, 7 - s)) + random20) >> 20;
    return c < 126u ? c : 126u;
}
// The scale under which the largest magnitude of a block stays within 448 = 1.75 * 2^8 whichever way it is rounded.
__device__ __forceinline__ int e4m3_scale(uint32_t max_bits)
{
    const int s = (int)((max_bits + 0x200000u) >> 23) - 8;
    return s > 0 ? s : 0;
}

// A wavefront takes a block of 256 elements (the elements that share the scales), four to a lane, so that the largest
// magnitudes are wavefront maxima and nothing passes between wavefronts.
template <int P, int G, bool MASTER>
__global__ __launch_bounds__(ST_BLOCK) void k_adamw8(const Co3StepChunk *__restrict__ plan, float *__restrict__ master_all,
                                                      uint8_t *__restrict__ m_all, uint8_t *__restrict__ ms_all,
                                                      uint8_t *__restrict__ r_all, uint8_t *__restrict__ rs_all, Co3StepFix c,
                                                      Co3StepVar var, float factor, const Co3StepDev *__restrict__ dev)
{
    const Co3StepChunk ch = plan[blockIdx.x];
    if (dev) {
        factor = dev->factor;
        var = dev->var;
        if (factor < 0.0f) return;
    }
    const float step = var.step * ch.lr_scale, decay = (var.lr * ch.lr_scale) * ch.weight_decay;
    const auto p = at<P>(ch.param);
    const auto g = at<G>(const_cast<void *>(ch.grad));
    const auto w32 = at<CO3_F32>(master_all + (MASTER ? ch.state : 0));
    const int lane = threadIdx.x & (CO3_WAVE - 1);
    for (int b = threadIdx.x / CO3_WAVE * CO3_STEP_BLOCK; b < ch.count; b += ST_TILE) {
        const int i = b + lane * ST_VEC;
        const int64_t block = (ch.state + b) / CO3_STEP_BLOCK;
        uint32_t *mp = reinterpret_cast<uint32_t *>(m_all + ch.state + i), *rp = reinterpret_cast<uint32_t *>(r_all + ch.state + i);
        const uint32_t mc = *mp, rc = *rp;             // whole words: the state arrays go on to the end of the block
        const int ms = ms_all[block], rs = rs_all[block];
        const int here = ch.count - i < ST_VEC ? ch.count - i : ST_VEC;      // elements of this lane, may be none or fewer
        float gx[ST_VEC] = {0.f, 0.f, 0.f, 0.f}, wx[ST_VEC] = {0.f, 0.f, 0.f, 0.f}, mx[ST_VEC], rx[ST_VEC];
        if (here == ST_VEC) {
            Elems<G>::load4(g + i, gx);
            if (MASTER) Elems<CO3_F32>::load4(w32 + i, wx);
            else Elems<P>::load4(p + i, wx);
        } else {
            for (int e = 0; e < here; ++e) {
                gx[e] = Elems<G>::load1(g + i + e);
                wx[e] = MASTER ? w32[i + e] : Elems<P>::load1(p + i + e);
            }
        }
        uint32_t mtop = 0, rtop = 0;
#pragma unroll
        for (int e = 0; e < ST_VEC; ++e) {
            const float r = e4m3_value((rc >> (8 * e)) & 0xffu, rs);
            float m = e4m3_value((mc >> (8 * e)) & 0xffu, ms), v = r * r;
            step_moments(c, factor, gx[e], m, v);
            const float root = __builtin_sqrtf(v);
            wx[e] = step_weight(c, var.rbc2, decay, step, wx[e], m, root);
            mx[e] = e < here ? m : 0.0f;
            rx[e] = e < here ? root : 0.0f;
            const uint32_t ma = __float_as_uint(mx[e]) & 0x7fffffffu, ra = __float_as_uint(rx[e]) & 0x7fffffffu;
            mtop = ma > mtop ? ma : mtop;
            rtop = ra > rtop ? ra : rtop;
        }
        const int ms2 = e4m3_scale(wave_max_u32(mtop)), rs2 = e4m3_scale(wave_max_u32(rtop));
        const uint32_t pair = (uint32_t)((ch.state + i) >> 1);
        uint32_t mo = 0, ro = 0;
#pragma unroll
        for (int e = 0; e < ST_VEC; ++e) {
            const uint32_t h = co3_step_fin((pair + e / 2) * CO3_STEP_H0 + var.key);
            const uint32_t x = (e & 1 ? h >> 12 : h << 4) & 0xffff0u;
            const uint32_t mb = __float_as_uint(mx[e]);
            uint32_t mq = e4m3_code(__uint_as_float(mb & 0x7fffffffu), ms2, x + 8u) | (mb >> 24 & 0x80u);
            uint32_t rq = e4m3_code(rx[e], rs2, (x ^ 0xffff0u) + 8u);
            if (rq == 0u && rx[e] != 0.0f) rq = 1u;       // a divisor does not vanish
            if (e >= here) {                              // behind the tensor's last element: as it was
                mq = (mc >> (8 * e)) & 0xffu;
                rq = (rc >> (8 * e)) & 0xffu;
            }
            mo |= mq << (8 * e);
            ro |= rq << (8 * e);
        }
        *mp = mo;
        *rp = ro;
        if (lane == 0) {
            ms_all[block] = (uint8_t)ms2;
            rs_all[block] = (uint8_t)rs2;
        }
        if (here == ST_VEC) {
            if (MASTER) Elems<CO3_F32>::store4(w32 + i, wx);
            Elems<P>::store4(p + i, wx);
        } else {
            for (int e = 0; e < here; ++e) {
                if (MASTER) w32[i + e] = wx[e];
                Elems<P>::store1(p + i + e, wx[e]);
            }
        }
    }
}

// ---- launches -------------------------------------------------------------------------------------------------
hipError_t co3_launch_grad_sumsq(const co3_step_layout *L, const void *plan, double *partials, hipStream_t st)
{
    if (L->chunks == 0) return hipSuccess;
    const auto *pl = static_cast<const Co3StepChunk *>(plan);
    Co3LaunchTimer timer(CO3_K_GRAD_SUMSQ, st);
    const dim3 grid((uint32_t)L->partials), block(ST_BLOCK);
    switch (L->grad_type) {
    case CO3_F32: k_grad_sumsq<CO3_F32><<<grid, block, 0, st>>>(pl, L->chunks, partials); break;
    case CO3_BF16: k_grad_sumsq<CO3_BF16><<<grid, block, 0, st>>>(pl, L->chunks, partials); break;
    default: k_grad_sumsq<CO3_F16><<<grid, block, 0, st>>>(pl, L->chunks, partials); break;
    }
    return hipGetLastError();
}

hipError_t co3_launch_norm_finish(const double *partials, int64_t count, double grad_scale, double max_norm, float *out, hipStream_t st)
{
    k_norm_finish<<<1, ST_BLOCK, 0, st>>>(partials, count, grad_scale, max_norm, out);
    return hipGetLastError();
}

hipError_t co3_launch_step_begin(const double *partials, int64_t count, const co3_adamw_args *a, const float *lr_dev, void *state,
                                 hipStream_t st)
{
    Co3LaunchTimer timer(CO3_K_STEP_BEGIN, st);
    k_step_begin<<<1, ST_BLOCK, 0, st>>>(partials, count, *a, lr_dev, static_cast<Co3StepDev *>(state));
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
