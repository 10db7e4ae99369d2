// AdamW (decoupled weight decay) over many tensors in few launches.
#include <float.h>
#include <math.h>

#include "checks.hpp"

namespace dm {
namespace {

constexpr int NT = 256;
constexpr int STATE_BLOCK = 256;   // elements of an 8-bit state that share a scale: 4 of each lane of a wave
constexpr int CHUNK = 4096;        // elements of a block
// blocks of a launch: a grid holds less than 2^32 threads along x (more wrap, without an error)
constexpr int64_t BLOCKS = (((int64_t)1 << 32) - 1) / NT;
constexpr float E4M3_MAX = 448.f;  // largest e4m3 value
// blocks whose largest value is below 2^-100 are zeros (its reciprocal times 448 would overflow)
constexpr float LEAST = 0x1p-100f;

struct Item {
    void* param;
    float* master;
    const float* grad;
    void *m, *v;
    float *m_scale, *v_scale;
    int64_t n;
    float decay, keep;  // keep = 1 - lr decay
};
// tensors of a launch: what the 4 KB of kernel arguments hold
constexpr int ITEMS = 44;
struct Job {
    Item item[ITEMS];
    uint32_t first[ITEMS];  // first block of each
    int n;
    float lr, b1, c1, b2, c2, eps, inv1, inv2, gscale;  // c = 1 - b; inv = 1 / (1 - b^step)
    const float* scalars;
};
static_assert(sizeof(Job) <= 4096, "kernel arguments");

// Every operation rounds by itself: the step is the same in all variants
// and wherever an element lies, and an 8-bit code depends on nothing but its
// block's values.
#pragma clang fp contract(off)

// 4 consecutive elements
template <typename T> __device__ __forceinline__ void load4(const T* p, int n, float x[4]) {
    typedef T T4 __attribute__((ext_vector_type(4)));
    if (n == 4) {
        const T4 r = *reinterpret_cast<const T4*>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = to_f((T)r[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = i < n ? to_f(p[i]) : 0.f;
    }
}
template <typename T> __device__ __forceinline__ void save4(T* p, int n, const float x[4]) {
    typedef T T4 __attribute__((ext_vector_type(4)));
    if (n == 4) {
        *reinterpret_cast<T4*>(p) = T4{from_f<T>(x[0]), from_f<T>(x[1]), from_f<T>(x[2]), from_f<T>(x[3])};
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n) p[i] = from_f<T>(x[i]);
    }
}
// 4 e4m3 codes times a scale, and back
__device__ __forceinline__ void load4(const uint8_t* p, int n, float scale, float x[4]) {
    uint32_t r = 0;
    if (n == 4) {
        r = *reinterpret_cast<const uint32_t*>(p);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n) r |= (uint32_t)p[i] << (8 * i);
    }
    x[0] = __builtin_amdgcn_cvt_f32_fp8((int)r, 0) * scale;
    x[1] = __builtin_amdgcn_cvt_f32_fp8((int)r, 1) * scale;
    x[2] = __builtin_amdgcn_cvt_f32_fp8((int)r, 2) * scale;
    x[3] = __builtin_amdgcn_cvt_f32_fp8((int)r, 3) * scale;
}
// ROOT: what is not zero keeps the smallest code (a second moment that
// became zero would let its element's step grow without bound)
template <bool ROOT> __device__ __forceinline__ float pack4(uint8_t* p, int n, const float x[4]) {
    const float top = group_max<64>(fmaxf(fmaxf(fabsf(x[0]), fabsf(x[1])), fmaxf(fabsf(x[2]), fabsf(x[3]))));
    const bool held = top >= LEAST;
    // (both by a reciprocal, as a plain form of it on the device computes them: one ulp of the scale moves codes
    // that lie next to a tie, and an element whose second moment is tiny turns that into a step of its own)
    const float f = held ? (1.f / top) * E4M3_MAX : 0.f;
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * f, x[1] * f, 0, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(x[2] * f, x[3] * f, r, true);
    uint32_t c = (uint32_t)r;
    if (ROOT) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (x[i] > 0.f && ((c >> (8 * i)) & 0xFFu) == 0) c |= 1u << (8 * i);
    }
    if (n == 4) {
        *reinterpret_cast<uint32_t*>(p) = c;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n) p[i] = (uint8_t)(c >> (8 * i));
    }
    return held ? top * (1.f / E4M3_MAX) : 0.f;
}

// One pass over everything, 4 elements a lane at a time.  Bound by memory: 12.6
// million fp16 weights with fp32 copies and states (30 bytes each, 378 MB) in
// 76 us, 5.0 TB/s; 302 million bf16 weights with fp32 copies and 8-bit states
// (18 bytes each) in 1090, 5.0.  16 tensors of 32 to 4096: 6.5 us, a launch.
template <typename T, bool MASTER, int BITS>
__global__ __launch_bounds__(NT) void adamw_k(Job job) {
    const int lane = threadIdx.x & 63;
    // this block's tensor: the last that begins at or before it
    const bool mine = lane < job.n && job.first[lane < ITEMS ? lane : 0] <= blockIdx.x;
    const int it = __builtin_amdgcn_readfirstlane(__popcll(__ballot(mine)) - 1);
    const Item& t = job.item[it];
    float lr = job.lr, inv1 = job.inv1, inv2 = job.inv2, gs = job.gscale, keep = t.keep;
    if (job.scalars) {
        lr = job.scalars[0];
        inv1 = job.scalars[1];
        inv2 = job.scalars[2];
        gs = job.scalars[3];
        keep = 1.f - lr * t.decay;
    }
    const int64_t c0 = (int64_t)(blockIdx.x - job.first[it]) * CHUNK;
#pragma unroll
    for (int s = 0; s < CHUNK; s += NT * 4) {
        const int64_t e = c0 + s + threadIdx.x * 4;
        const int64_t w0 = c0 + s + (threadIdx.x >> 6) * STATE_BLOCK;  // the wave's first element
        if (w0 >= t.n) return;
        const int n = e >= t.n ? 0 : t.n - e < 4 ? (int)(t.n - e) : 4;
        float g[4], w[4], m[4], v[4];
        load4(t.grad + e, n, g);
        if (MASTER) load4(t.master + e, n, w);
        else load4((const T*)t.param + e, n, w);
        const int64_t blk = w0 / STATE_BLOCK;
        if (BITS == 32) {
            load4((const float*)t.m + e, n, m);
            load4((const float*)t.v + e, n, v);
        } else {
            load4((const uint8_t*)t.m + e, n, t.m_scale[blk], m);
            load4((const uint8_t*)t.v + e, n, t.v_scale[blk], v);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = v[i] * v[i];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float gi = g[i] * gs;
            m[i] = m[i] * job.b1 + gi * job.c1;
            v[i] = v[i] * job.b2 + (gi * gi) * job.c2;
            const float u = (m[i] * inv1) / (sqrtf(v[i] * inv2) + job.eps);
            w[i] = w[i] * keep - u * lr;
        }
        if (MASTER) save4(t.master + e, n, w);
        save4((T*)t.param + e, n, w);
        if (BITS == 32) {
            save4((float*)t.m + e, n, m);
            save4((float*)t.v + e, n, v);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = sqrtf(v[i]);
            if (n < 4) {  // elements behind the end have no part in the block's largest value
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (i >= n) m[i] = v[i] = 0.f;
            }
            const float ms = pack4<false>((uint8_t*)t.m + e, n, m), vs = pack4<true>((uint8_t*)t.v + e, n, v);
            if (lane == 0) {
                t.m_scale[blk] = ms;
                t.v_scale[blk] = vs;
            }
        }
    }
}
#pragma clang fp contract(on)

template <typename T, bool MASTER> void launch(const Job& j, int bits, unsigned blocks, hipStream_t st) {
    if (bits == 32) adamw_k<T, MASTER, 32><<<dim3(blocks), NT, 0, st>>>(j);
    else adamw_k<T, MASTER, 8><<<dim3(blocks), NT, 0, st>>>(j);
}

void launch(const Job& j, int dtype, bool master, int bits, unsigned blocks, hipStream_t st) {
    if (dtype == DM_F32) launch<float, false>(j, bits, blocks, st);
    else if (dtype == DM_F16) master ? launch<half_t, true>(j, bits, blocks, st) : launch<half_t, false>(j, bits, blocks, st);
    else master ? launch<bf16_t, true>(j, bits, blocks, st) : launch<bf16_t, false>(j, bits, blocks, st);
}

// The step computes in float32: a number that is none there would make every
// weight infinite or NaN.
bool finite32(double x) { return isfinite((float)x); }

int check_item(const dm_adamw_tensor& t, int i, const dm_adamw_desc& a) {
    if (t.n < 0) return set_error(DM_ERR_ARG, "tensor %d: n=%lld", i, (long long)t.n);
    if (t.n > BLOCKS * CHUNK)
        return set_error(DM_ERR_UNSUPPORTED, "tensor %d: n=%lld is more than a launch holds", i, (long long)t.n);
    if (!(t.decay >= 0.) || !finite32(t.decay)) return set_error(DM_ERR_ARG, "tensor %d: decay=%g", i, t.decay);
    if (t.n == 0) return DM_OK;
    const void* p[4] = {t.param, t.grad, t.m, t.v};
    const char* n[4] = {"param", "grad", "m", "v"};
    for (int k = 0; k < 4; ++k)
        if (!p[k] || !aligned16(p[k]))
            return set_error(DM_ERR_ARG, "tensor %d: %s is NULL or not 16-byte aligned", i, n[k]);
    if (t.master && a.dtype == DM_F32)
        return set_error(DM_ERR_ARG, "tensor %d: float32 weights have no master copy", i);
    if (t.master && !aligned16(t.master)) return set_error(DM_ERR_ARG, "tensor %d: master is not 16-byte aligned", i);
    const bool scales = t.m_scale && t.v_scale && ((uintptr_t)t.m_scale & 3u) == 0 && ((uintptr_t)t.v_scale & 3u) == 0;
    if (a.state_bits == 8 && !scales)
        return set_error(DM_ERR_ARG, "tensor %d: a state scale is NULL or not 4-byte aligned", i);
    if (a.state_bits == 32 && (t.m_scale || t.v_scale))
        return set_error(DM_ERR_ARG, "tensor %d: states in 32 bits have no scales", i);
    return DM_OK;
}

}  // namespace
}  // namespace dm

using namespace dm;

extern "C" {

int adamw_step(const dm_adamw_desc* a, const dm_adamw_tensor* tensors, int32_t count, void* stream) {
    if (!a) return set_error(DM_ERR_ARG, "descriptor is NULL");
    DM_TRY(check_dtype(a->dtype));
    if (a->state_bits != 8 && a->state_bits != 32)
        return set_error(DM_ERR_UNSUPPORTED, "states in %d bits: 8 or 32", a->state_bits);
    if (!(a->beta1 >= 0. && a->beta1 < 1.) || !(a->beta2 >= 0. && a->beta2 < 1.))
        return set_error(DM_ERR_ARG, "beta1=%g beta2=%g outside [0,1)", a->beta1, a->beta2);
    // (an eps that float32 holds as zero makes 0 / 0 of an element without a gradient)
    if (!((float)a->eps >= FLT_MIN) || !finite32(a->eps))
        return set_error(DM_ERR_ARG, "eps=%g must be > 0, a normal float32 number", a->eps);
    if (!a->scalars) {
        if (!finite32(a->lr) || a->lr < 0.) return set_error(DM_ERR_ARG, "lr=%g", a->lr);
        if (!finite32(a->grad_scale)) return set_error(DM_ERR_ARG, "grad_scale=%g", a->grad_scale);
        if (a->step < 1) return set_error(DM_ERR_ARG, "step=%lld: the first step is 1", (long long)a->step);
    } else {
        DM_TRY(check_ptr(a->scalars, "scalars"));
    }
    if (count < 0 || (count > 0 && !tensors)) return set_error(DM_ERR_ARG, "tensors missing");
    bool any = false, master = false;
    for (int i = 0; i < count; ++i) {
        DM_TRY(check_item(tensors[i], i, *a));
        if (tensors[i].n == 0) continue;
        if (any && master != (tensors[i].master != nullptr))
            return set_error(DM_ERR_ARG, "tensor %d: all tensors of a call have a master copy, or none", i);
        any = true;
        master = tensors[i].master != nullptr;
    }
    if (!any) return DM_OK;
    const hipStream_t st = S(stream);
    Job j{};
    j.b1 = (float)a->beta1; j.c1 = (float)(1. - a->beta1);
    j.b2 = (float)a->beta2; j.c2 = (float)(1. - a->beta2);
    j.eps = (float)a->eps;
    j.scalars = a->scalars;
    if (!a->scalars) {
        j.lr = (float)a->lr;
        j.inv1 = (float)(1. / (1. - pow(a->beta1, (double)a->step)));
        j.inv2 = (float)(1. / (1. - pow(a->beta2, (double)a->step)));
        j.gscale = (float)a->grad_scale;
    }
    uint32_t blocks = 0;
    for (int i = 0; i <= count; ++i) {
        const int64_t nb = i < count ? (tensors[i].n + CHUNK - 1) / CHUNK : 0;
        if (j.n > 0 && (i == count || j.n == ITEMS || blocks + nb > BLOCKS)) {
            launch(j, a->dtype, master, a->state_bits, blocks, st);
            j.n = 0;
            blocks = 0;
        }
        if (nb == 0) continue;
        const dm_adamw_tensor& t = tensors[i];
        j.item[j.n] = Item{t.param, t.master, t.grad, t.m, t.v, t.m_scale, t.v_scale, t.n, (float)t.decay,
                           (float)(1. - a->lr * t.decay)};
        j.first[j.n++] = blocks;
        blocks += (uint32_t)nb;
    }
    return check_launch("adamw_step");
}

}  // extern "C"
