// Element-wise arithmetic shared by the kernels that act on stored activations: eight elements at a time in fp32, and the
// activation functions of the MLP block with their slopes.
#pragma once
#include "common.h"

namespace cube3d {

constexpr int VEC = 8;      // elements of one access per lane

template <typename T> struct __attribute__((aligned(sizeof(T) * VEC))) Pack8 {
    T v[VEC];
};

template <typename T> __device__ __forceinline__ float to_f32(T x);
template <> __device__ __forceinline__ float to_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ float to_f32<unsigned short>(unsigned short x) { return bf16_bits_to_f32(x); }
template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ unsigned short from_f32<unsigned short>(float x) { return f32_to_bf16_bits(x); }

// eight results to the stored type (bf16: four packed conversions, round to nearest even)
template <typename T> __device__ __forceinline__ Pack8<T> pack_out(const float (&v)[VEC]);
template <> __device__ __forceinline__ Pack8<float> pack_out<float>(const float (&v)[VEC])
{
    Pack8<float> o;
#pragma unroll
    for (int e = 0; e < VEC; ++e) o.v[e] = v[e];
    return o;
}
template <> __device__ __forceinline__ Pack8<unsigned short> pack_out<unsigned short>(const float (&v)[VEC])
{
    uint4 w;
    w.x = pack_bf16x2(v[0], v[1]);
    w.y = pack_bf16x2(v[2], v[3]);
    w.z = pack_bf16x2(v[4], v[5]);
    w.w = pack_bf16x2(v[6], v[7]);
    return __builtin_bit_cast(Pack8<unsigned short>, w);
}

// Phi(z), the standard normal distribution function, and phi(z), its density, in fp32 without
// branches.  For t = |z| < 6 the lower tail is Phi(-t) = 2^(-r(t)) / 2 with r(t) = -log2(2 Phi(-t)),
// a smooth function (r(0) = 0, r ~ t^2 log2(e) / 2 for large t) taken as t times a degree-9 polynomial
// (least-squares fit at 4000 Chebyshev nodes of [0, 6]: 1.2e-6 relative to the tail); beyond 6, where
// the tail is below 1e-9, the Gaussian bound 2^(-t^2 log2(e) / 2) / 2 stands in, which goes to zero
// as t grows.  The upper side is 1 - Phi(-t).  The tail keeps its relative accuracy (4e-6 after fp32
// rounding of r) however small it is, which 1 + erf(z / sqrt 2) does not; z Phi(z) is within 4e-7 of
// the exact value for |z| < 12.  One v_exp_f32 per function instead of the library erf's two ranges.
struct NormalFn {
    float cdf, pdf;
};

__device__ __forceinline__ NormalFn normal_fn(float z)
{
    const float t = fabsf(z);
    const float tq = t * t * 0.72134752f;               // t^2 / 2 in units of log2
    float r = 1.945418582e-08f;
    r = fmaf(r, t, -6.227335234e-07f);
    r = fmaf(r, t, 8.505122423e-06f);
    r = fmaf(r, t, -6.270727317e-05f);
    r = fmaf(r, t, 2.353099990e-04f);
    r = fmaf(r, t, 8.306837117e-05f);
    r = fmaf(r, t, -7.032936905e-03f);
    r = fmaf(r, t, 5.248502642e-02f);
    r = fmaf(r, t, 4.592124820e-01f);
    r = fmaf(r, t, 1.151104450e+00f);
    r = t < 6.f ? r * t : tq;
    const float tail = 0.5f * __builtin_amdgcn_exp2f(-r);
    NormalFn f;
    f.cdf = z < 0.f ? tail : 1.f - tail;
    f.pdf = 0.39894228040143268f * __builtin_amdgcn_exp2f(-tq);
    return f;
}

template <int KIND> __device__ __forceinline__ float act_value(float z)
{
    if (KIND == CUBE3D_ACT_RELU) return z > 0.f ? z : 0.f;
    return z * normal_fn(z).cdf;
}

template <int KIND> __device__ __forceinline__ float act_slope(float z)
{
    if (KIND == CUBE3D_ACT_RELU) return z > 0.f ? 1.f : 0.f;
    const NormalFn f = normal_fn(z);
    return f.cdf + z * f.pdf;
}

// The activation of a product's epilogue: the rectifier keeps NaN.  (The passes over stored activations make it 0, as they always have.)
template <int KIND> __device__ __forceinline__ float epilogue_act(float z)
{
    if (KIND == CUBE3D_ACT_RELU) return z <= 0.f ? 0.f : z;
    return act_value<KIND>(z);
}

// A product's epilogue on one value z of the fp32 result, which sits at element `at` of the output (and of residual and Z): keeps
// Z and returns y = act(z) + residual.
__device__ __forceinline__ float epilogue_element(const Epilogue &e, float z, int64_t at)
{
    if (e.z) {
        if (e.z_f32) static_cast<float *>(e.z)[at] = z;
        else static_cast<unsigned short *>(e.z)[at] = f32_to_bf16_bits(z);
    }
    float y = e.act == CUBE3D_ACT_GELU ? epilogue_act<CUBE3D_ACT_GELU>(z) : e.act == CUBE3D_ACT_RELU ? epilogue_act<CUBE3D_ACT_RELU>(z) : z;
    if (e.residual)
        y += e.residual_f32 ? static_cast<const float *>(e.residual)[at] : bf16_bits_to_f32(static_cast<const unsigned short *>(e.residual)[at]);
    return y;
}

}  // namespace cube3d
