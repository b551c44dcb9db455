// Element-wise activation between the two linear layers of the MLP block (Section 3.2), forward
// and backward, over a whole cube buffer: the activation acts on every processor's shard
// independently, so on one GPU it is a single streaming pass.  HBM-bandwidth work.
//   forward   h = act(z)
//   backward  dz = dh * act'(z)
// act = rectifier max(z, 0) (slope 0 at 0) or the Gaussian error linear unit in its exact form
// z * Phi(z) (no tanh or logistic stand-in), Phi evaluated in fp32.  Eight elements per lane per step,
// 16-byte accesses.
#include "activation.h"

namespace cube3d {

namespace {

constexpr int UNROLL = 2;

template <int KIND, typename TZ, typename TH>
__global__ __launch_bounds__(256) void act_fwd_kernel(const TZ *__restrict__ z, TH *__restrict__ h, int64_t n)
{
    const int64_t nvec = n / VEC, stride = (int64_t)gridDim.x * 256;
    const Pack8<TZ> *zv = reinterpret_cast<const Pack8<TZ> *>(z);
    Pack8<TH> *hv = reinterpret_cast<Pack8<TH> *>(h);
    int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    for (; i + (UNROLL - 1) * stride < nvec; i += UNROLL * stride) {   // UNROLL loads in flight per lane
        Pack8<TZ> a[UNROLL];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) a[u] = zv[i + u * stride];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            float o[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) o[e] = act_value<KIND>(to_f32<TZ>(a[u].v[e]));
            hv[i + u * stride] = pack_out<TH>(o);
        }
    }
    for (; i < nvec; i += stride) {
        const Pack8<TZ> a = zv[i];
        float o[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) o[e] = act_value<KIND>(to_f32<TZ>(a.v[e]));
        hv[i] = pack_out<TH>(o);
    }
    if (blockIdx.x == 0)
        for (int64_t i = nvec * VEC + threadIdx.x; i < n; i += 256) h[i] = from_f32<TH>(act_value<KIND>(to_f32<TZ>(z[i])));
}

template <int KIND, typename TZ, typename TG, typename TD>
__global__ __launch_bounds__(256) void act_bwd_kernel(const TZ *__restrict__ z, const TG *__restrict__ dh,
                                                      TD *__restrict__ dz, int64_t n)
{
    const int64_t nvec = n / VEC, stride = (int64_t)gridDim.x * 256;
    const Pack8<TZ> *zv = reinterpret_cast<const Pack8<TZ> *>(z);
    const Pack8<TG> *gv = reinterpret_cast<const Pack8<TG> *>(dh);
    Pack8<TD> *dv = reinterpret_cast<Pack8<TD> *>(dz);
    int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    for (; i + (UNROLL - 1) * stride < nvec; i += UNROLL * stride) {
        Pack8<TZ> a[UNROLL];
        Pack8<TG> g[UNROLL];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            a[u] = zv[i + u * stride];
            g[u] = gv[i + u * stride];
        }
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            float o[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) o[e] = to_f32<TG>(g[u].v[e]) * act_slope<KIND>(to_f32<TZ>(a[u].v[e]));
            dv[i + u * stride] = pack_out<TD>(o);
        }
    }
    for (; i < nvec; i += stride) {
        const Pack8<TZ> a = zv[i];
        const Pack8<TG> g = gv[i];
        float o[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) o[e] = to_f32<TG>(g.v[e]) * act_slope<KIND>(to_f32<TZ>(a.v[e]));
        dv[i] = pack_out<TD>(o);
    }
    if (blockIdx.x == 0)
        for (int64_t i = nvec * VEC + threadIdx.x; i < n; i += 256)
            dz[i] = from_f32<TD>(to_f32<TG>(dh[i]) * act_slope<KIND>(to_f32<TZ>(z[i])));
}

unsigned grid_for(int64_t n)
{
    const int64_t want = (n / VEC + 255) / 256;
    const int64_t cap = 256 * 8;   // eight blocks per CU
    return (unsigned)(want < 1 ? 1 : want > cap ? cap : want);
}

template <int KIND, typename TZ> int fwd_out(int h_dtype, int64_t n, const void *z, void *h, hipStream_t s)
{
    const TZ *zp = static_cast<const TZ *>(z);
    if (h_dtype == CUBE3D_F32)
        hipLaunchKernelGGL((act_fwd_kernel<KIND, TZ, float>), dim3(grid_for(n)), dim3(256), 0, s, zp, static_cast<float *>(h), n);
    else
        hipLaunchKernelGGL((act_fwd_kernel<KIND, TZ, unsigned short>), dim3(grid_for(n)), dim3(256), 0, s, zp,
                           static_cast<unsigned short *>(h), n);
    return launch_status();
}

template <int KIND, typename TZ, typename TG>
int bwd_out(int dz_dtype, int64_t n, const void *z, const void *dh, void *dz, hipStream_t s)
{
    const TZ *zp = static_cast<const TZ *>(z);
    const TG *gp = static_cast<const TG *>(dh);
    if (dz_dtype == CUBE3D_F32)
        hipLaunchKernelGGL((act_bwd_kernel<KIND, TZ, TG, float>), dim3(grid_for(n)), dim3(256), 0, s, zp, gp,
                           static_cast<float *>(dz), n);
    else
        hipLaunchKernelGGL((act_bwd_kernel<KIND, TZ, TG, unsigned short>), dim3(grid_for(n)), dim3(256), 0, s, zp, gp,
                           static_cast<unsigned short *>(dz), n);
    return launch_status();
}

template <int KIND, typename TZ>
int bwd_g(int g_dtype, int dz_dtype, int64_t n, const void *z, const void *dh, void *dz, hipStream_t s)
{
    return g_dtype == CUBE3D_F32 ? bwd_out<KIND, TZ, float>(dz_dtype, n, z, dh, dz, s)
                                 : bwd_out<KIND, TZ, unsigned short>(dz_dtype, n, z, dh, dz, s);
}

}  // namespace

int activation_fwd(int kind, int z_dtype, int h_dtype, int64_t n, const void *z, void *h, hipStream_t s)
{
    if (kind == CUBE3D_ACT_RELU)
        return z_dtype == CUBE3D_F32 ? fwd_out<CUBE3D_ACT_RELU, float>(h_dtype, n, z, h, s)
                                     : fwd_out<CUBE3D_ACT_RELU, unsigned short>(h_dtype, n, z, h, s);
    return z_dtype == CUBE3D_F32 ? fwd_out<CUBE3D_ACT_GELU, float>(h_dtype, n, z, h, s)
                                 : fwd_out<CUBE3D_ACT_GELU, unsigned short>(h_dtype, n, z, h, s);
}

int activation_bwd(int kind, int z_dtype, int g_dtype, int dz_dtype, int64_t n, const void *z, const void *dh, void *dz,
                   hipStream_t s)
{
    if (kind == CUBE3D_ACT_RELU)
        return z_dtype == CUBE3D_F32 ? bwd_g<CUBE3D_ACT_RELU, float>(g_dtype, dz_dtype, n, z, dh, dz, s)
                                     : bwd_g<CUBE3D_ACT_RELU, unsigned short>(g_dtype, dz_dtype, n, z, dh, dz, s);
    return z_dtype == CUBE3D_F32 ? bwd_g<CUBE3D_ACT_GELU, float>(g_dtype, dz_dtype, n, z, dh, dz, s)
                                 : bwd_g<CUBE3D_ACT_GELU, unsigned short>(g_dtype, dz_dtype, n, z, dh, dz, s);
}

}  // namespace cube3d
