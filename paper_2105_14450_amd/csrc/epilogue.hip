// Backward pass of a linear layer's epilogue: dZ = dY act'(Z) and db = column sums of dZ, in one pass over cubes of Y shards.
// HBM-bandwidth work: Z and dY are read once, dZ is written once; as activation and bias gradient of their own dZ would be
// read a second time.  The sums take dZ in fp32, before it is rounded.
//
// As in the bias gradient of the collectives, a lane owns V consecutive columns, the four wavefronts of a workgroup take
// the rows of a group in turn, and the groups' partial sums are added in ascending order by a second launch.
#include <type_traits>

#include "activation.h"

namespace cube3d {

namespace {

template <typename T, int V> struct __attribute__((aligned(sizeof(T) * V))) Run {
    T v[V];
};

template <int KIND, typename TZ, typename TG, typename TD, int V>
__global__ __launch_bounds__(256) void epilogue_bwd_kernel(CubeGeom g, int RG, int NRG, const TZ *z, const TG *dy, TD *dz, float *__restrict__ part)
{
    __shared__ float lds[4][64 * V];
    constexpr int U = 2;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int r = blockIdx.z, rg = blockIdx.y;
    const int64_t c0 = ((int64_t)blockIdx.x * 64 + lane) * V;
    const bool live = c0 < g.Nb;                       // Nb % V == 0: a lane is all in or all out
    const int64_t row_lo = (int64_t)rg * RG, row_hi = row_lo + RG < g.Ms ? row_lo + RG : g.Ms;
    const int64_t base = (int64_t)r * g.Ms * g.Nb + c0;
    float acc[V];
#pragma unroll
    for (int e = 0; e < V; ++e) acc[e] = 0.f;
    for (int64_t t0 = row_lo + wave; t0 < row_hi; t0 += 4 * U) {
        Run<TZ, V> zv[U];
        Run<TG, V> gv[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t t = t0 + 4 * u;
            if (live && t < row_hi) {
                zv[u] = *reinterpret_cast<const Run<TZ, V> *>(z + base + t * g.Nb);
                gv[u] = *reinterpret_cast<const Run<TG, V> *>(dy + base + t * g.Nb);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t t = t0 + 4 * u;
            if (live && t < row_hi) {
                Run<TD, V> o;
                float x[V];
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    x[e] = to_f32<TG>(gv[u].v[e]) * act_slope<KIND>(to_f32<TZ>(zv[u].v[e]));
                    acc[e] += x[e];
                }
                if constexpr (V == VEC) {
                    typedef Run<TD, V> Out;
                    o = __builtin_bit_cast(Out, pack_out<TD>(x));
                } else {
#pragma unroll
                    for (int e = 0; e < V; ++e) o.v[e] = from_f32<TD>(x[e]);
                }
                *reinterpret_cast<Run<TD, V> *>(dz + base + t * g.Nb) = o;
            }
        }
    }
    if (part == nullptr) return;
#pragma unroll
    for (int e = 0; e < V; ++e) lds[wave][e * 64 + lane] = acc[e];
    __syncthreads();
    float *out = part + ((int64_t)r * NRG + rg) * g.Nb + (int64_t)blockIdx.x * 64 * V;
    for (int x = threadIdx.x; x < 64 * V; x += 256) {
        const int at = x % V * 64 + x / V;             // column x of the chunk
        if ((int64_t)blockIdx.x * 64 * V + x < g.Nb) out[x] = ((lds[0][at] + lds[1][at]) + lds[2][at]) + lds[3][at];
    }
}

int piece(const CubeGeom &g) { return g.Nb % VEC == 0 ? VEC : 1; }

// Rows per workgroup: as many as keep about 2048 workgroups, between 16 and 256; depends on the shape only.
int row_group(const CubeGeom &g)
{
    const int64_t chunks = (g.Nb + 64 * piece(g) - 1) / (64 * piece(g)) * (int64_t)g.q * g.q * g.q;
    int RG = 256;
    while (RG > 16 && chunks * ((g.Ms + RG - 1) / RG) < 2048) RG /= 2;
    while ((g.Ms + RG - 1) / RG > 65535) RG *= 2;
    return RG;
}

}  // namespace

size_t epilogue_bwd_workspace(const CubeGeom &g)
{
    const int RG = row_group(g);
    return (size_t)g.q * g.q * g.q * ((g.Ms + RG - 1) / RG) * g.Nb * sizeof(float);
}

int epilogue_bwd(const CubeGeom &g, int kind, int z_dtype, int dy_dtype, int dz_dtype, const void *z, const void *dy, void *dz,
                 float *dbias_diag, float *workspace, hipStream_t stream)
{
    const int RG = row_group(g), NRG = (int)((g.Ms + RG - 1) / RG), V = piece(g);
    const int64_t chunks = (g.Nb + 64 * V - 1) / (64 * V);
    if (chunks >= 1ll << 24 || (g.Ns + 63) / 64 > 65535) return CUBE3D_ESHAPE;
    const dim3 grid((unsigned)chunks, (unsigned)NRG, (unsigned)(g.q * g.q * g.q));
    auto launch = [&](auto kind_c, auto tz, auto tg, auto td) {
        typedef decltype(tz) TZ;
        typedef decltype(tg) TG;
        typedef decltype(td) TD;
        constexpr int KIND = decltype(kind_c)::value;
        float *part = dbias_diag ? workspace : nullptr;
        if (V == VEC)
            hipLaunchKernelGGL((epilogue_bwd_kernel<KIND, TZ, TG, TD, VEC>), grid, dim3(256), 0, stream, g, RG, NRG,
                               static_cast<const TZ *>(z), static_cast<const TG *>(dy), static_cast<TD *>(dz), part);
        else
            hipLaunchKernelGGL((epilogue_bwd_kernel<KIND, TZ, TG, TD, 1>), grid, dim3(256), 0, stream, g, RG, NRG,
                               static_cast<const TZ *>(z), static_cast<const TG *>(dy), static_cast<TD *>(dz), part);
        return launch_status();
    };
    const float f = 0.f;
    const unsigned short b = 0;
    auto with_dz = [&](auto kind_c, auto tz, auto tg) { return dz_dtype == CUBE3D_F32 ? launch(kind_c, tz, tg, f) : launch(kind_c, tz, tg, b); };
    auto with_dy = [&](auto kind_c, auto tz) { return dy_dtype == CUBE3D_F32 ? with_dz(kind_c, tz, f) : with_dz(kind_c, tz, b); };
    auto with_z = [&](auto kind_c) { return z_dtype == CUBE3D_F32 ? with_dy(kind_c, f) : with_dy(kind_c, b); };
    const int rc = kind == CUBE3D_ACT_RELU ? with_z(std::integral_constant<int, CUBE3D_ACT_RELU>{})
                                           : with_z(std::integral_constant<int, CUBE3D_ACT_GELU>{});
    if (rc != CUBE3D_OK || !dbias_diag) return rc;
    return cube_bias_finish(g, NRG, 1.f, workspace, dbias_diag, stream);
}

}  // namespace cube3d
