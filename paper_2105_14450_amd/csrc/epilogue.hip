// Backward pass of a linear layer's epilogue: dZ = dY act'(Z) and db = column sums of dZ, in one pass over cubes of Y shards.
// HBM-bandwidth work: Z and dY are read once, dZ is written once; as activation and bias gradient of their own dZ would be
// read a second time.  The sums take dZ in fp32, before it is rounded.  8192 x 8192 bf16 with GELU, 403 MB: 91 us = 4.4 TB/s, a copy of
// 1 GiB making 4.8.
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

template <typename To, typename From> __device__ __forceinline__ To bit_cast_to(const From &x) { return __builtin_bit_cast(To, x); }

// V elements at any alignment, or the first `valid` of them
template <typename T, int V> struct __attribute__((packed, aligned(sizeof(T)))) LooseRun {
    T v[V];
};
template <bool LOOSE, typename T, int V> __device__ __forceinline__ Run<T, V> get_run(const T *from, int valid)
{
    if constexpr (!LOOSE) return *reinterpret_cast<const Run<T, V> *>(from);
    if (valid == V) return bit_cast_to<Run<T, V>>(*reinterpret_cast<const LooseRun<T, V> *>(from));
    Run<T, V> x;
#pragma unroll
    for (int e = 0; e < V; ++e) x.v[e] = e < valid ? from[e] : T(0);
    return x;
}
template <bool LOOSE, typename T, int V> __device__ __forceinline__ void put_run(T *to, int valid, const Run<T, V> &x)
{
    if constexpr (!LOOSE) {
        *reinterpret_cast<Run<T, V> *>(to) = x;
        return;
    }
    if (valid == V) {
        *reinterpret_cast<LooseRun<T, V> *>(to) = bit_cast_to<LooseRun<T, V>>(x);
        return;
    }
#pragma unroll
    for (int e = 0; e < V; ++e)
        if (e < valid) to[e] = x.v[e];
}

// Grid: chunks of 2^shift lanes' columns, row groups, processors.  A wavefront takes 64 / 2^shift rows at a time (narrow blocks: several).
template <int KIND, typename TZ, typename TG, typename TD, int V, bool LOOSE>
__global__ __launch_bounds__(256) void epilogue_bwd_kernel(CubeGeom g, int RG, int NRG, int shift, const TZ *z, const TG *dy, TD *dz,
                                                           float *__restrict__ part)
{
    __shared__ float lds[4][64 * V];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int r = blockIdx.z, rg = blockIdx.y, width = 1 << shift, rows = 64 >> shift;
    const int64_t c0 = ((int64_t)blockIdx.x * width + (lane & (width - 1))) * V;
    const bool live = c0 < g.Nb;                       // (Nb % V == 0: a lane is all in or all out)
    const int valid = LOOSE ? (int)min((int64_t)V, g.Nb - c0) : V;
    const int64_t row_lo = (int64_t)rg * RG, row_hi = row_lo + RG < g.Ms ? row_lo + RG : g.Ms;
    const int64_t t_lo = row_lo + wave * rows + (lane >> shift), step = (int64_t)(4 * rows) * g.Nb;      // elements between a lane's rows
    int64_t at = ((int64_t)r * g.Ms + t_lo) * g.Nb + c0;
    float acc[V];
#pragma unroll
    for (int e = 0; e < V; ++e) acc[e] = 0.f;
    const int turns = live && t_lo < row_hi ? (int)((row_hi - t_lo + 4 * rows - 1) / (4 * rows)) : 0;
    for (int n = 0; n < turns; ++n, at += step) {      // (two and four rows at a time: 94.7 and 95.3 us for 91.0 at 8192 x 8192 bf16)
        const Run<TZ, V> zv = get_run<LOOSE, TZ, V>(z + at, valid);
        const Run<TG, V> gv = get_run<LOOSE, TG, V>(dy + at, valid);
        Run<TD, V> o;
        float x[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            x[e] = to_f32<TG>(gv.v[e]) * act_slope<KIND>(to_f32<TZ>(zv.v[e]));
            acc[e] += x[e];
        }
        if constexpr (V == VEC) {
            typedef Run<TD, V> Out;
            o = __builtin_bit_cast(Out, pack_out<TD>(x));
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) o.v[e] = from_f32<TD>(x[e]);
        }
        put_run<LOOSE, TD, V>(dz + at, valid, o);
    }
    if (part == nullptr) return;
#pragma unroll
    for (int e = 0; e < V; ++e) lds[wave][e * 64 + lane] = acc[e];
    __syncthreads();
    float *out = part + ((int64_t)r * NRG + rg) * g.Nb + (int64_t)blockIdx.x * width * V;
    for (int x = threadIdx.x; x < width * V; x += 256) {
        if ((int64_t)blockIdx.x * width * V + x >= g.Nb) continue;
        float sum = 0.f;                               // column x of the chunk: the wavefronts' rows in ascending order
        for (int k = 0; k < rows; ++k) {
            const int at = x % V * 64 + k * width + x / V;
            sum += ((lds[0][at] + lds[1][at]) + lds[2][at]) + lds[3][at];
        }
        out[x] = sum;
    }
}

// Columns a lane owns: eight, or four or two where that is what blocks are a multiple of.  Long odd blocks: eight in accesses of any
// alignment, the last lane of a row what is left (us, in eights / single elements: 8192 x 4101 bf16 51 / 80, fp32 110 / 126; but
// 30000 x 129 30 / 23; in twos, 8192 x 4098 bf16 49 / 52, fp32 111 / 93)
int piece(const CubeGeom &g)
{
    return g.Nb % VEC == 0 ? VEC : g.Nb % 4 == 0 ? 4 : g.Nb % 2 == 0 ? 2 : g.Nb >= 512 ? VEC : 1;
}

// Lanes on a row, as a power of two
int lane_shift(const CubeGeom &g)
{
    int shift = 0;
    while (shift < 6 && (piece(g) << shift) < g.Nb) ++shift;
    return shift;
}

int64_t chunk_count(const CubeGeom &g)
{
    const int64_t width = (int64_t)piece(g) << lane_shift(g);
    return (g.Nb + width - 1) / width;
}

// Rows per workgroup, from two turns of its wavefronts to 64: as many as keep 512 workgroups, or 1024 for large layers (us with 512 /
// 1024 / 2048: 32768 x 512 30 / 36 / 53, 20000 x 1000 29 / 34 / 44, where the second launch adds up many partial sums of few columns;
// 8192 x 8192 94.6 / 91.0 / 93.8).  Depends on the shape only.
int row_group(const CubeGeom &g)
{
    const int64_t chunks = chunk_count(g) * g.q * g.q * g.q, turn = 4 * (64 >> lane_shift(g));
    const int64_t enough = g.M * g.N < (1ll << 25) ? 512 : 1024;
    int64_t RG = 64 * turn;
    while (RG > 2 * turn && chunks * ((g.Ms + RG - 1) / RG) < enough) RG /= 2;
    while ((g.Ms + RG - 1) / RG > 65535) RG *= 2;
    return (int)RG;
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
    const int64_t chunks = chunk_count(g);
    const int shift = lane_shift(g);
    if (chunks >= 1ll << 24 || (g.Ns + 63) / 64 > 65535) return CUBE3D_ESHAPE;
    const dim3 grid((unsigned)chunks, (unsigned)NRG, (unsigned)(g.q * g.q * g.q));
    auto launch = [&](auto kind_c, auto tz, auto tg, auto td) {
        typedef decltype(tz) TZ;
        typedef decltype(tg) TG;
        typedef decltype(td) TD;
        constexpr int KIND = decltype(kind_c)::value;
        float *part = dbias_diag ? workspace : nullptr;
        auto of_width = [&](auto v, auto loose) {
            hipLaunchKernelGGL((epilogue_bwd_kernel<KIND, TZ, TG, TD, decltype(v)::value, decltype(loose)::value>), grid, dim3(256), 0, stream, g,
                               RG, NRG, shift, static_cast<const TZ *>(z), static_cast<const TG *>(dy), static_cast<TD *>(dz), part);
        };
        const std::integral_constant<int, VEC> eight{};
        if (g.Nb % V) of_width(eight, std::true_type{});
        else if (V == VEC) of_width(eight, std::false_type{});
        else if (V == 4) of_width(std::integral_constant<int, 4>{}, std::false_type{});
        else if (V == 2) of_width(std::integral_constant<int, 2>{}, std::false_type{});
        else of_width(std::integral_constant<int, 1>{}, std::false_type{});
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
