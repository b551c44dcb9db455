// The global norm of many gradient arrays, and the arrays scaled to a largest norm.
//   S = sum of g^2 over every element of every array;  norm = scale sqrt(S);  out = f g,  f = scale min(1, max / norm)
// HBM-bandwidth work: the norm reads every gradient once, clipping reads it again (f is known only then) and writes it.
//
// Squares are formed and added in fp64: an fp32 square overflows from |g| = 1.8e19 on and loses bits below 1e-19, and gradients
// of 1e-25 are ordinary in bf16 without loss scaling.
//
// The arrays' addresses and sizes travel in the kernels' arguments (nothing is copied to the device), MAX_ARRAYS of them
// per launch.  An array is cut into units of UNIT elements; workgroup w takes the units w, w + grid, ... of the launch, so
// that arrays of any sizes share the chip evenly, and leaves one partial sum.  Which units a workgroup adds and in what
// order depends on the sizes and the number of CUs only: two calls give the same bits.
#include <algorithm>
#include <new>

#include "activation.h"

namespace cube3d {

namespace {

constexpr int MAX_ARRAYS = 112;         // per launch: 3.9 KB of arguments
constexpr int UNIT = 8192;              // elements: four accesses of eight per lane
constexpr int LANES = 256;
constexpr int STEPS = UNIT / (LANES * VEC);
constexpr int GROUPS_PER_CU = 8;

struct Arrays {
    const void *src[MAX_ARRAYS];
    void *dst[MAX_ARRAYS];
    int64_t n[MAX_ARRAYS];
    int64_t first[MAX_ARRAYS + 1];      // first unit of an array; first[count] = units of the launch
    unsigned char types[MAX_ARRAYS];    // bit 0: src is fp32, bit 1: dst is fp32
    int count;
};
static_assert(sizeof(Arrays) <= 4000, "fits a kernel's arguments");

// The array that unit `u` belongs to (the same for all lanes).  Arrays without elements own no unit.
__device__ __forceinline__ int array_of(const Arrays &a, int64_t u)
{
    int lo = 0, hi = a.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (a.first[mid] <= u) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

template <typename T> __device__ __forceinline__ double squares(const void *base, int64_t n, int64_t start, double sum)
{
    const T *src = static_cast<const T *>(base);
    if (start + UNIT <= n) {
        Pack8<T> v[STEPS];
#pragma unroll
        for (int s = 0; s < STEPS; ++s) v[s] = *reinterpret_cast<const Pack8<T> *>(src + start + (s * LANES + (int)threadIdx.x) * VEC);
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const double x = to_f32<T>(v[s].v[e]);
                sum = fma(x, x, sum);
            }
    } else {
        for (int64_t i = start + threadIdx.x; i < n; i += LANES) {
            const double x = to_f32<T>(src[i]);
            sum = fma(x, x, sum);
        }
    }
    return sum;
}

// Sum over the workgroup, the same order always; valid in thread 0.
template <int THREADS> __device__ __forceinline__ double block_sum(double x, double *lds)
{
#pragma unroll
    for (int d = 32; d > 0; d /= 2) x += __shfl_down(x, d);
    if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = x;
    __syncthreads();
    if (threadIdx.x == 0)
        for (int w = 1; w < THREADS / 64; ++w) x += lds[w];
    return x;
}

__global__ __launch_bounds__(LANES) void grad_squares_kernel(const Arrays a, double *__restrict__ partials)
{
    __shared__ double lds[LANES / 64];
    double sum = 0;
    for (int64_t u = blockIdx.x; u < a.first[a.count]; u += gridDim.x) {
        const int t = array_of(a, u);
        const int64_t start = (u - a.first[t]) * UNIT;
        if (a.types[t] & 1) sum = squares<float>(a.src[t], a.n[t], start, sum);
        else sum = squares<unsigned short>(a.src[t], a.n[t], start, sum);
    }
    sum = block_sum<LANES>(sum, lds);
    if (threadIdx.x == 0) partials[blockIdx.x] = sum;
}

constexpr int FINISH_LANES = 1024;

__global__ __launch_bounds__(FINISH_LANES) void grad_norm_finish_kernel(const double *__restrict__ partials, int n, double scale,
                                                                        double *__restrict__ sumsq, float *__restrict__ norm)
{
    __shared__ double lds[FINISH_LANES / 64];
    double sum = 0;
    for (int i = threadIdx.x; i < n; i += FINISH_LANES) sum += partials[i];
    sum = block_sum<FINISH_LANES>(sum, lds);
    if (threadIdx.x == 0) {
        *sumsq = sum;
        if (norm) *norm = (float)(scale * sqrt(sum));
    }
}

template <typename TS, typename TD>
__device__ __forceinline__ void scale_unit(const void *from, void *to, int64_t n, int64_t start, float f)
{
    const TS *src = static_cast<const TS *>(from);
    TD *dst = static_cast<TD *>(to);
    if (start + UNIT <= n) {
        Pack8<TS> v[STEPS];
#pragma unroll
        for (int s = 0; s < STEPS; ++s) v[s] = *reinterpret_cast<const Pack8<TS> *>(src + start + (s * LANES + (int)threadIdx.x) * VEC);
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            float x[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) x[e] = to_f32<TS>(v[s].v[e]) * f;
            *reinterpret_cast<Pack8<TD> *>(dst + start + (s * LANES + (int)threadIdx.x) * VEC) = pack_out<TD>(x);
        }
    } else {
        for (int64_t i = start + threadIdx.x; i < n; i += LANES) dst[i] = from_f32<TD>(to_f32<TS>(src[i]) * f);
    }
}

__global__ __launch_bounds__(LANES) void grad_clip_kernel(const Arrays a, double scale, double max_norm, const double *__restrict__ sumsq)
{
    // (the same few operations in every lane, so that no launch is needed for one number)
    // A norm is finite where grad_norm_finish_kernel's fp32 value is: the caller sees there what is done here.
    const double norm = scale * sqrt(*sumsq);
    const float f = (float)(norm > max_norm && (float)norm < __builtin_huge_valf() ? scale * (max_norm / norm) : scale);
    for (int64_t u = blockIdx.x; u < a.first[a.count]; u += gridDim.x) {
        const int t = array_of(a, u);
        if (f == 1.f && a.src[t] == a.dst[t]) continue;
        const int64_t start = (u - a.first[t]) * UNIT;
        switch (a.types[t]) {
        case 0: scale_unit<unsigned short, unsigned short>(a.src[t], a.dst[t], a.n[t], start, f); break;
        case 1: scale_unit<float, unsigned short>(a.src[t], a.dst[t], a.n[t], start, f); break;
        case 2: scale_unit<unsigned short, float>(a.src[t], a.dst[t], a.n[t], start, f); break;
        default: scale_unit<float, float>(a.src[t], a.dst[t], a.n[t], start, f); break;
        }
    }
}

// Arrays `at` ... of the list, as many as a launch takes; returns how many.
int fill(Arrays *a, const cube3d_tensor *src, const cube3d_tensor *dst, int at, int count)
{
    int k = 0;
    int64_t units = 0;
    for (; k < MAX_ARRAYS && at + k < count; ++k) {
        const cube3d_tensor &s = src[at + k];
        a->src[k] = s.data;
        a->dst[k] = dst ? dst[at + k].data : nullptr;
        a->n[k] = s.n;
        a->types[k] = (unsigned char)((s.dtype == CUBE3D_F32 ? 1 : 0) | (dst && dst[at + k].dtype == CUBE3D_F32 ? 2 : 0));
        a->first[k] = units;
        units += (s.n + UNIT - 1) / UNIT;
    }
    a->first[k] = units;
    a->count = k;
    return k;
}

// (a pure function of the sizes and the device, so that the workspace query and the launches agree)
unsigned groups(int64_t units)
{
    const int64_t most = (int64_t)num_compute_units() * GROUPS_PER_CU;
    return (unsigned)(units < most ? units : most);
}

}  // namespace

int64_t grad_norm_partials(const cube3d_tensor *grads, int count)
{
    int64_t total = 0;
    for (int at = 0; at < count; at += MAX_ARRAYS) {
        int64_t units = 0;
        for (int k = at; k < count && k < at + MAX_ARRAYS; ++k) units += (grads[k].n + UNIT - 1) / UNIT;
        total += groups(units);
    }
    return total;
}

int grad_norm(const cube3d_tensor *grads, int count, float scale, double *sumsq, float *norm, double *partials, hipStream_t stream)
{
    int done = 0;
    for (int at = 0; at < count;) {
        Arrays a;
        at += fill(&a, grads, nullptr, at, count);
        const unsigned grid = groups(a.first[a.count]);
        if (grid == 0) continue;
        hipLaunchKernelGGL(grad_squares_kernel, dim3(grid), dim3(LANES), 0, stream, a, partials + done);
        if (const int rc = launch_status(); rc != CUBE3D_OK) return rc;
        done += (int)grid;
    }
    hipLaunchKernelGGL(grad_norm_finish_kernel, dim3(1), dim3(FINISH_LANES), 0, stream, partials, done, (double)scale, sumsq, norm);
    return launch_status();
}

int grad_clip(const cube3d_tensor *grads, const cube3d_tensor *out, int count, float scale, float max_norm, const double *sumsq,
              hipStream_t stream)
{
    for (int at = 0; at < count;) {
        Arrays a;
        at += fill(&a, grads, out, at, count);
        const unsigned grid = groups(a.first[a.count]);
        if (grid == 0) continue;
        hipLaunchKernelGGL(grad_clip_kernel, dim3(grid), dim3(LANES), 0, stream, a, (double)scale, (double)max_norm, sumsq);
        if (const int rc = launch_status(); rc != CUBE3D_OK) return rc;
    }
    return CUBE3D_OK;
}

int check_clip_overlap(const cube3d_tensor *grads, const cube3d_tensor *out, int count)
{
    struct Range {
        uintptr_t begin, end;
        int index;      // of a gradient, or ~index of a result
        bool operator<(const Range &o) const { return begin < o.begin; }
    };
    if (count == 0) return CUBE3D_OK;
    Range *r = new (std::nothrow) Range[2 * (size_t)count];
    if (!r) return CUBE3D_ELAUNCH;
    size_t n = 0;
    for (int k = 0; k < count; ++k) {
        if (grads[k].n == 0) continue;
        const int64_t se = grads[k].dtype == CUBE3D_F32 ? 4 : 2, de = out[k].dtype == CUBE3D_F32 ? 4 : 2;
        const uintptr_t s = (uintptr_t)grads[k].data, d = (uintptr_t)out[k].data;
        r[n++] = Range{d, d + (uintptr_t)(out[k].n * de), ~k};
        if (s != d || se != de) r[n++] = Range{s, s + (uintptr_t)(grads[k].n * se), k};
    }
    std::sort(r, r + n);
    // in ascending order of the begins, a result may not begin before what lies behind it has ended, nor anything inside a result
    int rc = CUBE3D_OK;
    uintptr_t end_all = 0, end_out = 0;
    for (size_t i = 0; i < n && rc == CUBE3D_OK; ++i) {
        const bool is_out = r[i].index < 0;
        if (r[i].begin < end_out || (is_out && r[i].begin < end_all)) rc = CUBE3D_EINVAL;
        if (r[i].end > end_all) end_all = r[i].end;
        if (is_out && r[i].end > end_out) end_out = r[i].end;
    }
    // (equal begins: whichever comes first, the second one lies inside it)
    delete[] r;
    return rc;
}

}  // namespace cube3d
