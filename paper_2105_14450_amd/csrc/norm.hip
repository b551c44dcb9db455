// The norms on either side of a block with the gate, the residual scale and the residual sum between them (Section 3.2), on
// matrices in the storage of activations, forward and backward:
//   forward    v = Npost(u),  r = x + s g v,  n = Npre(r)
//   backward   Dr = dr + Npre'(dn),  dx = Dr,  du = Npost'(s g Dr),  and the column sums of the parameters' gradients
// with N(t) = (t - mean) rstd gamma + beta over a row and, for t = dn gamma and r^ = (r - mean) rstd,
//   Npre'(dn) = rstd (t - mean(t) - r^ mean(t r^))        (mean(t) for LAYER only).
//
// A row's columns lie in q blocks, q * Ri processors apart: row and column offsets come from index maps, so that the rows of
// the whole cube are one matrix here.
#include "activation.h"

namespace cube3d {

namespace {

// ---- any size: one workgroup per row, the row read again for every step ---------------------------------

constexpr int ROW_LANES = 256;

// Sums of K values over the workgroup, in all lanes.  `slot` alternates from call to call: what one call left in LDS is read
// until the next one's barrier, and overwritten behind that.
template <int K, int THREADS> __device__ __forceinline__ void row_sum(float (&x)[K], float (*lds)[THREADS / 64 * 4], int &slot)
{
    slot ^= 1;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int d = 32; d > 0; d /= 2) x[k] += __shfl_xor(x[k], d);
    float *s = lds[slot];
    if (threadIdx.x % 64 == 0)
#pragma unroll
        for (int k = 0; k < K; ++k) s[threadIdx.x / 64 * 4 + k] = x[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
        x[k] = s[k];
#pragma unroll
        for (int w = 1; w < THREADS / 64; ++w) x[k] += s[4 * w + k];
    }
}

__device__ __forceinline__ float vector_at(const float *v, const AxisMap &m, int c, float absent)
{
    return v ? v[axis_offset_fast(m, c)] : absent;
}

template <typename TS, typename TB> __global__ __launch_bounds__(ROW_LANES) void norm_fwd_rows_kernel(const NormArgs a)
{
    __shared__ float lds[2][ROW_LANES / 64 * 4];
    const TS *x = static_cast<const TS *>(a.x);
    const TB *u = static_cast<const TB *>(a.u);
    TS *r = static_cast<TS *>(a.r_out);
    TB *n = static_cast<TB *>(a.n_out);
    const float inv = 1.f / (float)a.cols;
    int slot = 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const int64_t at = axis_offset_fast(a.row, row);
        float post_mean = 0.f, post_rstd = 0.f, pre_mean = 0.f, pre_rstd = 0.f;
        if (a.post_kind != CUBE3D_NORM_NONE) {
            float s[1] = {0.f};
            if (a.post_kind == CUBE3D_NORM_LAYER) {
                for (int c = threadIdx.x; c < a.cols; c += ROW_LANES) s[0] += to_f32<TB>(u[at + axis_offset_fast(a.col, c)]);
                row_sum<1, ROW_LANES>(s, lds, slot);
                post_mean = s[0] * inv;
                s[0] = 0.f;
            }
            for (int c = threadIdx.x; c < a.cols; c += ROW_LANES) {
                const float d = to_f32<TB>(u[at + axis_offset_fast(a.col, c)]) - post_mean;
                s[0] = fmaf(d, d, s[0]);
            }
            row_sum<1, ROW_LANES>(s, lds, slot);
            post_rstd = 1.f / sqrtf(s[0] * inv + a.post_eps);
        }
        // r of one column, in fp32
        auto stream = [&](int c, int64_t i) {
            const float xv = to_f32<TS>(x[i]);
            if (!a.u) return xv;
            float v = to_f32<TB>(u[i]);
            if (a.post_kind != CUBE3D_NORM_NONE)
                v = (v - post_mean) * post_rstd * vector_at(a.p.post_gamma, a.vec, c, 1.f) + vector_at(a.p.post_beta, a.vec, c, 0.f);
            return xv + a.scale * vector_at(a.p.gate, a.vec, c, 1.f) * v;
        };
        if (a.pre_kind != CUBE3D_NORM_NONE) {
            float s[1] = {0.f};
            if (a.pre_kind == CUBE3D_NORM_LAYER) {
                for (int c = threadIdx.x; c < a.cols; c += ROW_LANES) s[0] += stream(c, at + axis_offset_fast(a.col, c));
                row_sum<1, ROW_LANES>(s, lds, slot);
                pre_mean = s[0] * inv;
                s[0] = 0.f;
            }
            for (int c = threadIdx.x; c < a.cols; c += ROW_LANES) {
                const float d = stream(c, at + axis_offset_fast(a.col, c)) - pre_mean;
                s[0] = fmaf(d, d, s[0]);
            }
            row_sum<1, ROW_LANES>(s, lds, slot);
            pre_rstd = 1.f / sqrtf(s[0] * inv + a.pre_eps);
        }
        for (int c = threadIdx.x; c < a.cols; c += ROW_LANES) {
            const int64_t i = at + axis_offset_fast(a.col, c);
            const float v = stream(c, i);
            if (n) n[i] = from_f32<TB>((v - pre_mean) * pre_rstd * vector_at(a.p.pre_gamma, a.vec, c, 1.f) +
                                       vector_at(a.p.pre_beta, a.vec, c, 0.f));
            if (r) r[i] = from_f32<TS>(v);      // (behind the last read of x: r may be x)
        }
        if (a.stats_out && threadIdx.x == 0)
            *reinterpret_cast<f32x4 *>(a.stats_out + 4 * row) = f32x4{post_mean, post_rstd, pre_mean, pre_rstd};
    }
}

// What a column of the backward pass is made of.  (m1, m2: mean(t) and mean(t r^) of the norm ahead of the next block, m3, m4 of
// the norm behind the block.)
struct ColumnParams {
    float post_gamma, post_beta, gate, pre_gamma;
};

__device__ __forceinline__ ColumnParams column_params(const NormArgs &a, int c)
{
    return ColumnParams{vector_at(a.p.post_gamma, a.vec, c, 1.f), vector_at(a.p.post_beta, a.vec, c, 0.f),
                        vector_at(a.p.gate, a.vec, c, 1.f), vector_at(a.p.pre_gamma, a.vec, c, 1.f)};
}

// Row sums of the backward pass: scalars[row] = mean(t), mean(t r^), mean(tp), mean(tp u^)
template <typename TS, typename TB> __global__ __launch_bounds__(ROW_LANES) void norm_bwd_rows_kernel(const NormArgs a, float *__restrict__ scalars)
{
    __shared__ float lds[2][ROW_LANES / 64 * 4];
    const TS *dr = static_cast<const TS *>(a.dr), *r = static_cast<const TS *>(a.x);
    const TB *dn = static_cast<const TB *>(a.dn), *u = static_cast<const TB *>(a.u);
    const float inv = 1.f / (float)a.cols;
    int slot = 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const int64_t at = axis_offset_fast(a.row, row);
        const f32x4 st = *reinterpret_cast<const f32x4 *>(a.stats + 4 * row);
        float m[2] = {0.f, 0.f}, mp[2] = {0.f, 0.f};
        if (a.pre_kind != CUBE3D_NORM_NONE) {
            for (int c = threadIdx.x; c < a.cols; c += ROW_LANES) {
                const int64_t i = at + axis_offset_fast(a.col, c);
                const float t = to_f32<TB>(dn[i]) * vector_at(a.p.pre_gamma, a.vec, c, 1.f), hat = (to_f32<TS>(r[i]) - st[2]) * st[3];
                m[0] += t;
                m[1] = fmaf(t, hat, m[1]);
            }
            row_sum<2, ROW_LANES>(m, lds, slot);
            m[0] = a.pre_kind == CUBE3D_NORM_LAYER ? m[0] * inv : 0.f;
            m[1] *= inv;
        }
        if (a.post_kind != CUBE3D_NORM_NONE) {
            for (int c = threadIdx.x; c < a.cols; c += ROW_LANES) {
                const int64_t i = at + axis_offset_fast(a.col, c);
                const ColumnParams p = column_params(a, c);
                float g = dr ? to_f32<TS>(dr[i]) : 0.f;
                if (a.pre_kind != CUBE3D_NORM_NONE)
                    g += st[3] * (to_f32<TB>(dn[i]) * p.pre_gamma - m[0] - (to_f32<TS>(r[i]) - st[2]) * st[3] * m[1]);
                const float t = a.scale * p.gate * g * p.post_gamma, hat = (to_f32<TB>(u[i]) - st[0]) * st[1];
                mp[0] += t;
                mp[1] = fmaf(t, hat, mp[1]);
            }
            row_sum<2, ROW_LANES>(mp, lds, slot);
            mp[0] = a.post_kind == CUBE3D_NORM_LAYER ? mp[0] * inv : 0.f;
            mp[1] *= inv;
        }
        if (threadIdx.x == 0) *reinterpret_cast<f32x4 *>(scalars + 4 * row) = f32x4{m[0], m[1], mp[0], mp[1]};
    }
}

// Everything that remains is element-wise but for the column sums: a workgroup takes 64 columns of a group of rows, a lane
// one column of every fourth row, and leaves partial sums [group][vector][column].
constexpr int VECTORS = 5;      // post_gamma, post_beta, gate, pre_gamma, pre_beta
template <typename TS, typename TB>
__global__ __launch_bounds__(256) void norm_bwd_columns_kernel(const NormArgs a, const float *__restrict__ scalars, float *__restrict__ partials,
                                                               int rows_per_group)
{
    __shared__ float lds[4][VECTORS][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, c = blockIdx.x * 64 + lane;
    const bool live = c < a.cols;
    const int64_t col = live ? axis_offset_fast(a.col, c) : 0;
    const ColumnParams p = live ? column_params(a, c) : ColumnParams{0.f, 0.f, 0.f, 0.f};
    const TS *dr = static_cast<const TS *>(a.dr), *r = static_cast<const TS *>(a.x);
    const TB *dn = static_cast<const TB *>(a.dn), *u = static_cast<const TB *>(a.u);
    TS *dx = static_cast<TS *>(a.dx);
    TB *du = static_cast<TB *>(a.du);
    const bool pre = a.pre_kind != CUBE3D_NORM_NONE, post = a.post_kind != CUBE3D_NORM_NONE;
    float sum[VECTORS] = {0.f, 0.f, 0.f, 0.f, 0.f};
    const int64_t first = (int64_t)blockIdx.y * rows_per_group, last = min(first + rows_per_group, a.rows);
    for (int64_t row = first + wave; row < last && live; row += 4) {
        const int64_t i = axis_offset_fast(a.row, row) + col;
        const f32x4 none = {0.f, 0.f, 0.f, 0.f};
        const f32x4 st = pre || post ? *reinterpret_cast<const f32x4 *>(a.stats + 4 * row) : none;
        const f32x4 m = pre || post ? *reinterpret_cast<const f32x4 *>(scalars + 4 * row) : none;
        float g = dr ? to_f32<TS>(dr[i]) : 0.f;
        if (pre) {
            const float d = to_f32<TB>(dn[i]), hat = (to_f32<TS>(r[i]) - st[2]) * st[3];
            sum[3] = fmaf(d, hat, sum[3]);
            sum[4] += d;
            g += st[3] * (d * p.pre_gamma - m[0] - hat * m[1]);
        }
        if (dx) dx[i] = from_f32<TS>(g);
        g *= a.scale;
        if (post) {
            const float hat = (to_f32<TB>(u[i]) - st[0]) * st[1];
            sum[2] = fmaf(g, hat * p.post_gamma + p.post_beta, sum[2]);
            g *= p.gate;
            sum[0] = fmaf(g, hat, sum[0]);
            sum[1] += g;
            g = st[1] * (g * p.post_gamma - m[2] - hat * m[3]);
        } else {
            if (a.read_u) sum[2] = fmaf(g, to_f32<TB>(u[i]), sum[2]);
            g *= p.gate;
        }
        if (du) du[i] = from_f32<TB>(g);
    }
#pragma unroll
    for (int v = 0; v < VECTORS; ++v) lds[wave][v][lane] = sum[v];
    __syncthreads();
    if (!a.sums || !live) return;
    for (int v = wave; v < VECTORS; v += 4)
        partials[((int64_t)blockIdx.y * VECTORS + v) * a.cols + c] = ((lds[0][v][lane] + lds[1][v][lane]) + lds[2][v][lane]) + lds[3][v][lane];
}

// The groups' partial sums of one vector, in ascending order, to its diagonal storage (zeros off the diagonal).  A workgroup takes
// 64 of the Cs columns of a processor, its wavefronts runs of the groups.
constexpr int FINISH_WAVES = 16;
__global__ __launch_bounds__(64 * FINISH_WAVES) void norm_bwd_finish_kernel(const NormArgs a, const float *__restrict__ partials, int groups,
                                                                            cube3d_norm_params out)
{
    __shared__ float lds[FINISH_WAVES][64];
    float *const vectors[VECTORS] = {out.post_gamma, out.post_beta, out.gate, out.pre_gamma, out.pre_beta};
    float *dst = vectors[0];
#pragma unroll
    for (int v = 1; v < VECTORS; ++v)
        if ((int)blockIdx.z == v) dst = vectors[v];
    if (!dst) return;
    const int q = a.q, Cs = a.vec.P2, lane = threadIdx.x % 64, wave = threadIdx.x / 64, x = blockIdx.x * 64 + lane;
    const int proc = blockIdx.y, l = proc % q, j = proc / q % q, i = proc / (q * q);
    const bool live = x < Cs;
    if (j != l) {
        if (wave == 0 && live) dst[(int64_t)proc * Cs + x] = 0.f;
        return;
    }
    const int c = j * (q * Cs) + i * Cs + x;
    const int per = (groups + FINISH_WAVES - 1) / FINISH_WAVES, lo = min(wave * per, groups), hi = min(lo + per, groups);
    float sum = 0.f;
    if (live)
        for (int g = lo; g < hi; ++g) sum += partials[((int64_t)g * VECTORS + blockIdx.z) * a.cols + c];
    lds[wave][lane] = sum;
    __syncthreads();
    if (wave == 0 && live) {
#pragma unroll
        for (int w = 1; w < FINISH_WAVES; ++w) sum += lds[w][lane];
        dst[(int64_t)proc * Cs + x] = sum;
    }
}

// Rows per workgroup of the column pass: enough workgroups for every CU, few enough partial sums.
int rows_per_group(const NormArgs &a)
{
    const int64_t tiles = (a.cols + 63) / 64;
    int64_t rows = 256;
    while (rows > 16 && tiles * ((a.rows + rows - 1) / rows) < 4096) rows /= 2;
    while ((a.rows + rows - 1) / rows > 32768) rows *= 2;
    return (int)rows;
}

template <typename F> int by_types(const NormArgs &a, F &&f)
{
    const bool s = a.stream_f32, b = a.block_f32;
    if (s) return b ? f(float{}, float{}) : f(float{}, (unsigned short)0);
    return b ? f((unsigned short)0, float{}) : f((unsigned short)0, (unsigned short)0);
}

unsigned row_grid(int64_t rows)
{
    const int64_t most = (int64_t)num_compute_units() * 8;
    return (unsigned)(rows < most ? rows : most);
}

}  // namespace

int norm_fwd(const NormArgs &a, hipStream_t stream)
{
    return by_types(a, [&](auto s, auto b) {
        hipLaunchKernelGGL((norm_fwd_rows_kernel<decltype(s), decltype(b)>), dim3(row_grid(a.rows)), dim3(ROW_LANES), 0, stream, a);
        return launch_status();
    });
}

size_t norm_bwd_workspace(const NormArgs &a)
{
    const int64_t per = rows_per_group(a), groups = (a.rows + per - 1) / per;
    return ((size_t)a.rows * 4 + (size_t)groups * VECTORS * a.cols) * sizeof(float);
}

int norm_bwd(const NormArgs &a, const cube3d_norm_params &gradients, void *workspace, hipStream_t stream)
{
    float *scalars = static_cast<float *>(workspace), *partials = scalars + a.rows * 4;
    const int per = rows_per_group(a);
    const unsigned groups = (unsigned)((a.rows + per - 1) / per);
    const int rc = by_types(a, [&](auto s, auto b) {
        typedef decltype(s) TS;
        typedef decltype(b) TB;
        if (a.pre_kind != CUBE3D_NORM_NONE || a.post_kind != CUBE3D_NORM_NONE)
            hipLaunchKernelGGL((norm_bwd_rows_kernel<TS, TB>), dim3(row_grid(a.rows)), dim3(ROW_LANES), 0, stream, a, scalars);
        if (const int e = launch_status(); e != CUBE3D_OK) return e;
        hipLaunchKernelGGL((norm_bwd_columns_kernel<TS, TB>), dim3((unsigned)((a.cols + 63) / 64), groups), dim3(256), 0, stream, a,
                           scalars, partials, per);
        return launch_status();
    });
    if (rc != CUBE3D_OK || !a.sums) return rc;
    const unsigned q3 = (unsigned)(a.q * a.q * a.q);
    hipLaunchKernelGGL(norm_bwd_finish_kernel, dim3((unsigned)((a.vec.P2 + 63) / 64), q3, VECTORS), dim3(64 * FINISH_WAVES), 0, stream, a,
                       partials, (int)groups, gradients);
    return launch_status();
}

}  // namespace cube3d
