// The norms on either side of a block with the gate, the residual scale and the residual sum between them (Section 3.2), on
// matrices in the storage of activations, forward and backward:
//   forward    v = Npost(u),  r = x + s g v,  n = Npre(r)
//   backward   Dr = dr + Npre'(dn),  dx = Dr,  du = Npost'(s g Dr),  and the column sums of the parameters' gradients
// with N(t) = (t - mean) rstd gamma + beta over a row and, for t = dn gamma and r^ = (r - mean) rstd,
//   Npre'(dn) = rstd (t - mean(t) - r^ mean(t r^))        (mean(t) for LAYER only).
//
// A row's columns lie in q blocks, q * Ri processors apart: row and column offsets come from index maps, so that the rows of
// the whole cube are one matrix here.
#include <type_traits>

#include "activation.h"

namespace cube3d {

namespace {

constexpr int VECTORS = 5;      // post_gamma, post_beta, gate, pre_gamma, pre_beta

// ---- any size: one workgroup per row, the row read again for every step ---------------------------------
// For what registers do not hold.  V consecutive columns at a time: eight where they lie side by side in every array, else four, two or
// one.  Bound by the latency of narrow loads and of the passes over a row, of which a forward pass makes up to four.

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

template <typename T, int V> struct __attribute__((aligned(sizeof(T) * V))) Columns {
    T v[V];
};

template <typename T, int V> __device__ __forceinline__ void get(const T *from, int64_t at, float (&x)[V])
{
    const Columns<T, V> c = *reinterpret_cast<const Columns<T, V> *>(from + at);
#pragma unroll
    for (int e = 0; e < V; ++e) x[e] = to_f32<T>(c.v[e]);
}
template <typename T, int V> __device__ __forceinline__ void put(T *to, int64_t at, const float (&x)[V])
{
    Columns<T, V> c;
#pragma unroll
    for (int e = 0; e < V; ++e) c.v[e] = from_f32<T>(x[e]);
    *reinterpret_cast<Columns<T, V> *>(to + at) = c;
}
// V elements of a vector in diagonal storage
template <int V> __device__ __forceinline__ void vector_at(const float *v, int64_t at, float absent, float (&x)[V])
{
    if (v) get<float, V>(v, at, x);
    else
#pragma unroll
        for (int e = 0; e < V; ++e) x[e] = absent;
}

template <typename TS, typename TB, int V, int LANES> __global__ __launch_bounds__(LANES) void norm_fwd_rows_kernel(const NormArgs a)
{
    __shared__ float lds[2][LANES / 64 * 4];
    const TS *x = static_cast<const TS *>(a.x);
    const TB *u = static_cast<const TB *>(a.u);
    TS *r = static_cast<TS *>(a.r_out);
    TB *n = static_cast<TB *>(a.n_out);
    const float inv = 1.f / (float)a.cols;
    int slot = 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const int64_t at = axis_offset_fast(a.row, row);
        float post_mean = 0.f, post_rstd = 0.f, pre_mean = 0.f, pre_rstd = 0.f;
        // sum over the row of f(value), f of V columns at a time
        auto total = [&](auto &&values, auto &&f) {
            float s[1] = {0.f};
            for (int c = threadIdx.x * V; c < a.cols; c += LANES * V) {
                float v[V];
                values(c, at + axis_offset_fast(a.col, c), v);
#pragma unroll
                for (int e = 0; e < V; ++e) s[0] += f(v[e]);
            }
            row_sum<1, LANES>(s, lds, slot);
            return s[0];
        };
        if (a.post_kind != CUBE3D_NORM_NONE) {
            auto block = [&](int, int64_t i, float (&v)[V]) { get<TB, V>(u, i, v); };
            if (a.post_kind == CUBE3D_NORM_LAYER) post_mean = total(block, [](float v) { return v; }) * inv;
            post_rstd = 1.f / sqrtf(total(block, [&](float v) { return (v - post_mean) * (v - post_mean); }) * inv + a.post_eps);
        }
        // r of V columns, in fp32
        auto stream = [&](int c, int64_t i, float (&v)[V]) {
            get<TS, V>(x, i, v);
            if (!a.u) return;
            const int64_t vec = axis_offset_fast(a.vec, c);
            float w[V], gate[V];
            get<TB, V>(u, i, w);
            if (a.post_kind != CUBE3D_NORM_NONE) {
                float gamma[V], beta[V];
                vector_at<V>(a.p.post_gamma, vec, 1.f, gamma);
                vector_at<V>(a.p.post_beta, vec, 0.f, beta);
#pragma unroll
                for (int e = 0; e < V; ++e) w[e] = (w[e] - post_mean) * post_rstd * gamma[e] + beta[e];
            }
            vector_at<V>(a.p.gate, vec, 1.f, gate);
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] += a.scale * gate[e] * w[e];
        };
        if (a.pre_kind != CUBE3D_NORM_NONE) {
            if (a.pre_kind == CUBE3D_NORM_LAYER) pre_mean = total(stream, [](float v) { return v; }) * inv;
            pre_rstd = 1.f / sqrtf(total(stream, [&](float v) { return (v - pre_mean) * (v - pre_mean); }) * inv + a.pre_eps);
        }
        for (int c = threadIdx.x * V; c < a.cols; c += LANES * V) {
            const int64_t i = at + axis_offset_fast(a.col, c);
            float v[V];
            stream(c, i, v);
            if (n) {
                const int64_t vec = axis_offset_fast(a.vec, c);
                float y[V], gamma[V], beta[V];
                vector_at<V>(a.p.pre_gamma, vec, 1.f, gamma);
                vector_at<V>(a.p.pre_beta, vec, 0.f, beta);
#pragma unroll
                for (int e = 0; e < V; ++e) y[e] = (v[e] - pre_mean) * pre_rstd * gamma[e] + beta[e];
                put<TB, V>(n, i, y);
            }
            if (r) put<TS, V>(r, i, v);      // (behind the last read of x: r may be x)
        }
        if (a.stats_out && threadIdx.x == 0)
            *reinterpret_cast<f32x4 *>(a.stats_out + 4 * row) = f32x4{post_mean, post_rstd, pre_mean, pre_rstd};
    }
}

// What V columns of the backward pass are multiplied with.
template <int V> struct ColumnParams {
    float post_gamma[V], post_beta[V], gate[V], pre_gamma[V];
    __device__ __forceinline__ void look_up(const NormArgs &a, int c)
    {
        const int64_t vec = axis_offset_fast(a.vec, c);
        vector_at<V>(a.p.post_gamma, vec, 1.f, post_gamma);
        vector_at<V>(a.p.post_beta, vec, 0.f, post_beta);
        vector_at<V>(a.p.gate, vec, 1.f, gate);
        vector_at<V>(a.p.pre_gamma, vec, 1.f, pre_gamma);
    }
};

// Row sums of the backward pass: scalars[row] = mean(t), mean(t r^), mean(tp), mean(tp u^)
template <typename TS, typename TB, int V, int LANES>
__global__ __launch_bounds__(LANES) void norm_bwd_rows_kernel(const NormArgs a, float *__restrict__ scalars)
{
    __shared__ float lds[2][LANES / 64 * 4];
    const TS *dr = static_cast<const TS *>(a.dr), *r = static_cast<const TS *>(a.x);
    const TB *dn = static_cast<const TB *>(a.dn), *u = static_cast<const TB *>(a.u);
    const bool pre = a.pre_kind != CUBE3D_NORM_NONE;
    const float inv = 1.f / (float)a.cols;
    int slot = 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const int64_t at = axis_offset_fast(a.row, row);
        const f32x4 st = *reinterpret_cast<const f32x4 *>(a.stats + 4 * row);
        float m[2] = {0.f, 0.f}, mp[2] = {0.f, 0.f};
        if (pre) {
            for (int c = threadIdx.x * V; c < a.cols; c += LANES * V) {
                const int64_t i = at + axis_offset_fast(a.col, c);
                float t[V], hat[V], gamma[V];
                get<TB, V>(dn, i, t);
                get<TS, V>(r, i, hat);
                vector_at<V>(a.p.pre_gamma, axis_offset_fast(a.vec, c), 1.f, gamma);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    t[e] *= gamma[e];
                    m[0] += t[e];
                    m[1] = fmaf(t[e], (hat[e] - st[2]) * st[3], m[1]);
                }
            }
            row_sum<2, LANES>(m, lds, slot);
            m[0] = a.pre_kind == CUBE3D_NORM_LAYER ? m[0] * inv : 0.f;
            m[1] *= inv;
        }
        if (a.post_kind != CUBE3D_NORM_NONE) {
            for (int c = threadIdx.x * V; c < a.cols; c += LANES * V) {
                const int64_t i = at + axis_offset_fast(a.col, c);
                ColumnParams<V> p;
                p.look_up(a, c);
                float g[V], t[V], hat[V], w[V];
                if (dr) get<TS, V>(dr, i, g);
                else
#pragma unroll
                    for (int e = 0; e < V; ++e) g[e] = 0.f;
                if (pre) {
                    get<TB, V>(dn, i, t);
                    get<TS, V>(r, i, hat);
#pragma unroll
                    for (int e = 0; e < V; ++e) g[e] += st[3] * (t[e] * p.pre_gamma[e] - m[0] - (hat[e] - st[2]) * st[3] * m[1]);
                }
                get<TB, V>(u, i, w);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float tp = a.scale * p.gate[e] * g[e] * p.post_gamma[e];
                    mp[0] += tp;
                    mp[1] = fmaf(tp, (w[e] - st[0]) * st[1], mp[1]);
                }
            }
            row_sum<2, LANES>(mp, lds, slot);
            mp[0] = a.post_kind == CUBE3D_NORM_LAYER ? mp[0] * inv : 0.f;
            mp[1] *= inv;
        }
        if (threadIdx.x == 0) *reinterpret_cast<f32x4 *>(scalars + 4 * row) = f32x4{m[0], m[1], mp[0], mp[1]};
    }
}

// Everything that remains is element-wise but for the column sums: a workgroup takes 64 V columns of a group of rows, a lane V of
// every fourth row, and leaves partial sums [group][vector][column].  first_tile: of this launch (launch_in_parts).
template <typename TS, typename TB, int V>
__global__ __launch_bounds__(256) void norm_bwd_columns_kernel(const NormArgs a, const float *__restrict__ scalars, float *__restrict__ partials,
                                                               int rows_per_group, int wanted, int first_tile)
{
    __shared__ float lds[4][64 * V];
    const int tile = first_tile + blockIdx.x, lane = threadIdx.x % 64, wave = threadIdx.x / 64, c = (tile * 64 + lane) * V;
    const bool live = c < a.cols;
    const int64_t col = axis_offset_fast(a.col, live ? c : 0);
    ColumnParams<V> p;
    p.look_up(a, live ? c : 0);
    const TS *dr = static_cast<const TS *>(a.dr), *r = static_cast<const TS *>(a.x);
    const TB *dn = static_cast<const TB *>(a.dn), *u = static_cast<const TB *>(a.u);
    TS *dx = static_cast<TS *>(a.dx);
    TB *du = static_cast<TB *>(a.du);
    const bool pre = a.pre_kind != CUBE3D_NORM_NONE, post = a.post_kind != CUBE3D_NORM_NONE;
    float sum[VECTORS][V];
#pragma unroll
    for (int v = 0; v < VECTORS; ++v)
#pragma unroll
        for (int e = 0; e < V; ++e) sum[v][e] = 0.f;
    const int64_t first = (int64_t)blockIdx.y * rows_per_group, last = min(first + rows_per_group, a.rows);
    for (int64_t row = first + wave; row < last && live; row += 4) {
        const int64_t i = axis_offset_fast(a.row, row) + col;
        const f32x4 none = {0.f, 0.f, 0.f, 0.f};
        const f32x4 st = pre || post ? *reinterpret_cast<const f32x4 *>(a.stats + 4 * row) : none;
        const f32x4 m = pre || post ? *reinterpret_cast<const f32x4 *>(scalars + 4 * row) : none;
        float g[V], d[V], hat[V], w[V];
        if (dr) get<TS, V>(dr, i, g);
        else
#pragma unroll
            for (int e = 0; e < V; ++e) g[e] = 0.f;
        if (pre) {
            get<TB, V>(dn, i, d);
            get<TS, V>(r, i, hat);
        }
        if (post || a.read_u) get<TB, V>(u, i, w);
        if (pre) {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                hat[e] = (hat[e] - st[2]) * st[3];
                sum[3][e] = fmaf(d[e], hat[e], sum[3][e]);
                sum[4][e] += d[e];
                g[e] += st[3] * (d[e] * p.pre_gamma[e] - m[0] - hat[e] * m[1]);
            }
        }
        if (dx) put<TS, V>(dx, i, g);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            g[e] *= a.scale;
            if (post) {
                w[e] = (w[e] - st[0]) * st[1];
                sum[2][e] = fmaf(g[e], w[e] * p.post_gamma[e] + p.post_beta[e], sum[2][e]);
                g[e] *= p.gate[e];
                sum[0][e] = fmaf(g[e], w[e], sum[0][e]);
                sum[1][e] += g[e];
                g[e] = st[1] * (g[e] * p.post_gamma[e] - m[2] - w[e] * m[3]);
            } else {
                if (a.read_u) sum[2][e] = fmaf(g[e], w[e], sum[2][e]);
                g[e] *= p.gate[e];
            }
        }
        if (du) put<TB, V>(du, i, g);
    }
    if (!a.sums) return;
#pragma unroll
    for (int v = 0; v < VECTORS; ++v) {
        if (!(wanted >> v & 1)) continue;
        __syncthreads();
#pragma unroll
        for (int e = 0; e < V; ++e) lds[wave][e * 64 + lane] = sum[v][e];
        __syncthreads();
        for (int x = threadIdx.x; x < 64 * V; x += 256) {
            const int at = x % V * 64 + x / V, column = tile * 64 * V + x;
            if (column < a.cols)
                partials[((int64_t)blockIdx.y * VECTORS + v) * a.cols + column] = ((lds[0][at] + lds[1][at]) + lds[2][at]) + lds[3][at];
        }
    }
}

// The groups' partial sums of one vector, in ascending order, to its diagonal storage (zeros off the diagonal).  A workgroup takes
// 64 of the Cs columns of a processor, its wavefronts runs of the groups.  first_tile: of this launch.
constexpr int FINISH_WAVES = 16;
__global__ __launch_bounds__(64 * FINISH_WAVES) void norm_bwd_finish_kernel(const NormArgs a, const float *__restrict__ partials, int groups,
                                                                            cube3d_norm_params out, int first_tile)
{
    __shared__ float lds[FINISH_WAVES][64];
    float *const vectors[VECTORS] = {out.post_gamma, out.post_beta, out.gate, out.pre_gamma, out.pre_beta};
    float *dst = vectors[0];
#pragma unroll
    for (int v = 1; v < VECTORS; ++v)
        if ((int)blockIdx.z == v) dst = vectors[v];
    if (!dst) return;
    const int q = a.q, Cs = a.vec.P2, lane = threadIdx.x % 64, wave = threadIdx.x / 64, x = (first_tile + blockIdx.x) * 64 + lane;
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
#pragma unroll 8
        for (int g = lo; g < hi; ++g) sum += partials[((int64_t)g * VECTORS + blockIdx.z) * a.cols + c];
    lds[wave][lane] = sum;
    __syncthreads();
    if (wave == 0 && live) {
#pragma unroll
        for (int w = 1; w < FINISH_WAVES; ++w) sum += lds[w][lane];
        dst[(int64_t)proc * Cs + x] = sum;
    }
}

// ---- rows in registers ----------------------------------------------------------------------------------
// A row is held by `waves` wavefronts, eight columns times P a lane, and read once; short rows share a workgroup.  A lane keeps its
// columns from row to row: offsets and parameters are looked up once, the backward pass's column sums grow in registers, and the
// next row is on its way while the last one's sums are formed.
//
// Where eight consecutive columns lie side by side and aligned in every array (blocks and vector shards of a multiple of eight
// columns) every lane has eight.  Else (RAGGED) each vector shard is cut into runs of eight and a last one of what is left; whole runs
// still move in 16-byte accesses, which need no alignment.  us, forward / backward, here and in narrow accesses as above:
// 3000 x 4101 34 / 48 and 68 / 83, 20000 x 514 29 / 47 and 48 / 54, 3000 x 4001 with both norms and an fp32 stream 45 / 66 and
// 143 / 122, 32768 x 516 (q = 2) 64 / 139 and 274 / 288.  Runs of four are as fast there (3000 x 4100 31 / 48) and stay, and so does the
// backward pass of both norms with more than eight wavefronts a row (4000 x 6001: 395 us here with spills, 328).
//
// What bounds it: HBM.  TB/s of necessary bytes, forward / backward, a copy of 1 GiB making 4.8: 32768 x 8192 bf16 5.0 / 5.1;
// 8192 x 2048 (200 MB, in part from the Infinity Cache) 5.8 / 4.9; 16384 x 8192 with both norms and an fp32 stream 5.1 / 5.0;
// 16384 x 12288 5.6 / 5.0 (norm_bwd_long_kernel).  Row by row from memory, as above in single elements, the first was 1.0 / 1.7.

constexpr int SHORT_ROW = 512;          // columns of one wavefront

// Sum over the 64 lanes, in all of them, in a fixed order: within 16 lanes by exchanges inside the vector unit, then over the four rows.
__device__ __forceinline__ float lanes16_sum(float x)
{
    auto moved = [](float v, auto ctrl) {
        return __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), decltype(ctrl)::value, 0xf, 0xf, true));
    };
    x += moved(x, std::integral_constant<int, 0xb1>{});       // neighbours
    x += moved(x, std::integral_constant<int, 0x4e>{});       // pairs
    x += moved(x, std::integral_constant<int, 0x141>{});      // mirrored in eights
    x += moved(x, std::integral_constant<int, 0x140>{});      // mirrored in sixteens
    return x;
}
__device__ __forceinline__ float wave_sum(float x)
{
    x = lanes16_sum(x);
    const int i = (int)__float_as_uint(x);
    const float a = __uint_as_float((unsigned)__builtin_amdgcn_readlane(i, 0)), b = __uint_as_float((unsigned)__builtin_amdgcn_readlane(i, 16));
    const float c = __uint_as_float((unsigned)__builtin_amdgcn_readlane(i, 32)), d = __uint_as_float((unsigned)__builtin_amdgcn_readlane(i, 48));
    return (a + b) + (c + d);
}

// The wavefronts of one row: `waves` (at most 16) of them, the first of which is number `first` of the workgroup.
struct RowGroup {
    int waves, first, wave, lane;
    float (*lds)[2][16];        // [slot][value][wavefront], for the whole workgroup
    int slot;
};

// Sums of K values over a row, in all its lanes.  (All wavefronts of the workgroup call it together.)
template <int K> __device__ __forceinline__ void group_sum(RowGroup &g, float (&x)[K])
{
#pragma unroll
    for (int k = 0; k < K; ++k) x[k] = wave_sum(x[k]);
    if (g.waves == 1) return;
    g.slot ^= 1;        // (read until the next call's barrier, overwritten behind it)
    if (g.lane == 0)
#pragma unroll
        for (int k = 0; k < K; ++k) g.lds[g.slot][k][g.wave] = x[k];
    __syncthreads();
    const int l = g.lane % 16;
#pragma unroll
    for (int k = 0; k < K; ++k) x[k] = lanes16_sum(l < g.waves ? g.lds[g.slot][k][(g.first + l) % 16] : 0.f);
}

template <typename T> __device__ __forceinline__ void unpack(const Pack8<T> &v, float (&x)[VEC])
{
#pragma unroll
    for (int e = 0; e < VEC; ++e) x[e] = to_f32<T>(v.v[e]);
}

// Where a lane's columns begin, and how many there are: eight (0 beyond the row's end), or, RAGGED, eight of a vector's shard of Cs
// columns or what is left of it.  (Runs of a shard lie side by side in every array, at any alignment.)
struct Run {
    int c, valid;
};
template <bool RAGGED> __device__ __forceinline__ Run run_of(const NormArgs &a, int number)
{
    if constexpr (!RAGGED) return Run{number * VEC, number * VEC < a.cols ? VEC : 0};
    const int Cs = a.vec.P2, runs = (Cs + VEC - 1) / VEC, shard = number / runs, at = (number - shard * runs) * VEC;
    return Run{shard * Cs + at, shard < a.q * a.q ? min(Cs - at, VEC) : 0};
}

template <typename T> struct __attribute__((packed, aligned(sizeof(T)))) Loose8 {
    T v[VEC];
};
template <bool RAGGED, typename T> __device__ __forceinline__ Pack8<T> get_run(const T *from, int valid)
{
    if constexpr (!RAGGED) return *reinterpret_cast<const Pack8<T> *>(from);
    if (valid == VEC) return __builtin_bit_cast(Pack8<T>, *reinterpret_cast<const Loose8<T> *>(from));
    Pack8<T> x;
#pragma unroll
    for (int e = 0; e < VEC; ++e) x.v[e] = e < valid ? from[e] : T(0);
    return x;
}
template <bool RAGGED, typename T> __device__ __forceinline__ void put_run(T *to, int valid, const Pack8<T> &x)
{
    if constexpr (!RAGGED) {
        *reinterpret_cast<Pack8<T> *>(to) = x;
        return;
    }
    if (valid == VEC) {
        *reinterpret_cast<Loose8<T> *>(to) = __builtin_bit_cast(Loose8<T>, x);
        return;
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e)
        if (e < valid) to[e] = x.v[e];
}
template <bool RAGGED> __device__ __forceinline__ void vector_run(const float *v, int64_t at, int valid, float absent, float (&x)[VEC])
{
    if constexpr (!RAGGED) {
        vector_at<VEC>(v, at, absent, x);
        return;
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e) x[e] = v && e < valid ? v[at + e] : absent;
}

template <typename TS, typename TB, int P, bool RAGGED>
__global__ __launch_bounds__(1024) void norm_fwd_kernel(const NormArgs a, int waves, int rows_at_once)
{
    __shared__ float lds[2][2][16];
    RowGroup g;
    g.lane = threadIdx.x % 64;
    g.wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    g.waves = waves;
    const int group = g.wave / waves;
    g.first = group * waves;
    g.lds = lds;
    g.slot = 0;
    const TS *x = static_cast<const TS *>(a.x);
    const TB *u = static_cast<const TB *>(a.u);
    TS *r_out = static_cast<TS *>(a.r_out);
    TB *n_out = static_cast<TB *>(a.n_out);
    const bool post = a.post_kind != CUBE3D_NORM_NONE, pre = a.pre_kind != CUBE3D_NORM_NONE;
    const float inv = 1.f / (float)a.cols;
    int64_t col[P];
    int valid[P];
    bool live[P];
    // (two pieces a lane leave no registers for the parameters: those are read row by row)
    constexpr bool HELD = P == 1;
    float post_gamma[VEC], post_beta[VEC], gate[VEC], pre_gamma[VEC], pre_beta[VEC];
    int64_t vec[P];
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const Run run = run_of<RAGGED>(a, (p * waves + g.wave - g.first) * 64 + g.lane);
        valid[p] = run.valid;
        live[p] = run.valid > 0;
        const int cc = live[p] ? run.c : 0;
        col[p] = axis_offset_fast(a.col, cc);
        vec[p] = axis_offset_fast(a.vec, cc);
    }
    auto look_up_post = [&](int p) {
        vector_run<RAGGED>(a.p.post_gamma, vec[p], valid[p], 1.f, post_gamma);
        vector_run<RAGGED>(a.p.post_beta, vec[p], valid[p], 0.f, post_beta);
    };
    auto look_up_gate = [&](int p) { vector_run<RAGGED>(a.p.gate, vec[p], valid[p], 1.f, gate); };
    auto look_up_pre = [&](int p) {
        vector_run<RAGGED>(a.p.pre_gamma, vec[p], valid[p], 1.f, pre_gamma);
        vector_run<RAGGED>(a.p.pre_beta, vec[p], valid[p], 0.f, pre_beta);
    };
    if constexpr (HELD) {
        look_up_post(0);
        look_up_gate(0);
        look_up_pre(0);
    }
    Pack8<TS> xr[P];
    Pack8<TB> ur[P];
    const int64_t step = (int64_t)gridDim.x * rows_at_once;
    auto load = [&](int64_t row) {
        const int64_t at = axis_offset_fast(a.row, min(row, a.rows - 1));
#pragma unroll
        for (int p = 0; p < P; ++p) {
            xr[p] = get_run<RAGGED>(x + at + col[p], valid[p]);
            if (a.u) ur[p] = get_run<RAGGED>(u + at + col[p], valid[p]);
        }
    };
    // sum over the row of f(piece, element), lanes beyond its end aside
    auto total = [&](auto &&f) {
        float s[1] = {0.f};
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int e = 0; e < VEC; ++e) s[0] += (RAGGED ? e < valid[p] : live[p]) ? f(p, e) : 0.f;
        group_sum<1>(g, s);
        return s[0];
    };
    int64_t row = (int64_t)blockIdx.x * rows_at_once + group;
    load(row);
    // (all wavefronts of the workgroup take as many turns: row_sum has barriers)
    for (int64_t base = (int64_t)blockIdx.x * rows_at_once; base < a.rows; base += step, row += step) {
        float r[P][VEC], v[P][VEC];
#pragma unroll
        for (int p = 0; p < P; ++p) {
            unpack(xr[p], r[p]);
            if (a.u) unpack(ur[p], v[p]);
        }
        if (base + step < a.rows) load(row + step);
        float post_mean = 0.f, post_rstd = 0.f, pre_mean = 0.f, pre_rstd = 0.f;
        if (post) {
            if (a.post_kind == CUBE3D_NORM_LAYER) post_mean = total([&](int p, int e) { return v[p][e]; }) * inv;
            const float var = total([&](int p, int e) { return (v[p][e] - post_mean) * (v[p][e] - post_mean); }) * inv;
            post_rstd = 1.f / sqrtf(var + a.post_eps);
#pragma unroll
            for (int p = 0; p < P; ++p) {
                if constexpr (!HELD) look_up_post(p);
#pragma unroll
                for (int e = 0; e < VEC; ++e) v[p][e] = (v[p][e] - post_mean) * post_rstd * post_gamma[e] + post_beta[e];
            }
        }
        if (a.u) {
#pragma unroll
            for (int p = 0; p < P; ++p) {
                if constexpr (!HELD) look_up_gate(p);
#pragma unroll
                for (int e = 0; e < VEC; ++e) r[p][e] += a.scale * gate[e] * v[p][e];
            }
        }
        if (pre) {
            if (a.pre_kind == CUBE3D_NORM_LAYER) pre_mean = total([&](int p, int e) { return r[p][e]; }) * inv;
            const float var = total([&](int p, int e) { return (r[p][e] - pre_mean) * (r[p][e] - pre_mean); }) * inv;
            pre_rstd = 1.f / sqrtf(var + a.pre_eps);
        }
        if (row >= a.rows) continue;
        const int64_t at = axis_offset_fast(a.row, row);
#pragma unroll
        for (int p = 0; p < P; ++p) {
            if (!live[p]) continue;
            if (r_out) put_run<RAGGED>(r_out + at + col[p], valid[p], pack_out<TS>(r[p]));
            if (pre) {
                if constexpr (!HELD) look_up_pre(p);
                float n[VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) n[e] = (r[p][e] - pre_mean) * pre_rstd * pre_gamma[e] + pre_beta[e];
                put_run<RAGGED>(n_out + at + col[p], valid[p], pack_out<TB>(n));
            }
        }
        if (a.stats_out && g.wave == g.first && g.lane == 0)
            *reinterpret_cast<f32x4 *>(a.stats_out + 4 * row) = f32x4{post_mean, post_rstd, pre_mean, pre_rstd};
    }
}

// Workgroup w leaves the sums over its rows in partials[w].  MOST: wavefronts of a workgroup (most_waves); with sixteen there are no
// registers for both norms' parameters, which are read row by row then, and no row ahead.
template <typename TS, typename TB, bool PRE, bool POST, int MOST, bool RAGGED>
__global__ __launch_bounds__(64 * MOST) void norm_bwd_kernel(const NormArgs a, float *__restrict__ partials, int waves, int rows_at_once, int wanted)
{
    __shared__ float lds[2][2][16];
    extern __shared__ float tail[];      // rows_at_once > 1: their column sums, one vector at a time
    RowGroup g;
    g.lane = threadIdx.x % 64;
    g.wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    g.waves = waves;
    const int group = g.wave / waves;
    g.first = group * waves;
    g.lds = lds;
    g.slot = 0;
    const TS *dr = static_cast<const TS *>(a.dr), *r = static_cast<const TS *>(a.x);
    const TB *dn = static_cast<const TB *>(a.dn), *u = static_cast<const TB *>(a.u);
    TS *dx = static_cast<TS *>(a.dx);
    TB *du = static_cast<TB *>(a.du);
    const float inv = 1.f / (float)a.cols;
    const int own = (g.wave - g.first) * 64 + g.lane;
    const Run run = run_of<RAGGED>(a, own);
    const int c = run.c, valid = run.valid;
    const bool live = valid > 0;
    const int64_t col = axis_offset_fast(a.col, live ? c : 0), vec = axis_offset_fast(a.vec, live ? c : 0);
    float post_gamma[VEC], post_beta[VEC], gate[VEC], pre_gamma[VEC];
    constexpr bool HELD = !(PRE && POST && MOST == 16);
    auto look_up_pre = [&]() { vector_run<RAGGED>(a.p.pre_gamma, vec, valid, 1.f, pre_gamma); };
    auto look_up_post = [&]() {
        vector_run<RAGGED>(a.p.gate, vec, valid, 1.f, gate);
        if constexpr (POST) {
            vector_run<RAGGED>(a.p.post_gamma, vec, valid, 1.f, post_gamma);
            vector_run<RAGGED>(a.p.post_beta, vec, valid, 0.f, post_beta);
        }
    };
    if constexpr (HELD) {
        if constexpr (PRE) look_up_pre();
        look_up_post();
    }
    float sum[VECTORS][VEC];
#pragma unroll
    for (int v = 0; v < VECTORS; ++v)
#pragma unroll
        for (int e = 0; e < VEC; ++e) sum[v][e] = 0.f;
    Pack8<TS> dr_raw, r_raw;
    Pack8<TB> dn_raw, u_raw;
    f32x4 st_raw;
    const bool with_u = POST || a.read_u;
    auto load = [&](int64_t row) {
        const int64_t rr = min(row, a.rows - 1), at = axis_offset_fast(a.row, rr) + col;
        if (dr) dr_raw = get_run<RAGGED>(dr + at, valid);
        if constexpr (PRE) {
            dn_raw = get_run<RAGGED>(dn + at, valid);
            r_raw = get_run<RAGGED>(r + at, valid);
        }
        if (with_u) u_raw = get_run<RAGGED>(u + at, valid);
        if constexpr (PRE || POST) st_raw = *reinterpret_cast<const f32x4 *>(a.stats + 4 * rr);
    };
    const int64_t step = (int64_t)gridDim.x * rows_at_once;
    int64_t row = (int64_t)blockIdx.x * rows_at_once + group;
    load(row);
    for (int64_t base = (int64_t)blockIdx.x * rows_at_once; base < a.rows; base += step, row += step) {
        const bool here = live && row < a.rows;
        auto ok = [&](int e) { return RAGGED ? here && e < valid : here; };
        float d[VEC], t[VEC], hat[VEC], w[VEC];
        f32x4 st;
        if (dr) unpack(dr_raw, d);
        else
#pragma unroll
            for (int e = 0; e < VEC; ++e) d[e] = 0.f;
        if constexpr (PRE) {
            unpack(dn_raw, t);
            unpack(r_raw, hat);
        }
        if (with_u) unpack(u_raw, w);
        if constexpr (PRE || POST) st = st_raw;
        const int64_t at = axis_offset_fast(a.row, min(row, a.rows - 1)) + col;
        if (HELD && base + step < a.rows) load(row + step);
        if constexpr (PRE) {
            if constexpr (!HELD) look_up_pre();
            float m[2] = {0.f, 0.f};
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                hat[e] = (hat[e] - st[2]) * st[3];
                const float b = ok(e) ? t[e] : 0.f;
                sum[3][e] = fmaf(b, ok(e) ? hat[e] : 0.f, sum[3][e]);
                sum[4][e] += b;
                t[e] = ok(e) ? t[e] * pre_gamma[e] : 0.f;
                m[0] += t[e];
                m[1] = fmaf(t[e], ok(e) ? hat[e] : 0.f, m[1]);
            }
            group_sum<2>(g, m);
            const float m0 = a.pre_kind == CUBE3D_NORM_LAYER ? m[0] * inv : 0.f, m1 = m[1] * inv;
#pragma unroll
            for (int e = 0; e < VEC; ++e) d[e] += st[3] * (t[e] - m0 - hat[e] * m1);
        }
        if (dx && here) put_run<RAGGED>(dx + at, valid, pack_out<TS>(d));
#pragma unroll
        for (int e = 0; e < VEC; ++e) d[e] = ok(e) ? d[e] * a.scale : 0.f;
        if constexpr (!HELD) look_up_post();
        if constexpr (POST) {
            float m[2] = {0.f, 0.f};
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                w[e] = ok(e) ? (w[e] - st[0]) * st[1] : 0.f;
                sum[2][e] = fmaf(d[e], w[e] * post_gamma[e] + post_beta[e], sum[2][e]);
                d[e] *= gate[e];
                sum[0][e] = fmaf(d[e], w[e], sum[0][e]);
                sum[1][e] += d[e];
                d[e] *= post_gamma[e];
                m[0] += d[e];
                m[1] = fmaf(d[e], w[e], m[1]);
            }
            group_sum<2>(g, m);
            const float m0 = a.post_kind == CUBE3D_NORM_LAYER ? m[0] * inv : 0.f, m1 = m[1] * inv;
#pragma unroll
            for (int e = 0; e < VEC; ++e) d[e] = st[1] * (d[e] - m0 - w[e] * m1);
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                if (with_u) sum[2][e] = fmaf(d[e], ok(e) ? w[e] : 0.f, sum[2][e]);
                d[e] *= gate[e];
            }
        }
        if (du && here) put_run<RAGGED>(du + at, valid, pack_out<TB>(d));
        if (!HELD && base + step < a.rows) load(row + step);
    }
    if (!a.sums) return;
    float *out = partials + (int64_t)blockIdx.x * VECTORS * a.cols;
    const int width = waves * 64 * VEC;
#pragma unroll
    for (int v = 0; v < VECTORS; ++v) {
        if ((v < 2 && !POST) || (v > 2 && !PRE) || !(wanted >> v & 1)) continue;
        if (rows_at_once > 1) {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < VEC; ++e) tail[group * width + e * waves * 64 + own] = sum[v][e];
            __syncthreads();
            if (group == 0)
                for (int k = 1; k < rows_at_once; ++k)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) sum[v][e] += tail[k * width + e * waves * 64 + own];
        }
        if (RAGGED && group == 0) {
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (e < valid) out[(int64_t)v * a.cols + c + e] = sum[v][e];
        } else if (group == 0 && live) {
            f32x4 *dst = reinterpret_cast<f32x4 *>(out + (int64_t)v * a.cols + c);
            dst[0] = f32x4{sum[v][0], sum[v][1], sum[v][2], sum[v][3]};
            dst[1] = f32x4{sum[v][4], sum[v][5], sum[v][6], sum[v][7]};
        }
    }
}

// Consecutive columns that lie side by side and aligned in every array: eight, four, two or one
int widest(const NormArgs &a)
{
    for (int v : {VEC, VEC / 2, VEC / 4}) {
        bool fits = a.row.u % v == 0 && a.row.s1 % v == 0 && a.row.s2 % v == 0 && a.cols % v == 0;
        for (const AxisMap *m : {&a.col, &a.vec}) fits = fits && m->P1 % v == 0 && m->P2 % v == 0 && m->s1 % v == 0 && m->s2 % v == 0;
        if (fits) return v;
    }
    return 1;
}

template <typename F> int by_width(const NormArgs &a, F &&f)
{
    switch (widest(a)) {
    case VEC: return f(std::integral_constant<int, VEC>{});
    case VEC / 2: return f(std::integral_constant<int, VEC / 2>{});
    case VEC / 4: return f(std::integral_constant<int, VEC / 4>{});
    default: return f(std::integral_constant<int, 1>{});
    }
}

// Rows of up to 16384 columns, sixteen a lane: the registers hold a row and nothing else, so the parameters are read row by row and the
// column sums lie in LDS, where a lane finds its own (16 columns x 4 bytes x the row's lanes for each vector asked for: four vectors up to
// 9216 columns, three up to 12288, two up to 16384).  Where the vectors asked for do not fit, the two passes for any size take the call.  us, here / there: 16384 x 12288 bf16 402 / 668,
// 8192 x 16384 271 / 473, 16384 x 12288 with an fp32 stream and both norms 741 / 1300.
constexpr int LONG_SUMS = 38400;         // floats: 150 KB of the 160
template <typename TS, typename TB, bool PRE, bool POST>
__global__ __launch_bounds__(1024) void norm_bwd_long_kernel(const NormArgs a, float *__restrict__ partials, int waves, int wanted)
{
    constexpr int P = 2;
    __shared__ float lds[2][2][16];
    __shared__ __attribute__((aligned(16))) float sums[LONG_SUMS];
    RowGroup g;
    g.lane = threadIdx.x % 64;
    g.wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    g.waves = waves;
    g.first = 0;
    g.lds = lds;
    g.slot = 0;
    const TS *dr = static_cast<const TS *>(a.dr), *r = static_cast<const TS *>(a.x);
    const TB *dn = static_cast<const TB *>(a.dn), *u = static_cast<const TB *>(a.u);
    TS *dx = static_cast<TS *>(a.dx);
    TB *du = static_cast<TB *>(a.du);
    const float inv = 1.f / (float)a.cols;
    const int lanes = waves * 64;
    int64_t col[P], vec[P];
    bool live[P];
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const int c = (p * lanes + (int)threadIdx.x) * VEC;
        live[p] = c < a.cols;
        col[p] = axis_offset_fast(a.col, live[p] ? c : 0);
        vec[p] = axis_offset_fast(a.vec, live[p] ? c : 0);
    }
    // a lane's eight sums of vector v (the n-th of the wanted ones), piece p
    auto place = [&](int v, int p, int half) {
        const int n = __builtin_popcount(wanted & ((1 << v) - 1));
        return reinterpret_cast<f32x4 *>(sums) + ((n * P + p) * 2 + half) * lanes + threadIdx.x;
    };
#pragma unroll
    for (int v = 0; v < VECTORS; ++v)
#pragma unroll
        for (int p = 0; p < P; ++p)
            if (wanted >> v & 1) *place(v, p, 0) = *place(v, p, 1) = f32x4{0.f, 0.f, 0.f, 0.f};
    auto add = [&](int v, int p, auto &&f) {
        if (!(wanted >> v & 1)) return;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            f32x4 s = *place(v, p, half);
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] += f(4 * half + e);
            *place(v, p, half) = s;
        }
    };
    const bool with_u = POST || a.read_u;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const int64_t at = axis_offset_fast(a.row, row);
        float d[P][VEC], t[P][VEC], hat[P][VEC], w[P][VEC];
        f32x4 st = {0.f, 0.f, 0.f, 0.f};
        if constexpr (PRE || POST) st = *reinterpret_cast<const f32x4 *>(a.stats + 4 * row);
#pragma unroll
        for (int p = 0; p < P; ++p) {
            if (dr) get<TS, VEC>(dr, at + col[p], d[p]);
            else
#pragma unroll
                for (int e = 0; e < VEC; ++e) d[p][e] = 0.f;
            if constexpr (PRE) {
                get<TB, VEC>(dn, at + col[p], t[p]);
                get<TS, VEC>(r, at + col[p], hat[p]);
            }
            if (with_u) get<TB, VEC>(u, at + col[p], w[p]);
        }
        if constexpr (PRE) {
            float m[2] = {0.f, 0.f};
#pragma unroll
            for (int p = 0; p < P; ++p) {
                float gamma[VEC];
                vector_at<VEC>(a.p.pre_gamma, vec[p], 1.f, gamma);
#pragma unroll
                for (int e = 0; e < VEC; ++e) hat[p][e] = (hat[p][e] - st[2]) * st[3];
                add(3, p, [&](int e) { return t[p][e] * hat[p][e]; });
                add(4, p, [&](int e) { return t[p][e]; });
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    t[p][e] *= gamma[e];
                    m[0] += live[p] ? t[p][e] : 0.f;
                    m[1] = fmaf(live[p] ? t[p][e] : 0.f, live[p] ? hat[p][e] : 0.f, m[1]);
                }
            }
            group_sum<2>(g, m);
            const float m0 = a.pre_kind == CUBE3D_NORM_LAYER ? m[0] * inv : 0.f, m1 = m[1] * inv;
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int e = 0; e < VEC; ++e) d[p][e] += st[3] * (t[p][e] - m0 - hat[p][e] * m1);
        }
        float m[2] = {0.f, 0.f};
#pragma unroll
        for (int p = 0; p < P; ++p) {
            if (dx && live[p]) *reinterpret_cast<Pack8<TS> *>(dx + at + col[p]) = pack_out<TS>(d[p]);
            float gate[VEC];
            vector_at<VEC>(a.p.gate, vec[p], 1.f, gate);
#pragma unroll
            for (int e = 0; e < VEC; ++e) d[p][e] *= a.scale;
            if constexpr (POST) {
                float gamma[VEC], beta[VEC];
                vector_at<VEC>(a.p.post_gamma, vec[p], 1.f, gamma);
                vector_at<VEC>(a.p.post_beta, vec[p], 0.f, beta);
#pragma unroll
                for (int e = 0; e < VEC; ++e) w[p][e] = (w[p][e] - st[0]) * st[1];
                add(2, p, [&](int e) { return d[p][e] * (w[p][e] * gamma[e] + beta[e]); });
#pragma unroll
                for (int e = 0; e < VEC; ++e) d[p][e] *= gate[e];
                add(0, p, [&](int e) { return d[p][e] * w[p][e]; });
                add(1, p, [&](int e) { return d[p][e]; });
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    d[p][e] *= gamma[e];
                    m[0] += live[p] ? d[p][e] : 0.f;
                    m[1] = fmaf(live[p] ? d[p][e] : 0.f, live[p] ? w[p][e] : 0.f, m[1]);
                }
            } else {
                if (with_u) add(2, p, [&](int e) { return d[p][e] * w[p][e]; });
#pragma unroll
                for (int e = 0; e < VEC; ++e) d[p][e] *= gate[e];
            }
        }
        if constexpr (POST) {
            group_sum<2>(g, m);
            const float m0 = a.post_kind == CUBE3D_NORM_LAYER ? m[0] * inv : 0.f, m1 = m[1] * inv;
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int e = 0; e < VEC; ++e) d[p][e] = st[1] * (d[p][e] - m0 - w[p][e] * m1);
        }
#pragma unroll
        for (int p = 0; p < P; ++p)
            if (du && live[p]) *reinterpret_cast<Pack8<TB> *>(du + at + col[p]) = pack_out<TB>(d[p]);
    }
    float *out = partials + (int64_t)blockIdx.x * VECTORS * a.cols;
#pragma unroll
    for (int v = 0; v < VECTORS; ++v)
#pragma unroll
        for (int p = 0; p < P; ++p)
            if ((wanted >> v & 1) && live[p]) {
                f32x4 *dst = reinterpret_cast<f32x4 *>(out + (int64_t)v * a.cols + (p * lanes + (int)threadIdx.x) * VEC);
                dst[0] = *place(v, p, 0);
                dst[1] = *place(v, p, 1);
            }
}

// How rows are dealt out: wavefronts per row, rows per workgroup, pieces of eight columns per lane, workgroups, whether runs are ragged;
// waves = 0: not in registers.
struct RowPlan {
    int waves, rows_at_once, pieces;
    unsigned groups;
    bool ragged;
};

// Most wavefronts of a backward workgroup.  Both norms at once take some 150 registers a lane: twelve then (in sixteen they spill, or
// do without what is read ahead), or eight where those hold whole rows and an fp32 stream takes more registers.  us with eight /
// twelve, at 8192 rows with bf16 and with fp32 streams: 1024 columns 28.0 / 28.4, 30.6 / 32.7; 2048 44.4 / 42.8, 57.7 / 60.8;
// 2560 78 / 56, 76 / 79; 6144 147 / 127 and 190 / 179 (sixteen / twelve).
// (Ragged runs take a few registers more: one size less.  Sixteen wavefronts of one norm spill 12 to 17 registers and still are
// faster than the any-size kernels: 3000 x 8001 80 us for 150.)
int most_waves(const NormArgs &a, int waves, bool ragged)
{
    const bool both = a.pre_kind != CUBE3D_NORM_NONE && a.post_kind != CUBE3D_NORM_NONE;
    if (ragged) return both ? 8 : waves <= 12 ? 12 : 16;
    if (!both || waves > 12) return 16;
    return waves <= 2 || (waves <= 8 && a.stream_f32) ? 8 : 12;
}

RowPlan row_plan(const NormArgs &a, bool backward)
{
    const int width = widest(a);
    RowPlan p{0, 1, 1, 0, width != VEC};
    if (width == VEC / 2) return p;
    const int64_t runs = p.ragged ? (int64_t)a.q * a.q * ((a.vec.P2 + VEC - 1) / VEC) : a.cols / VEC, most = SHORT_ROW / VEC;
    if (runs > (p.ragged ? 16 : 32) * most) return p;
    p.pieces = runs > 16 * most ? 2 : 1;
    p.waves = (int)((runs + most * p.pieces - 1) / (most * p.pieces));
    if (backward && p.ragged && p.waves > most_waves(a, p.waves, true)) {
        p.waves = 0;
        return p;
    }
    const int64_t cus = num_compute_units();
    if (backward) {
        // A workgroup leaves a partial sum of every vector: as few of them as fill the CUs, of as many rows at once as that allows
        // (one norm, us with several rows at once / one on as many more workgroups: 2997 x 1152 17.8 / 20.0, 8192 x 512 14.8 / 28.0,
        // 32768 x 512 32.5 / 45.2, 8192 x 1024 20.8 / 26.8)
        const int fit = most_waves(a, p.waves, p.ragged) / p.waves;
        const int64_t each = (a.rows + cus - 1) / cus;
        p.rows_at_once = fit < each ? fit : (int)each;
    } else p.rows_at_once = p.waves == 1 ? 4 : p.waves == 2 ? 2 : 1;
    // about sixteen wavefronts a CU
    const int64_t per_cu = backward || p.waves * p.rows_at_once > 16 ? 1 : 16 / (p.waves * p.rows_at_once);
    int64_t groups = (a.rows + p.rows_at_once - 1) / p.rows_at_once;
    if (groups > cus * per_cu) groups = cus * per_cu;
    p.groups = (unsigned)groups;
    return p;
}

// Rows per workgroup of the column pass: enough workgroups for every CU, few enough partial sums.
int rows_per_group(const NormArgs &a)
{
    const int64_t width = 64 * widest(a), tiles = (a.cols + width - 1) / width;
    int64_t rows = 256;
    while (rows > 16 && tiles * ((a.rows + rows - 1) / rows) < 2048) rows /= 2;
    while ((a.rows + rows - 1) / rows > 32768) rows *= 2;
    return (int)rows;
}

template <typename F> int by_types(const NormArgs &a, F &&f)
{
    const bool s = a.stream_f32, b = a.block_f32;
    if (s) return b ? f(float{}, float{}) : f(float{}, (unsigned short)0);
    return b ? f((unsigned short)0, float{}) : f((unsigned short)0, (unsigned short)0);
}

// One wavefront a row where it takes at most eight turns, else a workgroup of four; in either case 32 wavefronts a CU.
// LANES and the number of workgroups are passed to `f`.
template <typename F> void by_lanes(const NormArgs &a, int v, F &&f)
{
    const bool one = a.cols <= 8 * 64 * v;
    const int64_t most = (int64_t)num_compute_units() * (one ? 32 : 8);
    const dim3 groups((unsigned)(a.rows < most ? a.rows : most));
    if (one) f(std::integral_constant<int, 64>{}, groups);
    else f(std::integral_constant<int, ROW_LANES>{}, groups);
}

}  // namespace

int norm_fwd(const NormArgs &a, hipStream_t stream)
{
    const RowPlan plan = row_plan(a, false);
    return by_types(a, [&](auto s, auto b) {
        typedef decltype(s) TS;
        typedef decltype(b) TB;
        const dim3 block(64 * plan.waves * plan.rows_at_once);
        if (plan.waves == 0)
            return by_width(a, [&](auto v) {
                constexpr int V = decltype(v)::value;
                by_lanes(a, V, [&](auto l, dim3 groups) {
                    constexpr int LANES = decltype(l)::value;
                    hipLaunchKernelGGL((norm_fwd_rows_kernel<TS, TB, V, LANES>), groups, dim3(LANES), 0, stream, a);
                });
                return launch_status();
            });
        if (plan.ragged)
            hipLaunchKernelGGL((norm_fwd_kernel<TS, TB, 1, true>), dim3(plan.groups), block, 0, stream, a, plan.waves, plan.rows_at_once);
        else if (plan.pieces == 1)
            hipLaunchKernelGGL((norm_fwd_kernel<TS, TB, 1, false>), dim3(plan.groups), block, 0, stream, a, plan.waves, plan.rows_at_once);
        else
            hipLaunchKernelGGL((norm_fwd_kernel<TS, TB, 2, false>), dim3(plan.groups), block, 0, stream, a, plan.waves, plan.rows_at_once);
        return launch_status();
    });
}

// (long rows: whether they fit depends on the vectors asked for, so there is room for either way)
size_t norm_bwd_workspace(const NormArgs &a)
{
    const RowPlan plan = row_plan(a, true);
    const size_t in_registers = (size_t)plan.groups * VECTORS * a.cols * sizeof(float);
    if (plan.waves > 0 && plan.pieces == 1) return in_registers;
    const int64_t per = rows_per_group(a), groups = (a.rows + per - 1) / per;
    const size_t by_columns = ((size_t)a.rows * 4 + (size_t)groups * VECTORS * a.cols) * sizeof(float);
    return by_columns > in_registers ? by_columns : in_registers;
}

namespace {

// A launch has fewer than 2^32 work-items along a grid dimension: `tiles` workgroups of `lanes` in as many launches as that takes.
template <typename F> int launch_in_parts(int64_t tiles, int lanes, F &&f)
{
    const int64_t most = (1ll << 32) / lanes - 1;
    for (int64_t first = 0; first < tiles; first += most) {
        f((unsigned)(tiles - first < most ? tiles - first : most), (int)first);
        if (const int rc = launch_status(); rc != CUBE3D_OK) return rc;
    }
    return CUBE3D_OK;
}

int finish(const NormArgs &a, const float *partials, unsigned groups, const cube3d_norm_params &gradients, hipStream_t stream)
{
    const unsigned q3 = (unsigned)(a.q * a.q * a.q);
    return launch_in_parts(((int64_t)a.vec.P2 + 63) / 64, 64 * FINISH_WAVES, [&](unsigned tiles, int first) {
        hipLaunchKernelGGL(norm_bwd_finish_kernel, dim3(tiles, q3, VECTORS), dim3(64 * FINISH_WAVES), 0, stream, a, partials, (int)groups, gradients,
                           first);
    });
}

}  // namespace

int norm_bwd(const NormArgs &a, const cube3d_norm_params &gradients, void *workspace, hipStream_t stream)
{
    const bool pre = a.pre_kind != CUBE3D_NORM_NONE, post = a.post_kind != CUBE3D_NORM_NONE;
    const cube3d_norm_params &d = gradients;
    const int wanted = (d.post_gamma ? 1 : 0) | (d.post_beta ? 2 : 0) | (d.gate ? 4 : 0) | (d.pre_gamma ? 8 : 0) | (d.pre_beta ? 16 : 0);
    const RowPlan plan = row_plan(a, true);
    if (plan.waves > 0 && plan.pieces == 2 && __builtin_popcount(wanted) * plan.waves * 2 * SHORT_ROW <= LONG_SUMS) {
        float *partials = static_cast<float *>(workspace);
        const int rc = by_types(a, [&](auto s, auto b) {
            typedef decltype(s) TS;
            typedef decltype(b) TB;
            auto launch = [&](auto pre_c, auto post_c) {
                hipLaunchKernelGGL((norm_bwd_long_kernel<TS, TB, decltype(pre_c)::value, decltype(post_c)::value>), dim3(plan.groups),
                                   dim3(64 * plan.waves), 0, stream, a, partials, plan.waves, wanted);
                return launch_status();
            };
            const std::true_type yes{};
            const std::false_type no{};
            return pre ? (post ? launch(yes, yes) : launch(yes, no)) : (post ? launch(no, yes) : launch(no, no));
        });
        return rc != CUBE3D_OK || !a.sums ? rc : finish(a, partials, plan.groups, gradients, stream);
    }
    if (plan.waves > 0 && plan.pieces == 1) {
        float *partials = static_cast<float *>(workspace);
        const dim3 grid(plan.groups), block(64 * plan.waves * plan.rows_at_once);
        const size_t lds = plan.rows_at_once > 1 ? sizeof(float) * plan.rows_at_once * plan.waves * SHORT_ROW : 0;
        const int rc = by_types(a, [&](auto s, auto b) {
            typedef decltype(s) TS;
            typedef decltype(b) TB;
            auto launch = [&](auto pre_c, auto post_c) {
                constexpr bool PRE = decltype(pre_c)::value, POST = decltype(post_c)::value;
                auto start = [&](auto most, auto ragged) {
                    hipLaunchKernelGGL((norm_bwd_kernel<TS, TB, PRE, POST, decltype(most)::value, decltype(ragged)::value>), grid, block, lds,
                                       stream, a, partials, plan.waves, plan.rows_at_once, wanted);
                };
                const std::integral_constant<int, 8> eight{};
                const std::integral_constant<int, 12> twelve{};
                const std::integral_constant<int, 16> sixteen{};
                const std::true_type ragged{};
                const std::false_type whole{};
                const int most = most_waves(a, plan.waves, plan.ragged);
                if constexpr (PRE && POST) {
                    if (plan.ragged) start(eight, ragged);
                    else if (most == 8) start(eight, whole);
                    else most == 12 ? start(twelve, whole) : start(sixteen, whole);
                } else if (plan.ragged) most == 12 ? start(twelve, ragged) : start(sixteen, ragged);
                else start(sixteen, whole);
                return launch_status();
            };
            const std::true_type yes{};
            const std::false_type no{};
            return pre ? (post ? launch(yes, yes) : launch(yes, no)) : (post ? launch(no, yes) : launch(no, no));
        });
        return rc != CUBE3D_OK || !a.sums ? rc : finish(a, partials, plan.groups, gradients, stream);
    }
    float *scalars = static_cast<float *>(workspace), *partials = scalars + a.rows * 4;
    const int per = rows_per_group(a);
    const unsigned groups = (unsigned)((a.rows + per - 1) / per);
    const int rc = by_types(a, [&](auto s, auto b) {
        typedef decltype(s) TS;
        typedef decltype(b) TB;
        return by_width(a, [&](auto v) {
            constexpr int V = decltype(v)::value;
            if (pre || post)
                by_lanes(a, V, [&](auto l, dim3 wide) {
                    constexpr int LANES = decltype(l)::value;
                    hipLaunchKernelGGL((norm_bwd_rows_kernel<TS, TB, V, LANES>), wide, dim3(LANES), 0, stream, a, scalars);
                });
            if (const int e = launch_status(); e != CUBE3D_OK) return e;
            return launch_in_parts(((int64_t)a.cols + 64 * V - 1) / (64 * V), 256, [&](unsigned tiles, int first) {
                hipLaunchKernelGGL((norm_bwd_columns_kernel<TS, TB, V>), dim3(tiles, groups), dim3(256), 0, stream, a, scalars, partials, per, wanted,
                                   first);
            });
        });
    });
    return rc != CUBE3D_OK || !a.sums ? rc : finish(a, partials, groups, gradients, stream);
}

}  // namespace cube3d
