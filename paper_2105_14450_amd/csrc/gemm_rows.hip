// The forward product of few rows (tokens) with what follows it: Y = act(X W + b) + R over a cube of shards, for M up to 64 (fp32 32) and, in
// blocks of that, to 512 (gemm_rows_plan says where).
//
// What bounds it: the weights, read once from HBM, M multiply-adds an element.  Nothing is shared between workgroups but X, so W goes
// from memory straight to registers and into the matrix cores, without LDS, barriers or waits for other wavefronts, and
// the contraction is cut into as many runs as it takes to have loads in flight on every CU.
//
// Tile.  A wavefront makes MT x 16 rows by 128 columns with 16 x 16 x 32 MFMAs (fp32: eight of 16 x 16 x 4).  A k-step is 32 contraction
// indices: lane l loads W[k0 + 8 (l / 16) + r, n0 + 8 (l % 16) : + 8] for r = 0 ... 7, whole 256-byte (fp8: 128, fp32: 512) pieces of
// a row per 16 lanes, all eight from one lane offset and eight scalar bases.  That is an 8 x 8 block per lane, which byte
// permutations turn around (fp32: it is only named the other way): column j of the block is the lane's part of the B operand of
// MFMA number j, whose 16 columns are then n0 + 8 c + j.  X, K-major, is its A operand as stored.  The accumulators of the eight
// MFMAs hold eight consecutive columns of four rows in a lane.
//
// Split.  The four wavefronts of a workgroup take its k-steps in turn, and add up through LDS; the runs of the contraction add up in
// a second launch, in ascending order (in place of that, one workgroup per strip leaves most CUs without work: 16 to 64 strips of 128
// columns).  No atomics: two calls give the same bits.
//
// Edges.  Eight consecutive indices of either operand lie side by side in one shard (rows_plan checks it).  Rows and
// columns beyond the output are read from its last ones and not stored; beyond the contraction both operands are zero.
#include "gemm_epilogue.h"

namespace cube3d {

namespace {

constexpr int COLS = 128, KSTEP = 32, WAVES = 4;
constexpr int most_rows_at_once(int64_t es) { return es == 4 ? 32 : 64; }

struct RowsParams {
    const char *A, *B;
    void *C;
    float *partials;            // [splits][M][N], or nullptr: the result is written here
    int M, N, K, steps, splits;
    float alpha;
    int out_f32;
    int64_t row_bytes;          // from one contraction index of W to the next
    GemmMaps maps;
    Epilogue e;
    int piece, bias_piece;
};

struct Bf16Rows {
    static constexpr int ELT = 2;
    typedef i32x4 Piece;                // 8 elements
    typedef i32x4 Frag;
    static constexpr int TURN = 2;      // columns turned at a time
    __device__ static __forceinline__ void turn(const Piece (&row)[8], int c, Frag (&col)[2])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const unsigned even = (unsigned)row[2 * i][c], odd = (unsigned)row[2 * i + 1][c];
            col[0][i] = (int)__builtin_amdgcn_perm(odd, even, 0x05040100u);
            col[1][i] = (int)__builtin_amdgcn_perm(odd, even, 0x07060302u);
        }
    }
    __device__ static __forceinline__ f32x4 mfma(Frag a, Frag b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
};

struct Fp8Rows {
    static constexpr int ELT = 1;
    typedef i32x2 Piece;
    typedef i32x2 Frag;
    static constexpr int TURN = 4;
    __device__ static __forceinline__ void turn(const Piece (&row)[8], int c, Frag (&col)[4])
    {
#pragma unroll
        for (int half = 0; half < 2; ++half) {      // contraction indices 0-3, 4-7
            const unsigned a = (unsigned)row[4 * half][c], b = (unsigned)row[4 * half + 1][c], d = (unsigned)row[4 * half + 2][c],
                           e = (unsigned)row[4 * half + 3][c];
            const unsigned ab01 = __builtin_amdgcn_perm(b, a, 0x05010400u), ab23 = __builtin_amdgcn_perm(b, a, 0x07030602u);
            const unsigned de01 = __builtin_amdgcn_perm(e, d, 0x05010400u), de23 = __builtin_amdgcn_perm(e, d, 0x07030602u);
            col[0][half] = (int)__builtin_amdgcn_perm(de01, ab01, 0x05040100u);
            col[1][half] = (int)__builtin_amdgcn_perm(de01, ab01, 0x07060302u);
            col[2][half] = (int)__builtin_amdgcn_perm(de23, ab23, 0x05040100u);
            col[3][half] = (int)__builtin_amdgcn_perm(de23, ab23, 0x07060302u);
        }
    }
    __device__ static __forceinline__ f32x4 mfma(Frag a, Frag b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_fp8_fp8(__builtin_bit_cast(long, a), __builtin_bit_cast(long, b), c, 0, 0, 0);
    }
};

// fp32 results: the operands widened to bf16, whose instruction has the same layout (see widens).  bf16 results do without: us not widened /
// widened, 16 x 16384 x 4096 18.1 / 18.6, 1 x 8192 x 8192 17.8 / 18.7, 64 x 8192 x 8192 25.9 / 27.7.
struct Fp8WideRows : Fp8Rows {
    __device__ static __forceinline__ f32x4 mfma(Frag a, Frag b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen_fp8(a), widen_fp8(b), c, 0, 0, 0);
    }
};

// fp32: the instruction takes four indices, one a group of lanes, so a k-step is eight of them, over the lane's own indices
struct F32Rows {
    static constexpr int ELT = 4;
    typedef float Piece __attribute__((ext_vector_type(8), aligned(16)));
    typedef Piece Frag;
    static constexpr int TURN = 1;
    __device__ static __forceinline__ void turn(const Piece (&row)[8], int c, Frag (&col)[1])
    {
#pragma unroll
        for (int r = 0; r < 8; ++r) col[0][r] = row[r][c];
    }
    __device__ static __forceinline__ f32x4 mfma(Frag a, Frag b, f32x4 c)
    {
#pragma unroll
        for (int r = 0; r < 8; ++r) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[r], b[r], c, 0, 0, 0);
        return c;
    }
};

// Eight columns of row m from column n on: the end of the way, from the full sum.
__device__ __forceinline__ void finish(const RowsParams &p, int m, int n, float (&x)[8])
{
    float bias[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) bias[e] = 0.f;
    if (p.maps.bias && p.bias_piece == 8) {
        const f32x4 *src = reinterpret_cast<const f32x4 *>(p.maps.bias + axis_offset_fast(p.maps.bias_n, n));
#pragma unroll
        for (int e = 0; e < 8; ++e) bias[e] = src[e / 4][e % 4];
    } else if (p.maps.bias) {
#pragma unroll
        for (int e = 0; e < 8; ++e) bias[e] = p.maps.bias[axis_offset_fast(p.maps.bias_n, n + e)];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = x[e] * p.alpha + bias[e];
    const int64_t row = axis_offset_fast(p.maps.c_m, m), at = row + axis_offset_fast(p.maps.c_n, n);
    if (p.piece == 8) {
        EpilogueRun<8>::Residual r;
        EpilogueRun<8>::load<ANY>(p.e, at, r);
        EpilogueRun<8>::apply<ANY>(p.e, x, r, p.C, p.out_f32, at);
    } else EpilogueRun<8>::apply_some(p.e, x, p.C, p.out_f32, row, p.maps.c_n, n, p.N);
}

// Grid: strips of 128 columns, runs of the contraction, blocks of 16 MT rows.
template <typename E, int MT> __global__ __launch_bounds__(64 * WAVES, MT == (E::ELT == 4 ? 2 : 4) ? 1 : 2) void gemm_rows_kernel(const RowsParams p)
{
    typedef typename E::Piece Piece;
    typedef typename E::Frag Frag;
    constexpr int PITCH = COLS + 4;
    __shared__ __attribute__((aligned(16))) float lds[WAVES][16 * PITCH];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), group = lane / 16, in_group = lane % 16;
    const int n0 = blockIdx.x * COLS, split = blockIdx.y, m0 = blockIdx.z * (16 * MT);
    const int first = (int)((int64_t)p.steps * split / p.splits), last = (int)((int64_t)p.steps * (split + 1) / p.splits);
    const char *b_row[8];
#pragma unroll
    for (int r = 0; r < 8; ++r) b_row[r] = p.B + r * p.row_bytes;
    const unsigned b_col = (unsigned)(axis_offset_fast(p.maps.b_mn, min(n0 + 8 * in_group, p.N - 8)) * E::ELT);
    unsigned a_row[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) a_row[t] = (unsigned)(axis_offset_fast(p.maps.a_mn, min(m0 + 16 * t + in_group, p.M - 1)) * E::ELT);

    f32x4 acc[MT][8];
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[t][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    Piece w[2][8];
    Frag x[2][MT];
    auto load = [&](int step, int buf) {
        const int k = step * KSTEP + 8 * group;
        const bool inside = k < p.K;            // (K % 8 == 0: all eight or none)
        const int kk = inside ? k : 0;
        const unsigned bo = b_col + (unsigned)(axis_offset_fast(p.maps.b_k, kk) * E::ELT), ao = (unsigned)(axis_offset_fast(p.maps.a_k, kk) * E::ELT);
#pragma unroll
        for (int r = 0; r < 8; ++r) w[buf][r] = *reinterpret_cast<const Piece *>(b_row[r] + bo);
#pragma unroll
        for (int t = 0; t < MT; ++t) x[buf][t] = *reinterpret_cast<const Frag *>(p.A + (a_row[t] + ao));
    };
    auto multiply = [&](int step, int buf) {
        if (step * KSTEP + KSTEP > p.K) {       // the last one: zeros beyond the end
            const bool inside = step * KSTEP + 8 * group < p.K;
#pragma unroll
            for (int r = 0; r < 8; ++r) w[buf][r] = inside ? w[buf][r] : Piece{};
#pragma unroll
            for (int t = 0; t < MT; ++t) x[buf][t] = inside ? x[buf][t] : Frag{};
        }
#pragma unroll
        for (int c = 0; c < 8 / E::TURN; ++c) {
            Frag col[E::TURN];
            E::turn(w[buf], c, col);
#pragma unroll
            for (int j = 0; j < E::TURN; ++j)
#pragma unroll
                for (int t = 0; t < MT; ++t) acc[t][c * E::TURN + j] = E::mfma(x[buf][t], col[j], acc[t][c * E::TURN + j]);
        }
    };
    int step = first + wave;
    if (step < last) load(step, 0);
    for (; step < last; step += 2 * WAVES) {
        if (step + WAVES < last) load(step + WAVES, 1);
        multiply(step, 0);
        if (step + WAVES >= last) break;
        if (step + 2 * WAVES < last) load(step + 2 * WAVES, 0);
        multiply(step + WAVES, 1);
    }

    // A lane holds rows 4 group + v and columns 8 in_group + j of every 16 rows: the wavefronts' sums in ascending order
    const int row = threadIdx.x / 16, col = threadIdx.x % 16 * 8;
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        if (t > 0) __syncthreads();
#pragma unroll
        for (int v = 0; v < 4; ++v)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                *reinterpret_cast<f32x4 *>(&lds[wave][(4 * group + v) * PITCH + 8 * in_group + 4 * h]) =
                    f32x4{acc[t][4 * h][v], acc[t][4 * h + 1][v], acc[t][4 * h + 2][v], acc[t][4 * h + 3][v]};
        __syncthreads();
        const int m = m0 + 16 * t + row, n = n0 + col;
        if (m >= p.M || n >= p.N) continue;
        float s[8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            f32x4 y = *reinterpret_cast<const f32x4 *>(&lds[0][row * PITCH + col + 4 * h]);
#pragma unroll
            for (int w2 = 1; w2 < WAVES; ++w2) y += *reinterpret_cast<const f32x4 *>(&lds[w2][row * PITCH + col + 4 * h]);
#pragma unroll
            for (int e = 0; e < 4; ++e) s[4 * h + e] = y[e];
        }
        if (p.partials) {
            f32x4 *dst = reinterpret_cast<f32x4 *>(p.partials + ((int64_t)split * p.M + m) * p.N + n);
            dst[0] = f32x4{s[0], s[1], s[2], s[3]};
            dst[1] = f32x4{s[4], s[5], s[6], s[7]};
        } else finish(p, m, n, s);
    }
}

// A lane adds eight columns of a row over the runs.
__global__ __launch_bounds__(256) void gemm_rows_join_kernel(const RowsParams p)
{
    const int per_row = p.N / 8;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= (int64_t)p.M * per_row) return;
    const int m = (int)(id / per_row), n = (int)(id - (int64_t)m * per_row) * 8;
    const float *src = p.partials + (int64_t)m * p.N + n;
    f32x4 lo = *reinterpret_cast<const f32x4 *>(src), hi = *reinterpret_cast<const f32x4 *>(src + 4);
#pragma unroll 4
    for (int s = 1; s < p.splits; ++s) {
        src += (int64_t)p.M * p.N;
        lo += *reinterpret_cast<const f32x4 *>(src);
        hi += *reinterpret_cast<const f32x4 *>(src + 4);
    }
    float x[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    finish(p, m, n, x);
}

bool eights(const AxisMap &m, int64_t extent, int64_t unit)
{
    return extent % 8 == 0 && m.P1 % 8 == 0 && m.P2 % 8 == 0 && m.s1 % 8 == 0 && m.s2 % 8 == 0 && m.u == unit;
}

template <typename E, int MT> int launch(const RowsParams &p, hipStream_t stream)
{
    const dim3 grid((unsigned)((p.N + COLS - 1) / COLS), (unsigned)p.splits, (unsigned)((p.M + 16 * MT - 1) / (16 * MT)));
    hipLaunchKernelGGL((gemm_rows_kernel<E, MT>), grid, dim3(64 * WAVES), 0, stream, p);
    if (const int rc = launch_status(); rc != CUBE3D_OK || p.splits == 1) return rc;
    const int64_t threads = (int64_t)p.M * (p.N / 8);
    hipLaunchKernelGGL(gemm_rows_join_kernel, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, stream, p);
    return launch_status();
}

template <typename E> int launch_rows(const RowsParams &p, hipStream_t stream)
{
    if (p.M <= 16) return launch<E, 1>(p, stream);
    if constexpr (E::ELT == 4) return launch<E, 2>(p, stream);
    else return p.M <= 32 ? launch<E, 2>(p, stream) : launch<E, 4>(p, stream);
}

}  // namespace

// Runs of the contraction, 0: not for this kernel.  A pure function of the shape and the device.
int gemm_rows_plan(const GemmArgs &g)
{
    if (!g.epilogue || !g.maps || g.batch != 1 || !g.a_kmajor || g.b_kmajor) return 0;
    if (g.Mo > 512 || g.No >= 1ll << 24 || g.Kc >= 1ll << 30) return 0;
    const GemmMaps &m = *g.maps;
    const int64_t es = g.in_dtype == CUBE3D_F32 ? 4 : g.in_dtype == CUBE3D_BF16 ? 2 : 1;
    if (!eights(m.a_k, g.Kc, 1) || !eights(m.b_mn, g.No, 1) || !eights(m.b_k, g.Kc, m.b_k.u) || m.b_k.u % 8) return 0;
    if (m.a_mn.u % 8 || m.a_mn.s1 % 8 || m.a_mn.s2 % 8) return 0;
    // offsets are 32 bits; those of a lane's eight rows lie behind its own
    if ((axis_offset(m.a_mn, g.Mo - 1) + axis_offset(m.a_k, g.Kc - 1) + 1) * es >= 1ll << 32) return 0;
    if ((axis_offset(m.b_mn, g.No - 1) + axis_offset(m.b_k, g.Kc - 1) + 1) * es >= 1ll << 32) return 0;
    // Short contractions: the second launch costs what the ring kernel's one chain of K-tiles does.  us here / on the ring's tiles,
    // weights from HBM, bf16: K = 2048, N = 8192 13.4 / 12.6 (1 row), 16.0 / 13.7 (32); 4096 x 4096 14.2 / 19.6, 16.6 / 21.9; 8192 x 2048
    // 14.8 / 32.6, 17.4 / 37.5; 8192 x 8192 32.5 / 37.3, 35.6 / 42.8; fp8 4096 x 4096 10.6 / 11.5, 13.9 / 13.4; 8192 x 2048 11.1 / 18.7,
    // 14.8 / 24.1; 16384 x 4096 (q = 2, 16 rows) 23.3 / 62.9.  64 rows: 4096 x 4096 20.5 / 21.6, 8192 x 2048 21.3 / 36.1, but
    // 12288 x 12288 102 / 90 (fp8 83 / 64): the sums of the runs count.
    // fp32, where the other kernels' one chain of K-tiles is longer: 512 x 512 7.8 / 9.1 (1 row), 8.6 / 9.3 (16); 2048 x 2048 11.8 / 19.3,
    // 13.0 / 19.6, 17.2 / 19.8 (32); 8192 x 2048 23 / 58, 24 / 58, 31 / 58; 8192 x 8192 56 / 66, 58 / 67; 32 rows, whose accumulators and
    // operands leave one wavefront a SIMD, 1024 x 4096 16.2 / 13.7, 2048 x 8192 28 / 23, 8192 x 8192 76 / 66
    const int64_t at_once = most_rows_at_once(es), blocks = (g.Mo + at_once - 1) / at_once;
    if (blocks > 1) {
        // Several blocks of rows read the weights once each, from the caches if need be: where the ring's tiles of 64 leave half of the CUs
        // without work for a long contraction.  bf16, here / there: 128 x 8192 x 2048 23 / 33, 256 x 8192 x 2048 31 / 44, 128 x 14336 x 4096
        // 51 / 84, 512 x 24576 x 1024 67 / 126, 128 x 9216 x 1152 22.9 / 22.3, but 128 x 8192 x 8192 52 / 40, 512 x 8200 x 1544 74 / 53;
        // fp8 128 x 16384 x 2048 30 / 48, 256 x 12000 x 1000 23.5 / 45, but 128 x 8192 x 2048 22 / 18; fp32 64 x 4096 x 1024 19 / 32,
        // 128 x 16384 x 1024 59 / 108, but 192 x 9216 x 1152 70 / 65.
        const int64_t tiles = ((g.Mo + 63) / 64) * ((g.No + 63) / 64);
        if (tiles > (es == 4 ? 48 : 128) || g.Kc < (es == 4 ? 4096 : es == 2 ? 8192 : 10240)) return 0;
    } else if (es == 4) {
        if (g.Kc < (g.Mo > 16 ? 2048 : 512) || (g.Mo > 16 && g.No > 4096)) return 0;
    } else if (g.Kc * es < 6144 || (g.Mo > 32 && g.No > 8192)) return 0;
    // As many runs as leave the busiest CU the fewest k-steps (20 KB per us and CU), against the traffic of their sums and a launch
    const int64_t strips = (g.No + COLS - 1) / COLS * blocks, steps = (g.Kc + KSTEP - 1) / KSTEP, cus = num_compute_units();
    const double step_us = KSTEP * COLS * es / 20.3e3, run_us = (double)g.Mo * g.No * 8 / 5e6;
    int best = 1;
    double least = 0;
    for (int64_t n = 1; n <= 64 && n * 2 * WAVES <= steps + 2 * WAVES - 1; ++n) {
        const double us = (double)((strips * n + cus - 1) / cus) * (double)((steps + n - 1) / n) * step_us + (n > 1 ? 2.5 + n * run_us : 0.);
        if (n == 1 || us < least) {
            best = (int)n;
            least = us;
        }
    }
    return best;
}

size_t gemm_rows_workspace(const GemmArgs &g, int splits)
{
    return splits > 1 ? (size_t)splits * g.Mo * g.No * sizeof(float) : 0;
}

int gemm_rows(const GemmArgs &g, int splits)
{
    RowsParams p{};
    p.A = static_cast<const char *>(g.A);
    p.B = static_cast<const char *>(g.B);
    p.C = g.C;
    p.partials = splits > 1 ? static_cast<float *>(g.workspace) : nullptr;
    p.M = (int)g.Mo; p.N = (int)g.No; p.K = (int)g.Kc;
    p.steps = (p.K + KSTEP - 1) / KSTEP;
    p.splits = splits;
    p.alpha = g.alpha;
    p.out_f32 = g.out_dtype == CUBE3D_F32;
    p.maps = *g.maps;
    for (AxisMap *x : {&p.maps.a_mn, &p.maps.a_k, &p.maps.b_mn, &p.maps.b_k, &p.maps.c_m, &p.maps.c_n, &p.maps.bias_n}) prepare_axis_map(*x);
    p.row_bytes = p.maps.b_k.u * (g.in_dtype == CUBE3D_F32 ? 4 : g.in_dtype == CUBE3D_BF16 ? 2 : 1);
    p.e = *g.epilogue;
    epilogue_pieces(g, &p.piece, &p.bias_piece);
    if (g.in_dtype == CUBE3D_F32) return launch_rows<F32Rows>(p, g.stream);
    if (g.in_dtype == CUBE3D_BF16) return launch_rows<Bf16Rows>(p, g.stream);
    return widens(g) ? launch_rows<Fp8WideRows>(p, g.stream) : launch_rows<Fp8Rows>(p, g.stream);
}

}  // namespace cube3d
