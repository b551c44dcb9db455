// What follows a product of the forward layout (struct Epilogue), on runs of consecutive output columns: the output stages of the
// product kernels hand over fp32 values row by row, and Z, the residual and the result move in whole 16-byte (bf16 runs of four: 8-byte)
// accesses wherever the output's placement allows.
#pragma once
#include "activation.h"

namespace cube3d {

// The activation is looked up per run: one uniform branch for eight elements, and no variant of a product kernel per activation.
template <int N> __device__ __forceinline__ void activate(int act, float (&x)[N])
{
    if (act == CUBE3D_ACT_GELU) {
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = act_value<CUBE3D_ACT_GELU>(x[e]);
    } else if (act == CUBE3D_ACT_RELU) {
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = act_value<CUBE3D_ACT_RELU>(x[e]);
    }
}

template <int N> struct EpilogueRun {
    static_assert(N == 4 || N == 8, "whole 16-byte accesses of fp32");
    typedef unsigned Half __attribute__((ext_vector_type(N / 2)));     // N bf16 values

    __device__ static __forceinline__ void put(void *base, bool f32, int64_t at, const float (&x)[N])
    {
        if (f32) {
            f32x4 *dst = reinterpret_cast<f32x4 *>(static_cast<float *>(base) + at);
#pragma unroll
            for (int k = 0; k < N / 4; ++k) dst[k] = f32x4{x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]};
        } else {
            Half v;
#pragma unroll
            for (int k = 0; k < N / 2; ++k) v[k] = pack_bf16x2(x[2 * k], x[2 * k + 1]);
            *reinterpret_cast<Half *>(static_cast<unsigned short *>(base) + at) = v;
        }
    }

    // z: values of N consecutive columns, at element `at` of the output
    __device__ static __forceinline__ void apply(const Epilogue &e, float (&x)[N], void *out, bool out_f32, int64_t at)
    {
        float r[N];
        if (e.residual) {
            if (e.residual_f32) {
                const f32x4 *src = reinterpret_cast<const f32x4 *>(static_cast<const float *>(e.residual) + at);
#pragma unroll
                for (int k = 0; k < N; ++k) r[k] = src[k / 4][k % 4];
            } else {
                const Half v = *reinterpret_cast<const Half *>(static_cast<const unsigned short *>(e.residual) + at);
#pragma unroll
                for (int k = 0; k < N; ++k) r[k] = __uint_as_float(k % 2 ? v[k / 2] & 0xffff0000u : v[k / 2] << 16);
            }
        }
        if (e.z) put(e.z, e.z_f32, at, x);
        activate<N>(e.act, x);
        if (e.residual) {
#pragma unroll
            for (int k = 0; k < N; ++k) x[k] += r[k];
        }
        put(out, out_f32, at, x);
    }

    // Element by element, where rows of the output's placement are not whole runs: columns col ... below `extent`.
    __device__ static __forceinline__ void apply_some(const Epilogue &e, float (&x)[N], void *out, bool out_f32, int64_t row_off, const AxisMap &c_n,
                                                      int col, int extent)
    {
#pragma unroll 1
        for (int k = 0; k < N && col + k < extent; ++k) {
            const int64_t at = row_off + axis_offset_fast(c_n, col + k);
            const float y = epilogue_element(e, x[0], at);
            if (out_f32) static_cast<float *>(out)[at] = y;
            else static_cast<unsigned short *>(out)[at] = f32_to_bf16_bits(y);
            // (rolled up, the next value moves to the front: a register cannot be chosen by a number)
#pragma unroll
            for (int i = 0; i + 1 < N; ++i) x[i] = x[i + 1];
        }
    }
};

// Output stage of a wavefront's NBM x NBN accumulator blocks of SIDE x SIDE with what follows the product, through a strip of LDS of
// its own in fp32: HR rows of JH blocks at a time, of which a lane reads CW consecutive columns of a row.  A lane's accumulator
// holds row lane % SIDE and columns 8 (v / 4) + 4 (lane / SIDE) + v % 4 of a block.  The 16-byte slots of a strip row are permuted
// by the row, so that neither side has bank conflicts.
template <int SIDE, typename Acc, int NBM, int NBN> struct TileEpilogue {
    static constexpr int VALS = SIDE * SIDE / 64;
    // strips of 16 x 64 (whole cache lines of bf16 results), 32 x 32 where a wavefront has one block a row, 16 x 16 of small tiles
    static constexpr int JH = SIDE == 32 && NBN % 2 == 0 ? 2 : 1, HR = JH == 2 ? 16 : SIDE, CW = SIDE == 32 ? 8 : 4;
    static constexpr int COLS = JH * SIDE, ROWB = COLS * 4, LPR = COLS / CW, RPP = 64 / LPR, SLOTS = ROWB / 16;
    static constexpr int BYTES = HR * ROWB;
    static_assert(HR % RPP == 0, "whole passes");

    __device__ static __forceinline__ int perm(int row) { return (ROWB >= 256 ? row * (ROWB / 256) : row / (256 / ROWB)) % SLOTS; }

    static constexpr int HALVES = SIDE / HR, STRIPS = (NBN / JH) * NBM * HALVES;

    // Accumulators of strip number S (column blocks, then block rows, then halves of them) into LDS
    template <int S> __device__ static __forceinline__ void write(const Acc (&acc)[NBM][NBN], char *strip, int g, int in_side)
    {
        constexpr int h = S % HALVES, i = S / HALVES % NBM, j0 = S / HALVES / NBM * JH;
        // (the statement ties these writes to their strip: merged with the other strips' the accumulators would be chosen by a
        // number, that is from memory)
        asm volatile("; strip %0" : : "n"(S));
        if (HALVES > 1 && in_side / HR != h) return;
        const int row = in_side % HR;
#pragma unroll
        for (int j = 0; j < JH; ++j)
#pragma unroll
            for (int v = 0; v < VALS; v += 4) {
                const int slot = (j * SIDE + 2 * v + 4 * g) / 4;
                *reinterpret_cast<f32x4 *>(strip + row * ROWB + ((slot ^ perm(row)) * 16)) =
                    f32x4{acc[i][j0 + j][v], acc[i][j0 + j][v + 1], acc[i][j0 + j][v + 2], acc[i][j0 + j][v + 3]};
            }
        asm volatile("; strip %0" : : "n"(S));
    }
    template <int S> __device__ static __forceinline__ void write_one_of(int s, const Acc (&acc)[NBM][NBN], char *strip, int g, int in_side)
    {
        if constexpr (S < STRIPS) {
            if (s == S) write<S>(acc, strip, g, in_side);
            else write_one_of<S + 1>(s, acc, strip, g, in_side);
        }
    }

    // Parameters `p` (of either kernel family): C, out_f32, alpha, maps, Mo, No, e, piece, bias_piece.  `strip`: BYTES of LDS.
    // A loop over the strips that is not unrolled: only the accumulators' registers are named in the code, and what follows
    // the product is there once (unrolled, it is many times the instruction cache).
    template <typename P> __device__ static __forceinline__ void store(const P &p, const Acc (&acc)[NBM][NBN], char *strip, int m0, int n0, int lane)
    {
        asm volatile("" : "+v"(lane));      // (opaque: formed ahead of the K loop, the addresses below would occupy registers all through it)
        const int g = lane / SIDE, in_side = lane % SIDE, rd_row = lane / LPR, rd_col = (lane % LPR) * CW;
#pragma unroll 1
        for (int s = 0; s < STRIPS; ++s) {
            write_one_of<0>(s, acc, strip, g, in_side);
            const int first = m0 + s / HALVES % NBM * SIDE + s % HALVES * HR, col = n0 + s / HALVES / NBM * COLS + rd_col;
            if (col >= p.No) continue;
            const int64_t col_off = axis_offset_fast(p.maps.c_n, col);
            const bool whole = p.piece >= CW;
            float bias[CW];
            if (p.maps.bias == nullptr) {
#pragma unroll
                for (int e = 0; e < CW; ++e) bias[e] = 0.f;
            } else if (p.bias_piece >= CW) {
                const f32x4 *src = reinterpret_cast<const f32x4 *>(p.maps.bias + axis_offset_fast(p.maps.bias_n, col));
#pragma unroll
                for (int e = 0; e < CW; ++e) bias[e] = src[e / 4][e % 4];
            } else {
#pragma unroll
                for (int e = 0; e < CW; ++e) bias[e] = p.maps.bias[axis_offset_fast(p.maps.bias_n, min(col + e, p.No - 1))];
            }
#pragma unroll 1
            for (int r = rd_row; r < HR && first + r < p.Mo; r += RPP) {
                const int64_t row_off = axis_offset_fast(p.maps.c_m, first + r);
                float x[CW];
#pragma unroll
                for (int k = 0; k < CW / 4; ++k) {
                    const f32x4 t = *reinterpret_cast<const f32x4 *>(strip + r * ROWB + (((rd_col / 4 + k) ^ perm(r)) * 16));
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[4 * k + e] = t[e] * p.alpha + bias[4 * k + e];
                }
                if (whole) EpilogueRun<CW>::apply(p.e, x, p.C, p.out_f32, row_off + col_off);
                else EpilogueRun<CW>::apply_some(p.e, x, p.C, p.out_f32, row_off, p.maps.c_n, col, p.No);
            }
        }
    }
};

}  // namespace cube3d
