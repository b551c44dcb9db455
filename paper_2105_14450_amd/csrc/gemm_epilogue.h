// What follows a product of the forward layout (struct Epilogue), on runs of consecutive output columns: the output stages of the
// product kernels hand over fp32 values row by row, and Z, the residual and the result move in whole 16-byte (bf16 runs of four: 8-byte)
// accesses wherever the output's placement allows.
#pragma once
#include "activation.h"

namespace cube3d {

// Eight fp8 codes as bf16, exactly
__device__ __forceinline__ bf16x8 widen_fp8(i32x2 codes)
{
    i32x4 wide;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        wide[2 * i] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)codes[i], 1.f, false));
        wide[2 * i + 1] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)codes[i], 1.f, true));
    }
    return __builtin_bit_cast(bf16x8, wide);
}

// GELU where nothing hides its arithmetic: z Phi(z) = max(z, 0) - t Phi(-t) with t = |z|, and Phi(-t) = 2^(-p(t)), p(t) = 1 + t
// times a degree-6 polynomial (equal-ripple fit of -log2 Phi(-t) on [0, 6]; beyond, p keeps growing: 30 at 6).  15 issue slots an
// element (v_exp_f32 counts four) for the 25 of act_value, which fp32 results take.  t Phi(-t) is within 7e-7 here; up to t = 6 Phi(-t) is
// within 8e-6 of itself, a 240th of half a bf16 step (2^-9 of a value at least); beyond, where t Phi(-t) is below 6e-9, it is within 5e-14
// (of itself 3e-4 at 7, and from 8 on more than half a step).  t is cut at 64 on the upper side, where Phi(-t) is zero, so that
// +infinity stays itself; -infinity gives NaN, as z Phi(z) does everywhere else, and NaN passes the comparison by.
__device__ __forceinline__ float gelu_short(float z)
{
    const float t = z > 64.f ? 64.f : fabsf(z);
    float s = 1.793782303e-06f;
    s = fmaf(s, t, -6.072620090e-05f);
    s = fmaf(s, t, 9.231860749e-04f);
    s = fmaf(s, t, -8.476848714e-03f);
    s = fmaf(s, t, 5.389093980e-02f);
    s = fmaf(s, t, 4.585415721e-01f);
    s = fmaf(s, t, 1.151214361e+00f);
    return fmaf(-t, __builtin_amdgcn_exp2f(-fmaf(s, t, 1.f)), fmaxf(z, 0.f));
}

// The activation is looked up per run: one uniform branch for eight elements, and no variant of a product kernel per activation.
template <int N> __device__ __forceinline__ void activate(int act, bool exact, float (&x)[N])
{
    if (act == CUBE3D_ACT_GELU) {
        if (exact) {
#pragma unroll
            for (int e = 0; e < N; ++e) x[e] = epilogue_act<CUBE3D_ACT_GELU>(x[e]);
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) x[e] = gelu_short(x[e]);
        }
    } else if (act == CUBE3D_ACT_RELU) {
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = epilogue_act<CUBE3D_ACT_RELU>(x[e]);
    }
}

// Variants of the output stage: bf16 results, rows in whole runs, and beside them nothing, Z in bf16, a residual in bf16 or in fp32; or
// whatever the call has.
enum EpilogueKind { PLAIN, WITH_Z, BF16_RESIDUAL, F32_RESIDUAL, ANY };

// STREAM: results past the caches (as the plain kernels do: always in the tuned one, large results in the ring).
template <int N, bool STREAM = false> struct EpilogueRun {
    static_assert(N == 4 || N == 8, "whole 16-byte accesses of fp32");
    typedef unsigned Half __attribute__((ext_vector_type(N / 2)));     // N bf16 values
    struct Residual {
        f32x4 wide[N / 4];
        Half half;
    };

    __device__ static __forceinline__ void put(void *base, bool f32, int64_t at, const float (&x)[N])
    {
        if (f32) {
            f32x4 *dst = reinterpret_cast<f32x4 *>(static_cast<float *>(base) + at);
#pragma unroll
            for (int k = 0; k < N / 4; ++k) {
                const f32x4 v = {x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]};
                if (STREAM) __builtin_nontemporal_store(v, dst + k);
                else dst[k] = v;
            }
        } else {
            Half v;
#pragma unroll
            for (int k = 0; k < N / 2; ++k) v[k] = pack_bf16x2(x[2 * k], x[2 * k + 1]);
            Half *dst = reinterpret_cast<Half *>(static_cast<unsigned short *>(base) + at);
            if (STREAM) __builtin_nontemporal_store(v, dst);
            else *dst = v;
        }
    }

    // The residual of N consecutive columns, at element `at` of the output
    template <EpilogueKind KIND> __device__ static __forceinline__ void load(const Epilogue &e, int64_t at, Residual &r)
    {
        if (KIND == F32_RESIDUAL || (KIND == ANY && e.residual && e.residual_f32)) {
            const f32x4 *src = reinterpret_cast<const f32x4 *>(static_cast<const float *>(e.residual) + at);
#pragma unroll
            for (int k = 0; k < N / 4; ++k) r.wide[k] = src[k];
        }
        if (KIND == BF16_RESIDUAL || (KIND == ANY && e.residual && !e.residual_f32))
            r.half = *reinterpret_cast<const Half *>(static_cast<const unsigned short *>(e.residual) + at);
    }

    // x: values of Z at element `at`
    template <EpilogueKind KIND>
    __device__ static __forceinline__ void apply(const Epilogue &e, float (&x)[N], const Residual &r, void *out, bool out_f32, int64_t at)
    {
        if (KIND == WITH_Z || (KIND == ANY && e.z)) put(e.z, KIND == ANY && e.z_f32, at, x);
        activate<N>(e.act, KIND == ANY && out_f32, x);
        if (KIND == F32_RESIDUAL || (KIND == ANY && e.residual && e.residual_f32)) {
#pragma unroll
            for (int k = 0; k < N; ++k) x[k] += r.wide[k / 4][k % 4];
        }
        if (KIND == BF16_RESIDUAL || (KIND == ANY && e.residual && !e.residual_f32)) {
#pragma unroll
            for (int k = 0; k < N; ++k) x[k] += __uint_as_float(k % 2 ? r.half[k / 2] & 0xffff0000u : r.half[k / 2] << 16);
        }
        put(out, KIND == ANY && out_f32, at, x);
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
// ROOM: bytes of LDS per wavefront.  A strip's values and residuals are read ahead of the next strip's writes.  Not AHEAD: kernels
// without registers to spare, where this holds for one block column and for two without a residual; two with one read a strip's
// residuals together, and what is left reads pass by pass.  us for read ahead or together / pass by pass: 2997 x 1152 x 4608 with a
// bf16 residual 50 / 54, 4635 x 576 x 4032 55 / 60, 6000 x 512 x 1000 20.6 / 22.
template <int SIDE, typename Acc, int NBM, int NBN, int ROOM, bool AHEAD, bool STREAM> struct TileEpilogue {
    static constexpr int VALS = SIDE * SIDE / 64;
    // strips 64 columns wide (whole cache lines of bf16 results), 32 where a wavefront has one block a row, 16 of small tiles
    static constexpr int JH = SIDE == 32 && NBN % 2 == 0 ? 2 : 1;
    static constexpr int COLS = JH * SIDE, ROWB = COLS * 4, SLOTS = ROWB / 16, HR = ROOM / ROWB < SIDE ? ROOM / ROWB : SIDE;
    static_assert(SIDE % HR == 0 && HR >= 16, "whole strips");
    static constexpr int BYTES = HR * ROWB;

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
    template <int LO, int HI> __device__ static __forceinline__ void write_one_of(int s, const Acc (&acc)[NBM][NBN], char *strip, int g, int in_side)
    {
        if constexpr (HI - LO == 1) write<LO>(acc, strip, g, in_side);
        else if (s < (LO + HI) / 2) write_one_of<LO, (LO + HI) / 2>(s, acc, strip, g, in_side);
        else write_one_of<(LO + HI) / 2, HI>(s, acc, strip, g, in_side);
    }

    // Parameters `p` (of either kernel family): C, out_f32, alpha, maps, Mo, No, e, piece, bias_piece.  `strip`: BYTES of LDS.
    // A loop over the strips that is not unrolled: only the accumulators' registers are named in the code, and what follows
    // the product is there once (unrolled, it is many times the instruction cache).  A strip's reads are issued ahead of the next
    // one's writes (LDS keeps a wavefront's accesses in order), which pass while the reads' values are on their way.
    // The usual combinations have loops of their own, in which neither a load nor a store depends on a condition: memory operations
    // complete in order, so a wait for a load is a wait for the stores ahead of it, and only where the compiler can count
    // what lies between does it wait for no more than that.  The biases are there before the first store for the same reason, and a
    // strip's residuals are loaded ahead of the previous strip's stores.
    template <typename P> __device__ static __forceinline__ void store(const P &p, const Acc (&acc)[NBM][NBN], char *strip, int m0, int n0, int lane)
    {
        constexpr int CW = SIDE == 32 ? 8 : 4;
        if (p.out_f32 || p.piece < CW || (p.maps.bias && p.bias_piece < CW) || (p.e.z && (p.e.z_f32 || p.e.residual)))
            store_kind<ANY, AHEAD ? CW : 4>(p, acc, strip, m0, n0, lane);
        else if (p.e.z) store_kind<WITH_Z, CW>(p, acc, strip, m0, n0, lane);
        else if (!p.e.residual) store_kind<PLAIN, CW>(p, acc, strip, m0, n0, lane);
        else if (p.e.residual_f32) store_kind<F32_RESIDUAL, CW>(p, acc, strip, m0, n0, lane);
        else store_kind<BF16_RESIDUAL, CW>(p, acc, strip, m0, n0, lane);
    }
    // CW: consecutive columns of a row that a lane reads
    template <EpilogueKind KIND, int CW, typename P>
    __device__ static __forceinline__ void store_kind(const P &p, const Acc (&acc)[NBM][NBN], char *strip, int m0, int n0, int lane)
    {
        asm volatile("" : "+v"(lane));      // (opaque: formed ahead of the K loop, the addresses below would occupy registers all through it)
        typedef EpilogueRun<CW, STREAM> Run;
        constexpr bool EARLY = AHEAD || KIND == PLAIN || KIND == WITH_Z || (KIND != ANY && NBN / JH == 1);
        constexpr int LPR = COLS / CW, RPP = 64 / LPR;              // lanes per strip row, rows per pass
        const int g = lane / SIDE, in_side = lane % SIDE, rd_row = lane / LPR, rd_col = (lane % LPR) * CW;
        constexpr int PASSES = HR / RPP, GROUP = NBM * HALVES, GROUPS = STRIPS / GROUP;     // strips of a block column
        static_assert(HR % RPP == 0, "whole passes");
        const bool whole = KIND != ANY || p.piece >= CW;
        const int64_t row_step = p.maps.c_m.u;
        float all_bias[GROUPS][CW];
#pragma unroll
        for (int j = 0; j < GROUPS; ++j) {
            const int c = n0 + j * COLS + rd_col;
#pragma unroll
            for (int e = 0; e < CW; ++e) all_bias[j][e] = 0.f;
            if (p.maps.bias == nullptr) continue;
            if (KIND != ANY || p.bias_piece >= CW) {
                const f32x4 *src = reinterpret_cast<const f32x4 *>(p.maps.bias + axis_offset_fast(p.maps.bias_n, c < p.No ? c : 0));
#pragma unroll
                for (int e = 0; e < CW; ++e) all_bias[j][e] = src[e / 4][e % 4];
            } else {
#pragma unroll
                for (int e = 0; e < CW; ++e) all_bias[j][e] = p.maps.bias[axis_offset_fast(p.maps.bias_n, min(c + e, p.No - 1))];
            }
        }
        write<0>(acc, strip, g, in_side);
#pragma unroll
        for (int j = 0; j < GROUPS; ++j)
#pragma unroll
            for (int e = 0; e < CW; ++e) asm volatile("" : "+v"(all_bias[j][e]));      // (waited for here, not in the loop)
        // Where strip s lies: its first row, this lane's column, their offsets.  Inside the output and inside one shard a strip's rows are
        // a fixed distance apart; the others ask the map row by row (a 64-bit multiplication takes 16 cycles, a map three of them).
        int64_t all_cols[GROUPS], pass_row[PASSES];
#pragma unroll
        for (int j = 0; j < GROUPS; ++j) all_cols[j] = axis_offset_fast(p.maps.c_n, max(min(n0 + j * COLS + rd_col, p.No - CW), 0));
#pragma unroll
        for (int ps = 0; ps < PASSES; ++ps) pass_row[ps] = (ps * RPP + rd_row) * row_step;
        struct At {
            int first, col;
            bool simple;
            int64_t first_off, col_off;
        };
        auto place = [&](int s) {
            At x;
            x.first = m0 + s / HALVES % NBM * SIDE + s % HALVES * HR;
            x.col = n0 + s / GROUP * COLS + rd_col;
            const AxisMap &m = p.maps.c_m;
            x.simple = x.first + HR <= p.Mo && x.first - (int)(((uint64_t)(unsigned)x.first * m.M2) >> m.N2) * m.P2 + HR <= m.P2;
            x.first_off = axis_offset_fast(m, x.first);
            x.col_off = all_cols[0];
#pragma unroll
            for (int j = 1; j < GROUPS; ++j)
                if (s / GROUP == j) x.col_off = all_cols[j];
            return x;
        };
        auto offset = [&](const At &x, int ps) {
            return x.col_off + (x.simple ? x.first_off + pass_row[ps]
                                         : axis_offset_fast(p.maps.c_m, min(x.first + ps * RPP + rd_row, p.Mo - 1)));
        };
        constexpr int HELD = EARLY || KIND != ANY ? PASSES : 1;
        typename Run::Residual residual[HELD];
        // (lanes beyond the output load the last row's or the last CW columns)
        auto load = [&](const At &x, int ps, typename Run::Residual &res) {
            if (KIND != PLAIN && KIND != WITH_Z && whole) Run::template load<KIND>(p.e, offset(x, ps), res);
        };
        At here = place(0);
        if constexpr (EARLY) {
#pragma unroll
            for (int ps = 0; ps < PASSES; ++ps) load(here, ps, residual[ps]);
        }
#pragma unroll 1
        for (int s = 0; s < STRIPS; ++s) {
            f32x4 t[HELD][CW / 4];
            auto read = [&](int ps) {
#pragma unroll
                for (int k = 0; k < CW / 4; ++k) {
                    const int r = ps * RPP + rd_row;
                    t[HELD > 1 ? ps : 0][k] = *reinterpret_cast<const f32x4 *>(strip + r * ROWB + (((rd_col / 4 + k) ^ perm(r)) * 16));
                }
            };
            float bias[CW];
#pragma unroll
            for (int e = 0; e < CW; ++e) bias[e] = all_bias[0][e];
#pragma unroll
            for (int j = 1; j < GROUPS; ++j)
                if (s / GROUP == j)
#pragma unroll
                    for (int e = 0; e < CW; ++e) bias[e] = all_bias[j][e];
            auto finish = [&](int ps) {
                const int r = ps * RPP + rd_row;
                float x[CW];
#pragma unroll
                for (int e = 0; e < CW; ++e) x[e] = t[HELD > 1 ? ps : 0][e / 4][e % 4] * p.alpha + bias[e];
                if (here.first + r >= p.Mo || here.col >= p.No) return;
                if (whole) Run::template apply<KIND>(p.e, x, residual[HELD > 1 ? ps : 0], p.C, p.out_f32, offset(here, ps));
                else Run::apply_some(p.e, x, p.C, p.out_f32, offset(here, ps) - here.col_off, p.maps.c_n, here.col, p.No);
            };
            if constexpr (EARLY) {
#pragma unroll
                for (int ps = 0; ps < PASSES; ++ps) read(ps);
                typename Run::Residual next[PASSES];
                const At there = place(min(s + 1, STRIPS - 1));
#pragma unroll
                for (int ps = 0; ps < PASSES; ++ps) load(there, ps, next[ps]);
                if (s + 1 < STRIPS) write_one_of<0, STRIPS>(s + 1, acc, strip, g, in_side);
#pragma unroll
                for (int ps = 0; ps < PASSES; ++ps) finish(ps);
#pragma unroll
                for (int ps = 0; ps < PASSES; ++ps) residual[ps] = next[ps];
                here = there;
            } else {
                if constexpr (KIND != ANY) {
#pragma unroll
                    for (int ps = 0; ps < PASSES; ++ps) load(here, ps, residual[ps]);
#pragma unroll
                    for (int ps = 0; ps < PASSES; ++ps) {
                        read(ps);
                        finish(ps);
                    }
                } else {
#pragma unroll 1
                    for (int ps = 0; ps < PASSES; ++ps) {
                        read(ps);
                        load(here, ps, residual[0]);
                        finish(ps);
                    }
                }
                if (s + 1 < STRIPS) {
                    write_one_of<0, STRIPS>(s + 1, acc, strip, g, in_side);
                    here = place(s + 1);
                }
            }
        }
    }
};

}  // namespace cube3d
