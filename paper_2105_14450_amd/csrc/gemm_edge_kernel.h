// Text of the product kernel for any size (gemm_edge.h), which includes it twice: as the product alone and with what follows it
// in the output stage.  One text, and not one function that both kernels call: behind a call the compiler keeps all
// arguments in registers from the start, and the kernels that load single elements spill.
template <typename E, int T, int GB, bool AK, bool BK>
__global__ __launch_bounds__(256, T == 128 || GB == 1 ? 2 : 3) void CUBE3D_EDGE_KERNEL(const CUBE3D_EDGE_PARAMS p)
{
    typedef Operand<E, T, GB, AK> OA;
    typedef Operand<E, T, GB, BK> OB;
    typedef typename Instr<E, T>::M M;
    typedef typename M::Frag Frag;
    typedef typename M::Acc Acc;
    constexpr int SIDE = M::SIDE, VALS = SIDE * SIDE / 64;      // an accumulator block and a lane's values of it
    constexpr int KW = Instr<E, T>::KW, W = KW == 1 ? T / 2 : T, NB = W / SIDE;
    constexpr int TK = OA::TK, STEPS = TK / M::KSTEP, D = depth(T, GB);
    constexpr int STAGE = OA::BYTES + OB::BYTES;
    constexpr int STRIP = W * 4 + 16;                   // bytes of a staged output row (fp32, padded)
    constexpr int LDS = 2 * STAGE > 4 * SIDE * STRIP ? 2 * STAGE : 4 * SIDE * STRIP;   // the strips reuse the K-tile buffers
    static_assert(STEPS % KW == 0, "whole k-steps per wavefront");
    __shared__ __attribute__((aligned(1024))) char smem[LDS];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = KW == 1 ? (wave >> 1) * W : 0, wn = KW == 1 ? (wave & 1) * W : 0, g = lane / SIDE, in_side = lane % SIDE;

    // Workgroup ids go round robin over the 8 XCDs: hand every XCD one contiguous run of tiles, so that the
    // panels its workgroups share come through one L2.
    const int total = gridDim.x, id = blockIdx.x, xcd = id % 8, each = total / 8, more = total % 8;
    const int item = xcd * each + min(xcd, more) + id / 8;
    const int tiles = p.tiles_m * p.tiles_n, batch = item / tiles, tile = item - batch * tiles;
    const int per_group = p.group_m * p.tiles_n, gid = tile / per_group, first_m = gid * p.group_m;
    const int gsz = min(p.tiles_m - first_m, p.group_m), in_group = tile - gid * per_group;
    const int m0 = (first_m + in_group % gsz) * T, n0 = (in_group / gsz) * T;

    OA a;
    OB b;
    a.init(p.A + batch * p.sA, p.maps.a_mn, p.maps.a_k, m0, p.Mo, p.Kc, tid);
    b.init(p.B + batch * p.sB, p.maps.b_mn, p.maps.b_k, n0, p.No, p.Kc, tid);
    typename OA::P va[D][OA::NV];
    typename OB::P vb[D][OB::NV];

    Acc acc[NB][NB];
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int v = 0; v < VALS; ++v) acc[i][j][v] = 0.f;

    auto frag_a = [&](const char *ta, int i, int step) -> Frag {
        if constexpr (AK) {
            const int row = wm + SIDE * i + in_side;
            return M::read_k(ta + row * BKB, (row / 2) % 8, step, g);
        } else return M::template read_mn<OA::RB>(ta, lane, wm + SIDE * i, step);
    };
    auto frag_b = [&](const char *ta, int j, int step) -> Frag {
        const char *tb = ta + OA::BYTES;
        if constexpr (BK) {
            const int row = wn + SIDE * j + in_side;
            return M::read_k(tb + row * BKB, (row / 2) % 8, step, g);
        } else return M::template read_mn<OB::RB>(tb, lane, wn + SIDE * j, step);
    };
    // The MFMAs of one K-tile, with `moves` (the LDS writes and loads of later K-tiles) behind the fragment
    // reads of the first EARLY steps: a wavefront that is alone on its SIMD has its MFMAs wait for those
    // reads only, and not for the writes.
    constexpr int MY_STEPS = STEPS / KW, EARLY = T == 128 ? 1 : MY_STEPS < 4 ? MY_STEPS : 4;
    constexpr bool MOVES_LAST = T == 128;
    auto compute = [&](const char *ta, auto &&moves) {
        Frag fa[EARLY][NB], fb[EARLY][NB];
        auto step_no = [&](int s) { return KW == 1 ? s : wave * MY_STEPS + s; };
        auto read = [&](int s) {
#pragma unroll
            for (int i = 0; i < NB; ++i) fa[s % EARLY][i] = frag_a(ta, i, step_no(s));
#pragma unroll
            for (int j = 0; j < NB; ++j) fb[s % EARLY][j] = frag_b(ta, j, step_no(s));
        };
#pragma unroll
        for (int s = 0; s < EARLY; ++s) read(s);
        if constexpr (!MOVES_LAST) moves();
#pragma unroll
        for (int s = 0; s < MY_STEPS; ++s) {
            if (s >= EARLY) read(s);
#pragma unroll
            for (int x = 0; x < M::MFMAS; ++x)      // (consecutive MFMAs on different accumulators where there are several)
#pragma unroll
                for (int i = 0; i < NB; ++i)
#pragma unroll
                    for (int j = 0; j < NB; ++j) acc[i][j] = M::mfma(fb[s % EARLY][j], fa[s % EARLY][i], acc[i][j], x);
        }
        if constexpr (MOVES_LAST) moves();
    };

    const int full = p.Kc / TK, ntiles = (p.Kc + TK - 1) / TK;
    // K-tile kt travels in register set kt % D and sits in LDS buffer kt & 1.  The loop proper takes only
    // whole K-tiles and has no branch around a load, so that each wait covers one K-tile's loads and leaves the
    // younger ones in flight; the last K-tiles look at every piece's bounds (beyond the last one they load
    // element 0 and write zeros).
    auto load = [&](auto tail, int d) {
        a.template load<tail.value>(va[d], p.maps.a_k, p.step_a, p.Kc);
        b.template load<tail.value>(vb[d], p.maps.b_k, p.step_b, p.Kc);
    };
    // (an even number of K-tiles per pass: buffer and LDS addresses are constants)
    auto buffer = [&](int d, int kt) { return smem + (D % 2 == 0 ? d & 1 : kt & 1) * STAGE; };
    auto store = [&](auto tail, int d, int kt) {
        char *t = buffer(d, kt);
        a.template store<tail.value>(va[d], t, kt * TK, p.Kc);
        b.template store<tail.value>(vb[d], t + OA::BYTES, kt * TK, p.Kc);
    };
    const std::integral_constant<bool, false> whole{};
    const std::integral_constant<bool, true> tail{};
#pragma unroll
    for (int d = 0; d < D; ++d) load(tail, d);
    store(tail, 0, 0);
    load(tail, 0);
    __syncthreads();
    int k0 = 0;
    for (; k0 + 2 * D < full; k0 += D) {
#pragma unroll
        for (int d = 0; d < D; ++d) {
            // (the buffer of K-tile kt + 1 was last read before the previous barrier)
            const int kt = k0 + d;
            compute(buffer(d, kt), [&] {
                store(whole, (d + 1) % D, kt + 1);
                load(whole, (d + 1) % D);
            });
            __syncthreads();
        }
    }
    for (; k0 < ntiles; k0 += D) {
#pragma unroll
        for (int d = 0; d < D; ++d) {
            const int kt = k0 + d;
            if (kt < ntiles)
                compute(buffer(d, kt), [&] {
                    store(tail, (d + 1) % D, kt + 1);
                    load(tail, (d + 1) % D);
                });
            __syncthreads();
        }
    }

    // Output.  A lane's accumulator holds row lane % SIDE and columns 8 (v / 4) + 4 (lane / SIDE) + v % 4 of its
    // block (operands exchanged in the MFMA): one strip of SIDE rows at a time goes through LDS as fp32 so that
    // a lane stores 16 consecutive bytes of a row.  Where four wavefronts share the tile their strips are
    // added in ascending order, each wavefront a quarter of the rows.
    char *strip = smem + wave * SIDE * STRIP;
#if CUBE3D_EDGE_EPILOGUE
    const int run = 8;                                   // columns per lane, whatever the result's type
#else
    const int run = p.out_f32 ? 4 : 8;                   // columns per 16-byte store
#endif
    const int lpr = W / run;                             // lanes per row: a power of two
    const int lcol = (lane % lpr) * run, col = n0 + wn + lcol;
    float bias[8];
    const bool has_bias = p.maps.bias != nullptr;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        bias[e] = (has_bias && e < run && col + e < p.No) ? p.maps.bias[axis_offset_fast(p.maps.bias_n, col + e)] : 0.f;
#if !CUBE3D_EDGE_EPILOGUE
    const int es = p.out_f32 ? 4 : 2;
#endif
    char *C = p.C + batch * p.sC;
    const int64_t col_off = col < p.No ? axis_offset_fast(p.maps.c_n, col) : 0;
#pragma unroll
    for (int i = 0; i < NB; ++i) {
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int v = 0; v < VALS; v += 4) {
                f32x4 w;
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = acc[i][j][v + e];
                *reinterpret_cast<f32x4 *>(strip + in_side * STRIP + (SIDE * j + 2 * v + 4 * g) * 4) = w;
            }
        __syncthreads();
        const int r_first = KW == 1 ? 0 : wave * (SIDE / KW), r_end = r_first + SIDE / KW;
        for (int r = r_first + lane / lpr; r < r_end; r += 64 / lpr) {
            const int row = m0 + wm + SIDE * i + r;
            if (row >= p.Mo || col >= p.No) continue;
            const int64_t row_off = axis_offset_fast(p.maps.c_m, row);
            float x[8];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
#if !CUBE3D_EDGE_EPILOGUE
                if (half && p.out_f32) break;
#endif
                const char *src = (KW == 1 ? strip : smem) + r * STRIP + lcol * 4 + half * 16;
                f32x4 t = *reinterpret_cast<const f32x4 *>(src);
#pragma unroll
                for (int k = 1; k < KW; ++k) t += *reinterpret_cast<const f32x4 *>(src + k * SIDE * STRIP);
#pragma unroll
                for (int e = 0; e < 4; ++e) x[4 * half + e] = t[e] * p.alpha + bias[4 * half + e];
            }
#if CUBE3D_EDGE_EPILOGUE
            if (p.piece == 8) {
                EpilogueRun<8>::Residual residual;
                EpilogueRun<8>::load<ANY>(p.e, row_off + col_off, residual);
                EpilogueRun<8>::apply<ANY>(p.e, x, residual, C, p.out_f32, row_off + col_off);
            }
            else EpilogueRun<8>::apply_some(p.e, x, C, p.out_f32, row_off, p.maps.c_n, col, p.No);
#else
            if (p.out_wide) {
                char *dst = C + (row_off + col_off) * es;
                if (p.out_f32) *reinterpret_cast<f32x4 *>(dst) = f32x4{x[0], x[1], x[2], x[3]};
                else *reinterpret_cast<i32x4 *>(dst) = i32x4{(int)pack_bf16x2(x[0], x[1]), (int)pack_bf16x2(x[2], x[3]),
                                                             (int)pack_bf16x2(x[4], x[5]), (int)pack_bf16x2(x[6], x[7])};
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (e < run && col + e < p.No) {
                        const int64_t at = row_off + axis_offset_fast(p.maps.c_n, col + e);
                        if (p.out_f32) reinterpret_cast<float *>(C)[at] = x[e];
                        else reinterpret_cast<unsigned short *>(C)[at] = f32_to_bf16_bits(x[e]);
                    }
            }
#endif
        }
        __syncthreads();
    }
}
