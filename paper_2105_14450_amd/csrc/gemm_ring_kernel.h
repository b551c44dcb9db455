// Text of the ring kernel (gemm_ring.h), which includes it twice: as the product alone and with what follows it in the output
// stage (one text and not one function, as in gemm_edge_kernel.h).
// Persistent workgroups: workgroup w makes the tiles w, w + gridDim.x, ...  STREAM: streaming stores of the output.
template <typename E, int TM, int TN, int NST, bool AK, bool BK, bool STREAM>
__global__ __launch_bounds__(512, 2 * ring_per_cu(TM, TN, NST)) void CUBE3D_RING_KERNEL(const CUBE3D_RING_PARAMS p)
{
    constexpr int BKB = ring_ktile_bytes(TN);
    typedef RingOperand<E, TM, BKB, AK> OA;
    typedef RingOperand<E, TN, BKB, BK> OB;
    typedef typename RingInstr<E, TM>::M M;
    typedef typename M::Frag Frag;
    typedef typename M::Acc Acc;
    constexpr int SIDE = M::SIDE, VALS = SIDE * SIDE / 64, WM = TM / 2, WN = TN / 2, NBM = WM / SIDE, NBN = WN / SIDE;
    constexpr int STEPS = OA::TK / M::KSTEP;
    // Fragments are read one unit ahead: a K-tile, or a k-step of the largest tiles, whose accumulators leave less room.
    constexpr int USTEPS = TM * TN > 128 * 128 ? 1 : STEPS, UNITS = STEPS / USTEPS;
    constexpr int STAGE = OA::BYTES + OB::BYTES, LPT = OA::LOADS + OB::LOADS;
    static_assert(UNITS == 1 || UNITS % 2 == 0, "the fragment buffers alternate per unit");
    static_assert((NST - 1) * LPT <= 63, "vmcnt range");
    constexpr int STRIP = ring_strip(TN);
    static_assert(RingOutput<M, NBM, NBN, 2, false, STREAM>::BYTES <= STRIP && RingOutput<M, NBM, NBN, 4, false, STREAM>::BYTES <= STRIP, "room for the output strips");
#if CUBE3D_RING_EPILOGUE
    typedef TileEpilogue<SIDE, Acc, NBM, NBN, STRIP, (NBM * NBN < 8), STREAM> Output;
    static_assert(Output::BYTES <= STRIP, "room for the output strips");
#else
    typedef std::integral_constant<int, 2> I2;
    typedef std::integral_constant<int, 4> I4;
#endif
    __shared__ __attribute__((aligned(1024))) char smem[ring_lds(TM, TN, NST)];

    const int tid = threadIdx.x, lane = tid & 63, wave8 = __builtin_amdgcn_readfirstlane(tid >> 6), wave = wave8 % 4;
    const int ntiles = (p.Kc + OA::TK - 1) / OA::TK, my_items = (p.items - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x;

    // K-tile c (counted over all items of the workgroup) sits in stage c % NST.  Behind barrier c, K-tile c + 1 has landed and
    // everybody has the fragments of c: K-tile c + NST goes to their stage.
    if (wave8 >= 4) {
        OA a;
        OB b;
        const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char *)smem + wave * 1024;
        uint64_t one_shard = 0;        // bit t: K-tile t of the current 64 lies in one shard of either operand
        int item = blockIdx.x, kt = 0;                  // next K-tile to load
        unsigned to = lds0;                             // and its stage
        auto start_item = [&]() {
            const Place at = place_item(p, item, TM, TN);
            a.init(p.A + at.batch * p.sA, p.maps.a_mn, p.maps.a_k, at.m0, p.Mo, wave, lane);
            b.init(p.B + at.batch * p.sB, p.maps.b_mn, p.maps.b_k, at.n0, p.No, wave, lane);
        };
        auto next_stage = [&]() { to = to + STAGE == lds0 + NST * STAGE ? lds0 : to + STAGE; };
        // any K-tile (behind the last item: beyond the contraction, zeros)
        auto load = [&]() {
            const int t = kt % 64;
            if (t == 0) {
                const bool whole_a = a.look_ahead(p.maps.a_k, p.Kc, kt, lane), whole_b = b.look_ahead(p.maps.b_k, p.Kc, kt, lane);
                one_shard = __ballot(whole_a && whole_b);
            }
            a.load_any(t, to);
            b.load_any(t, to + OA::BYTES);
            next_stage();
            if (++kt == ntiles && item + (int)gridDim.x < p.items) {
                item += gridDim.x;
                kt = 0;
                start_item();
            }
        };
        start_item();
#pragma unroll 1
        for (int s = 0; s < NST - 1; ++s) load();
        ring_barrier<(NST - 2) * LPT>();      // K-tile 0 is there
        load();
        const int total = ntiles * my_items;
        int left = total - NST;        // K-tiles still to load
        while (left > 0) {
            // a run of K-tiles in one shard each, but not the first of 64 or the last of the item
            const int t = kt % 64;
            int run = t == 0 ? 0 : min(min(__builtin_ctzll(~(one_shard >> t) | 1ull << (64 - t)), ntiles - 1 - kt), left);
            left -= run;
            kt += run;
            for (int u = t; run > 0; --run, ++u) {
                ring_barrier<(NST - 2) * LPT>();
                a.load_one_shard(u, to);
                b.load_one_shard(u, to + OA::BYTES);
                next_stage();
            }
            if (left > 0) {
                ring_barrier<(NST - 2) * LPT>();
                load();
                --left;
            }
        }
        ring_drain<NST, LPT>(total);
        ring_wait<0>();     // (fewer K-tiles than stages) nothing may arrive behind the workgroup's end
        return;
    }

    const int wm = (wave >> 1) * WM, wn = (wave & 1) * WN, g = lane / SIDE, in_side = lane % SIDE;
    char *strip = smem + NST * STAGE + wave * STRIP;
    Acc acc[NBM][NBN];
    Frag fa[2][USTEPS][NBM], fb[2][USTEPS][NBN];
    int stage = 0;
    // fragment r of a unit, A and B alternately in the order in which the MFMAs need them
    constexpr int FRAGS = USTEPS * (NBM + NBN);
    auto read = [&](int r, int buf, const char *ta, int unit) {
        const char *tb = ta + OA::BYTES;
        const int s = r / (NBM + NBN), x = r % (NBM + NBN), step = unit * USTEPS + s;
        if (x == 0 || x > NBN) {
            const int i = x == 0 ? 0 : x - NBN;
            if constexpr (AK) fa[buf][s][i] = M::read_k(ta + (wm + in_side) * BKB + i * SIDE * BKB, OA::swz(in_side), step, g);
            else fa[buf][s][i] = M::template read_mn<OA::RB>(ta, lane, wm + SIDE * i, step);
        } else {
            const int j = x - 1;
            if constexpr (BK) fb[buf][s][j] = M::read_k(tb + (wn + in_side) * BKB + j * SIDE * BKB, OB::swz(in_side), step, g);
            else fb[buf][s][j] = M::template read_mn<OB::RB>(tb, lane, wn + SIDE * j, step);
        }
    };
    // The MFMAs of a unit, with the reads of the next one ahead of them (one accumulator: the MFMAs wait for each other
    // anyway) or dealt out behind them, all but the last few.
    constexpr int MFMAS = USTEPS * M::MFMAS * NBM * NBN, GAPS = NBM * NBN == 1 ? 0 : MFMAS > 8 ? MFMAS - 4 : MFMAS > 4 ? MFMAS - 2 : MFMAS;
    auto multiply = [&](int buf, const char *next, int next_unit) {
        if constexpr (GAPS == 0) {
#pragma unroll
            for (int r = 0; r < FRAGS; ++r) read(r, buf ^ 1, next, next_unit);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int m = 0; m < MFMAS; ++m) {
            const int s = m / (M::MFMAS * NBM * NBN), x = m / (NBM * NBN) % M::MFMAS, i = m / NBN % NBM, j = m % NBN;
            acc[i][j] = M::mfma(fb[buf][s][j], fa[buf][s][i], acc[i][j], x);
            if constexpr (GAPS > 0) {
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int r = 0; r < FRAGS; ++r)
                    if (r * GAPS / FRAGS == m) read(r, buf ^ 1, next, next_unit);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    };
#if !CUBE3D_RING_EPILOGUE
    const std::true_type yes{};
    const std::false_type no{};
#endif
    // K-tile with its first unit's fragments in buffer `buf`; moves to the next stage
    auto k_tile = [&](auto buf_c) {
        constexpr int buf = decltype(buf_c)::value;
        const char *here = smem + stage * STAGE;
#pragma unroll
        for (int u = 0; u < UNITS - 1; ++u) multiply((buf + u) & 1, here, u + 1);
        __builtin_amdgcn_sched_barrier(0);
        ring_barrier<0>();
        stage = stage + 1 == NST ? 0 : stage + 1;
        multiply((buf + UNITS - 1) & 1, smem + stage * STAGE, 0);
        __builtin_amdgcn_sched_barrier(0);
    };

    ring_barrier<0>();
    for (int item = blockIdx.x; item < p.items; item += gridDim.x) {
#pragma unroll
        for (int i = 0; i < NBM; ++i)
#pragma unroll
            for (int j = 0; j < NBN; ++j)
#pragma unroll
                for (int v = 0; v < VALS; ++v) acc[i][j][v] = 0.f;
#pragma unroll
        for (int r = 0; r < FRAGS; ++r) read(r, 0, smem + stage * STAGE, 0);
        if constexpr (UNITS == 1) {
            for (int kt = 0; kt < ntiles; kt += 2) {
                k_tile(std::integral_constant<int, 0>{});
                if (kt + 1 < ntiles) k_tile(std::integral_constant<int, 1>{});
            }
        } else {
            for (int kt = 0; kt < ntiles; ++kt) k_tile(std::integral_constant<int, 0>{});
        }
        const Place at = place_item(p, item, TM, TN);
#if CUBE3D_RING_EPILOGUE
        Output::store(p, acc, strip, at.m0 + wm, at.n0 + wn, lane);
#else
        auto store = [&](auto oes, auto bias) {
            RingOutput<M, NBM, NBN, decltype(oes)::value, decltype(bias)::value, STREAM>::store(p, acc, strip, at.m0 + wm, at.n0 + wn, at.batch, lane);
        };
        // (a bias comes with the layout of the forward product, K-major times MN-major)
        if (AK && !BK && p.maps.bias != nullptr) p.out_f32 ? store(I4{}, yes) : store(I2{}, yes);
        else p.out_f32 ? store(I4{}, no) : store(I2{}, no);
#endif
    }
}
