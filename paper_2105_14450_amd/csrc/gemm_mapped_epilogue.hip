// Map-addressed instantiations of the tuned MFMA product kernel with bias, activation and residual in the output stage (the
// forward product over a cube of shards, see gemm_mapped.hip).
#include "gemm_mfma_kernel.h"

namespace cube3d {
using namespace mfk;

namespace {

// (fp8 operands with an fp32 Y or Z are widened, which this kernel does not do)
template <typename E, int T> int launch_epilogue(const GemmArgs &g)
{
    if constexpr (E::ELT > 1)
        if (g.out_dtype == CUBE3D_F32)
            return launch_cfg<E, T, T, 64, 4, true, false, float, true, EpilogueParams>(g, 1, g.C, 0, 0, 0, g.alpha);
    return launch_cfg<E, T, T, 64, 4, true, false, unsigned short, true, EpilogueParams>(g, 1, g.C, 0, 0, 0, g.alpha);
}

}  // namespace

int gemm_fast_epilogue(const GemmArgs &g, int tile)
{
    if (!g.maps || !g.epilogue || !g.a_kmajor || g.b_kmajor) return CUBE3D_EINVAL;
    if (widens(g)) return CUBE3D_ENOTIMPL;
    if (g.in_dtype == CUBE3D_FP8_E4M3) return tile == 256 ? launch_epilogue<Fp8, 256>(g) : CUBE3D_ENOTIMPL;
    if (g.in_dtype != CUBE3D_BF16) return CUBE3D_ENOTIMPL;
    if (tile == 256) return launch_epilogue<Bf16, 256>(g);
    return tile == 128 ? launch_epilogue<Bf16, 128>(g) : CUBE3D_ENOTIMPL;
}

}  // namespace cube3d
