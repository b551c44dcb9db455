// Instantiations of the ring kernel (gemm_ring.h): fp8 operands widened to bf16, with what follows the product.
#include "gemm_ring.h"

namespace cube3d {

int gemm_ring_fp8_wide(const GemmArgs &g, const edge::Params &p, const edge::RingPlan &r)
{
    return edge::ring_any<edge::Fp8Wide>(g, p, r);
}

}  // namespace cube3d
