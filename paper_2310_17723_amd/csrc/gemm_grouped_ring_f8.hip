// The ring kernel's grouped forms for E4M3 operands.
#include "gemm_ring.h"

namespace hero_gemm {
HERO_GROUPED_RING_8BIT(HERO_F8E4M3, HERO_F8E4M3)
}  // namespace hero_gemm
