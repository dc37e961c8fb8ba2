// The ring kernel's grouped forms for INT8 operands.
#include "gemm_ring.h"

namespace hero_gemm {
HERO_GROUPED_RING_8BIT(HERO_I8, HERO_I8)
}  // namespace hero_gemm
