// The ring kernel's grouped forms for 16-bit operands.
#include "gemm_ring.h"

namespace hero_gemm {
HERO_GROUPED_RING_16BIT(HERO_BF16)
HERO_GROUPED_RING_16BIT(HERO_F16)
}  // namespace hero_gemm
