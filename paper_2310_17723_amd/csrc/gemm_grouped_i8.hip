// The persistent kernel's grouped forms for INT8 operands.
#include "gemm_persistent.h"

namespace hero_gemm {
HERO_GROUPED_8BIT(HERO_I8, HERO_I8)
}  // namespace hero_gemm
