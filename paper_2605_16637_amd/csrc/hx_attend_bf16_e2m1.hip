// Attention's kernels: queries of bf16, a cache of 4 bits.
#include "hx_attend.hpp"

HX_ATTEND_TYPES(bf16_e2m1, __bf16, 4)
