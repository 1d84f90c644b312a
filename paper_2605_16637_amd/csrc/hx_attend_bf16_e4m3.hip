// Attention's kernels: queries of bf16, a cache of 8 bits.
#include "hx_attend.hpp"

HX_ATTEND_TYPES(bf16_e4m3, __bf16, true)
