// Attention's kernels: queries of f16, a cache of 8 bits.
#include "hx_attend.hpp"

HX_ATTEND_TYPES(f16_e4m3, _Float16, true)
