// Attention's kernels: queries of fp16, a cache of 4 bits.
#include "hx_attend.hpp"

HX_ATTEND_TYPES(f16_e2m1, _Float16, 4)
