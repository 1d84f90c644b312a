// Attention's kernels: queries of bf16, a cache of the same.
#include "hx_attend.hpp"

HX_ATTEND_TYPES(bf16, __bf16, false)
