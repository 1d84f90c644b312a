// Attention's kernels: queries of f16, a cache of the same.
#include "hx_attend.hpp"

HX_ATTEND_TYPES(f16, _Float16, 16)
