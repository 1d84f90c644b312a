// Which entries of a table's row a call gives back: whole numbers alone, the same on the host.
#pragma once

#include <cstdint>

#ifdef __HIPCC__
#define HX_HOST_DEVICE __host__ __device__
#else
#define HX_HOST_DEVICE
#endif

HX_HOST_DEVICE inline int hx_pages_of(int tokens, int shift) { return (int)(((int64_t)tokens + (1 << shift) - 1) >> shift); }

// Entries lo .. hi-1.  Unsigned, as a loop over them counts on past hi by a workgroup's threads, and hi may be INT32_MAX.
struct HxSpan {
    uint32_t lo, hi;
};

// The entries of a row of `len` tokens whose positions all lie in first .. last-1 and are filled.
HX_HOST_DEVICE inline HxSpan hx_filled_within(int first, int last, int len, int shift)
{
    const int lo = first < 0 ? 0 : first < len ? first : len, hi = last < 0 ? 0 : last < len ? last : len;
    return HxSpan{(uint32_t)hx_pages_of(lo, shift), (uint32_t)hi >> shift};
}
