// Which entries of a table's row a call gives back, and which a query sees in any case: whole numbers alone, the same on the host.
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

// Of a row's entries 0 .. own those that a query sees in any case, the first n_first and the last n_last, where it sees n_pages of them and they are more.
// Where they are not, `all` are seen, and fewer may be there than the first and the last ones would be.
struct HxSeen {
    bool all;
    int from, to;            // it chooses among from .. to-1; n_first + n_last <= n_pages <= own, so they and what lies around them are in the row
    int fixed;               // how many it sees in any case, 0 where all are seen

    HX_HOST_DEVICE int entry(int i) const { return i < from ? i : to + (i - from); }          // the i-th of them
};

HX_HOST_DEVICE inline HxSeen hx_seen_in_any_case(int own, int n_pages, int n_first, int n_last)
{
    const bool all = own < n_pages;
    return HxSeen{all, all ? 0 : n_first, all ? 0 : own - (n_last - 1), all ? 0 : n_first + n_last};
}
