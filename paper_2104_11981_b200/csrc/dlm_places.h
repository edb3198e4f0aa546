// Places of long texts, up to 2^31 - 1 of them (not installed): searches and strides whose sums stay in range.  Host code may use
// them, too.
#pragma once
#include <cstdint>

#ifdef __CUDACC__
#define DLM_BOTH __host__ __device__ __forceinline__
#else
#define DLM_BOTH inline
#endif

namespace dlm {

// How many of the ascending keys[0 .. count) are below v.  Unsigned, since the sum of both ends passes 2^31 - 1 above 2^30 keys.
template <typename Keys>
DLM_BOTH int lower_bound(const Keys& keys, int count, uint32_t v) {
    uint32_t lo = 0, hi = (uint32_t)count;
    while (lo < hi) {
        const uint32_t mid = (lo + hi) >> 1;
        if (keys[mid] < v)
            lo = mid + 1;
        else
            hi = mid;
    }
    return (int)lo;
}

// f(k) for every STEP-th place from `first` until `end`.  Unsigned, since the last step may pass 2^31 - 1.
template <uint32_t STEP, int UNROLL, typename F>
DLM_BOTH void each_place(uint32_t first, uint32_t end, const F& f) {
#pragma unroll UNROLL
    for (uint32_t k = first; k < end; k += STEP) f(k);
}

}  // namespace dlm

#undef DLM_BOTH
