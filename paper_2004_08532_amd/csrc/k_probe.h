// The first place among lo .. hi for which something holds that holds for every later one too, asked by the 64 lanes of a wave at once.
#pragma once
#include <stdint.h>

#ifdef __HIPCC__
#define KGE_PROBE __host__ __device__ __forceinline__
#else
#define KGE_PROBE inline
#endif

struct Probes {
    int64_t lo, hi;  // the place is there, or nowhere: then the search ends at hi
    KGE_PROBE bool open() const { return lo < hi; }
    // (one more than a 64th: the last lane's place is hi or would be behind it, so that hi is asked for in every round)
    KGE_PROBE int64_t step() const { return (hi - lo) / 64 + 1; }
    KGE_PROBE int64_t at(int lane) const {
        const int64_t x = lo + (lane + 1) * step() - 1;
        return x < hi ? x : hi;
    }
    KGE_PROBE void narrow(int first) {  // the first lane for whose place it holds, 63 without any
        const int64_t s = step(), top = lo + (first + 1) * s - 1, bottom = lo + first * s;
        lo = bottom < hi ? bottom : hi;
        hi = top < hi ? top : hi;
    }
};
