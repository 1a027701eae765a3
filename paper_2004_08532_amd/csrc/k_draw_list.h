// Draws from a list of a row's best candidates, shared by the kernels that end with one (k_draw.hip, k_top.hip).
#pragma once
#include "k_rows.h"

struct DrawArgs {
    RowScores in;
    const double* u;  // [rows][draws]
    int draws, top_k;
    double inv_t, top_p, min_p;
    int64_t* ids;
    float* logp;
};

#ifdef __HIPCC__
namespace {

__device__ __forceinline__ double unit_number(double u) { return u > 0.0 ? fmin(u, 1.0 - 0x1p-53) : 0.0; }  // (NaN: 0)

template <int THREADS> __device__ __forceinline__ void write_empty(const DrawArgs& a, int64_t row) {
    for (int d = threadIdx.x; d < a.draws; d += THREADS) {
        a.ids[row * a.draws + d] = -1;
        if (a.logp) a.logp[row * a.draws + d] = -INFINITY;
    }
}

// The draws from a sorted list of the row's best candidates.  list: LDS, the first `count` entries; sums: as many; spare and rank: 256 of each, not the list's.
template <int THREADS>
__device__ __forceinline__ void draw_from_list(const DrawArgs& a, int64_t row, uint64_t* list, uint64_t* spare, uint32_t* rank, int count, double* sums, int* kept) {
    if (count == 0) { write_empty<THREADS>(a, row); return; }
    const int lane = threadIdx.x & 63;
    const Scale scale(a.inv_t);
    const Weights weights(key_score((uint32_t)(list[0] >> 32)), scale);
    auto scan = [&](int n) {  // sums of weights -> running sums, by the first wave
        __syncthreads();
        if (threadIdx.x < 64) {
            double carry = 0.0;
            for (int e0 = 0; e0 < n; e0 += 64) {
                const double v = carry + wave_scan64(e0 + lane < n ? sums[e0 + lane] : 0.0, lane);
                if (e0 + lane < n) sums[e0 + lane] = v;
                carry = __shfl(v, 63, 64);
            }
        }
        __syncthreads();
    };
    for (int e = threadIdx.x; e < count; e += THREADS) sums[e] = weights.of(key_score((uint32_t)(list[e] >> 32)));
    if (threadIdx.x == 0) *kept = 0;
    scan(count);
    const double target = a.top_p < 1.0 ? a.top_p * sums[count - 1] : INFINITY;
    for (int e = threadIdx.x; e < count; e += THREADS) {
        const bool in = e == 0 || (sums[e - 1] < target && weights.of(key_score((uint32_t)(list[e] >> 32))) >= a.min_p);
        if (in) atomicMax(kept, e + 1);
    }
    __syncthreads();
    count = *kept;
    // into the order of positions: the key goes below the inverted position
    for (int e = threadIdx.x; e < count; e += THREADS) list[e] = list[e] << 32 | list[e] >> 32;
    __syncthreads();
    list = order_list<THREADS>(list, spare, rank, count);
    for (int e = threadIdx.x; e < count; e += THREADS) sums[e] = weights.of(key_score((uint32_t)list[e]));
    scan(count);
    const double total = sums[count - 1];
    for (int d = threadIdx.x; d < a.draws; d += THREADS) {
        const double want = unit_number(a.u[row * a.draws + d]) * total;
        int lo = 0, hi = count - 1;  // first entry whose running sum exceeds `want`
        while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if (sums[mid] > want) hi = mid; else lo = mid + 1;
        }
        // (An entry without weight is never drawn.  The running sums do not tell: they are added up in another order from lane to lane, so that one can
        // differ from the one before it by a rounding where nothing was added.)
        double w = weights.of(key_score((uint32_t)list[lo]));
        while (lo > 0 && !(w > 0.0)) w = weights.of(key_score((uint32_t)list[--lo]));
        a.ids[row * a.draws + d] = (int64_t)(uint32_t)~(uint32_t)(list[lo] >> 32);
        if (a.logp) a.logp[row * a.draws + d] = (float)log(w / total);
    }
}

}  // namespace
#endif
