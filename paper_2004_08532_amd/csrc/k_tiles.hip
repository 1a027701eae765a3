// Best score and sum of weights of every tile (256 scores) and group (16 tiles) of long rows: the one pass over the scores that
// kge_top_scores and kge_sample_scores make where nothing is cut, and the first one where something is.
//
// Weights are relative to the best score of their own tile, so that waves work for themselves: no score has to be known before the
// others are read.  A wave has four tiles of loads in flight; bound by the reads, and with sums by the weights' arithmetic as much.
#include "k_rows.h"

namespace {

template <int DT, bool SUMS>
__global__ __launch_bounds__(256) void k_tiles(TileArgs a) {
    __shared__ float bests[GROUP_TILES], worsts[4];
    __shared__ double sums[GROUP_TILES];
    const int64_t block = flat_block();
    if (block >= a.in.rows * a.groups) return;
    const int64_t row = block / a.groups, group = block - row * a.groups;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const auto* s = static_cast<const typename Score<DT>::type*>(a.in.p) + row * a.in.ld;
    float v[16];
    load_tiles<DT, 4, 4>(s, group * GROUP, a.in.n, v);
    if (a.clear) {
        for (int64_t x = group * 256 + threadIdx.x; x < a.clear_words; x += (int64_t)a.groups * 256) a.clear[row * a.clear_words + x] = 0;
    }
    float worst = INFINITY;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float best = wave_most(fmaxf(fmaxf(v[4 * i], v[4 * i + 1]), fmaxf(v[4 * i + 2], v[4 * i + 3])));
        if constexpr (SUMS) {
            const Weights w(best, a.inv_t);
            const double z = wave_sum64((w.of(v[4 * i]) + w.of(v[4 * i + 1])) + (w.of(v[4 * i + 2]) + w.of(v[4 * i + 3])));
            if (lane == 0) sums[i * 4 + wave] = z;
        } else {
#pragma unroll
            for (int q = 4 * i; q < 4 * i + 4; ++q) worst = v[q] > -INFINITY ? fminf(worst, v[q]) : worst;
        }
        if (lane == 0) bests[i * 4 + wave] = best;
    }
    if constexpr (!SUMS) {
        worst = -wave_most(-worst);
        if (lane == 0) worsts[wave] = worst;
    }
    __syncthreads();
    if (threadIdx.x >= 64) return;
    const float best = lane < GROUP_TILES ? bests[lane] : -INFINITY, top = wave_most(best);
    if (lane < GROUP_TILES && a.tile_best) a.tile_best[block * GROUP_TILES + lane] = best;
    if (lane == 0) a.group_best[block] = top;
    if constexpr (SUMS) {
        const Weights w(top, a.inv_t);
        const double z = lane < GROUP_TILES ? sums[lane] : 0.0;
        if (lane < GROUP_TILES && a.tile_sum) a.tile_sum[block * GROUP_TILES + lane] = z;
        const double all = wave_sum64(best > -INFINITY ? z * w.of(best) : 0.0);
        if (lane == 0) a.group_sum[block] = all;
    } else if (a.group_worst) {
        if (lane == 0) a.group_worst[block] = fminf(fminf(worsts[0], worsts[1]), fminf(worsts[2], worsts[3]));
    }
}

template <int DT> void launch(const TileArgs& a, bool sums, hipStream_t st) {
    const dim3 grid = flat_grid(a.in.rows * a.groups);
    if (sums) k_tiles<DT, true><<<grid, 256, 0, st>>>(a);
    else k_tiles<DT, false><<<grid, 256, 0, st>>>(a);
}

}  // namespace

void kge_launch_tiles(const TileArgs& a, bool sums, hipStream_t st) {
    if (a.in.dtype == KGE_F32) launch<KGE_F32>(a, sums, st);
    else if (a.in.dtype == KGE_BF16) launch<KGE_BF16>(a, sums, st);
    else launch<KGE_F16>(a, sums, st);
}
