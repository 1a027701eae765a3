// Sum of weights of every tile (256 scores), best score and sum of every group (16 tiles) of long rows: the one pass over the scores that
// kge_top_scores and kge_sample_scores make where nothing is cut, and the first one where something is.
//
// Weights are relative to the best score of the four tiles that a wave has at a time, so that waves work for themselves: no score has to be known
// before the others are read.  Every workgroup goes through a range of groups and has the next one's scores on their way while it works on one's: reads and
// arithmetic take about the same time: 20 M fp32 scores with best and lowest alone 16 us (5 TB/s, the rate of a large copy), 40 M bf16 scores with the
// tiles' best 15 us (5.3 TB/s).
#include "k_rows.h"

namespace {

template <int DT, int MODE>
__global__ __launch_bounds__(256) void k_tiles(TileArgs a) {
    constexpr bool SUMS = MODE == TILES_SUMS || MODE == TILES_BEST_SUMS, EACH = MODE == TILES_BEST || MODE == TILES_BEST_SUMS;
    __shared__ float bests[2][GROUP_TILES], worsts[2][4], tops[2][4];
    __shared__ double sums[2][GROUP_TILES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t blocks = a.in.rows * a.groups, start = (int64_t)flat_block() * a.per, end = min(start + a.per, blocks);
    if (start >= blocks) return;
    int64_t row = start / a.groups, group = start - row * a.groups;
    const Scale scale(a.inv_t);
    const auto* scores = static_cast<const typename Score<DT>::type*>(a.in.p);
    Quad<DT> x[4];
    auto load = [&](int64_t r, int64_t g) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i].load(scores + r * a.in.ld, g * GROUP + (wave * 4 + i) * 256 + lane * 4, a.in.n);
    };
    load(row, group);
    for (int64_t block = start; block < end; ++block) {
        float v[16];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i].values(group * GROUP + (wave * 4 + i) * 256, a.in.n, v + 4 * i);
        const int64_t this_row = row, this_group = group;
        if (++group == a.groups) { group = 0; ++row; }
        if (block + 1 < end) load(row, group);  // the next one's scores arrive while these are worked on
        const int half = (int)(block - start) & 1;
        const int tile = wave * 4 + tile_of_row(lane >> 4);
        if constexpr (EACH) {
            float m[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) m[i] = fmaxf(fmaxf(v[4 * i], v[4 * i + 1]), fmaxf(v[4 * i + 2], v[4 * i + 3]));
            const float most = max_four(m);
            if ((lane & 15) == 15) bests[half][tile] = most;
        }
        if constexpr (MODE != TILES_BEST) {
            const float best = best_of(v);  // of the wave's four tiles
            if constexpr (SUMS) {
                const Weights w(best, scale);
                const double z = sum_of_tiles(v, w, score_below(w.floor));
                if ((lane & 15) == 15) sums[half][tile] = z;
            } else {
                float worst = INFINITY;
#pragma unroll
                for (int q = 0; q < 16; ++q) worst = v[q] > -INFINITY ? fminf(worst, v[q]) : worst;
                worst = -wave_most(-worst);
                if (lane == 0) worsts[half][wave] = worst;
            }
            if (lane == 0) tops[half][wave] = best;
        }
        if (a.clear)
            for (int64_t w = this_group * 256 + threadIdx.x; w < a.clear_words; w += a.groups * 256) a.clear[this_row * a.clear_words + w] = 0;
        __syncthreads();  // (the halves: the next group's values do not wait for this one's to be read)
        if (wave != (int)(block & 3)) continue;
        if (EACH && lane < GROUP_TILES) a.tile_best[block * GROUP_TILES + lane] = bests[half][lane];
        if constexpr (MODE == TILES_BEST) continue;
        const float own = tops[half][(lane & 15) / 4], top = fmaxf(fmaxf(tops[half][0], tops[half][1]), fmaxf(tops[half][2], tops[half][3]));
        if (lane == 0) a.group_best[block] = top;
        if constexpr (SUMS) {
            const Weights w(top, scale);
            const double z = lane < GROUP_TILES ? sums[half][lane] : 0.0;
            if (MODE == TILES_SUMS && lane < GROUP_TILES) {
                a.tile_best[block * GROUP_TILES + lane] = own;
                a.tile_sum[block * GROUP_TILES + lane] = z;
            }
            const double all = wave_sum64(own > -INFINITY ? z * w.of(own) : 0.0);
            if (lane == 0) a.group_sum[block] = all;
        } else {
            if (lane == 0) a.group_worst[block] = fminf(fminf(worsts[half][0], worsts[half][1]), fminf(worsts[half][2], worsts[half][3]));
        }
    }
}

template <int DT> void launch(const TileArgs& a, int mode, hipStream_t st) {
    const dim3 grid = flat_grid(pieces(a.in.rows * a.groups, a.per));
    if (mode == TILES_SUMS) k_tiles<DT, TILES_SUMS><<<grid, 256, 0, st>>>(a);
    else if (mode == TILES_RANGE) k_tiles<DT, TILES_RANGE><<<grid, 256, 0, st>>>(a);
    else if (mode == TILES_BEST) k_tiles<DT, TILES_BEST><<<grid, 256, 0, st>>>(a);
    else k_tiles<DT, TILES_BEST_SUMS><<<grid, 256, 0, st>>>(a);
}

}  // namespace

void kge_launch_tiles(TileArgs a, TileMode mode, hipStream_t st) {
    a.per = groups_per_workgroup(a.in.rows * a.groups);
    if (a.in.dtype == KGE_F32) launch<KGE_F32>(a, mode, st);
    else if (a.in.dtype == KGE_BF16) launch<KGE_BF16>(a, mode, st);
    else launch<KGE_F16>(a, mode, st);
}
