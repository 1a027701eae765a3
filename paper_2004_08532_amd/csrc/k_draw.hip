// Candidates drawn from rows of scores by given random numbers (kge_sample_scores).
//
// With w_j = exp((s_j - best) / T) the candidates kept are the first K in order of their scores: K the least of top-k, the number that
// top-p takes (the fewest whose w reach top_p times the sum over the first top_k) and the number with w_j >= min_p.  A number u in
// [0, 1) falls on the first position j at which the sum of the kept w up to j exceeds u times the whole sum.
//
// Sums are kept per tile of 256 scores; a draw is a wave that finds its tile among the sums and its position in the tile.  All sums are
// formed in 64 bits, in a fixed order or as whole numbers, so a draw depends on the row and its number alone.
//
// What bounds them (fp32; a large copy takes 12 us for the first and 16 us for the last of these):
//     1024 rows of 14,951, 16 draws, nothing cut   k_draw_whole 30 us: a weight in 64 bits per score, 13 M wave instructions, 26 us of the vector units
//     the same, top-p 0.9, 1 draw                  k_draw_rows 63 us: bins, then weights in 64 bits, 22 M wave instructions, 45 us of the vector units
//     one such row                                 k_draw_rows 22 us: a chain of some twenty steps between barriers, on one CU
//     2 rows of 10 M, top-p 0.95, 64 draws         143 us in 9 launches: best and lowest score 16, bins 43, 29, 13 and 6, the cut 5, sums of what is
//                                                  kept 26, running sums 8, draws 6; the first bins and the sums are bound by their weights
#include "k_draw_list.h"
#include "k_probe.h"

namespace {

// What is kept: the scores above `over`, and of those equal to t the ones whose inverted position is at least `least` (in rows held by a
// workgroup) or the first `ties` of the row (in long ones).  t is not above `over`; NaN: none of them.
struct Kept {
    float over, t;
    uint32_t least, ties;
};
// The weights of what is kept are at least min_p and not 0.  (Asked by a whole wave.)
__device__ __forceinline__ void keep_from_min_p(Kept& k, const Weights& w, float best, double min_p) {
    float least = w.floor;
    if (min_p > 0.0) {
        least = key_score(lowest_key(order_key(least), order_key(best), [&](uint32_t key) { return w.of(key_score(key)) >= min_p; }));
    }
    if (!(k.t >= least)) k.t = __uint_as_float(0x7FC00000u);
    k.over = fmaxf(k.over, score_below(least));
}

// Position in a tile (256 scores from `first` on, read by the caller) at which the sum passes `target`, `base` of it in front of the tile; the tile's
// last kept position where rounding leaves none.  COUNTED: equal scores are kept by `ties`, `ties_before` of them lie in front of the tile.
template <int DT, bool COUNTED>
__device__ __forceinline__ void draw_in_tile(const Quad<DT>& x, int64_t first, int64_t n, const Kept& k, const Weights& weights, uint32_t ties_before,
                                             double base, double target, int lane, int64_t& id, double& weight) {
    float v[4];
    x.values(first, n, v);
    double w[4], sum = 0.0;
    uint32_t rank = ties_before;
    if constexpr (COUNTED) {
        const uint64_t below = ((uint64_t)1 << lane) - 1;
#pragma unroll
        for (int q = 0; q < 4; ++q) rank += __popcll(__ballot(v[q] == k.t) & below);
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const bool equal = v[q] == k.t;
        w[q] = weights.of(v[q], v[q] > k.over || (equal && (COUNTED ? rank < k.ties : ~(uint32_t)(first + lane * 4 + q) >= k.least)));
        rank += equal;
        sum += w[q];
    }
    const double incl = base + wave_scan64(sum, lane);
    const uint64_t past = __ballot(incl > target && sum > 0.0), any = __ballot(sum > 0.0);
    const int who = past ? __ffsll((unsigned long long)past) - 1 : any ? 63 - __clzll(any) : 0;
    if (lane == who) {
        double run = incl - sum;
        int at = -1;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (w[q] > 0.0) {
                const bool before = at < 0 || !(run > target);
                run += w[q];
                if (before) { at = q; weight = w[q]; }
            }
        }
        id = at < 0 ? -1 : first + lane * 4 + at;
    }
    id = __shfl((long long)id, who, 64);
    weight = __shfl(weight, who, 64);
}

// Tiles of rows of which nothing is left out have sums relative to the best of the four tiles that a wave had at a time, and what counts beside that can
// be too little beside the row's best: a tile with a sum whose scores are all below the row's floor.  Then one of the other three, whose best is not
// below it, is where the number falls: the tiles behind it, j = 1, 2, ..., and where those end the ones in front of it.
__device__ __forceinline__ int other_of_four(int tile, int j) {
    const int r = tile & 3;
    return r + j < 4 ? tile + j : tile - (r + j - 3);
}

// The draws of a row whose tile sums a workgroup has in LDS.  sums[t]: of tile t, relative to tile_best[t] (the row's best where that is null).
template <int DT, int WAVES, int TILES>
__device__ __forceinline__ void draw_from_tiles(const DrawArgs& a, int64_t row, const typename Score<DT>::type* s, int tiles, double* sums,
                                                const float* tile_best, const Kept& kept, const Weights& weights) {
    constexpr int WORDS = (TILES + 63) / 64;
    __shared__ uint64_t weighted[WORDS];  // tiles with a weight (the running sums differ by roundings also where nothing was added)
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    __syncthreads();
    if (wave == 0) {  // running sums
        double carry = 0.0;
#pragma unroll
        for (int t0 = 0; t0 < TILES; t0 += 64) {
            const int t = t0 + lane;
            double x = t < tiles ? sums[t] : 0.0;
            if (tile_best && t < tiles) x = tile_best[t] > -INFINITY ? x * weights.of(tile_best[t]) : 0.0;
            const uint64_t some = __ballot(x > 0.0);
            if (lane == 0) weighted[t0 / 64] = some;
            x = carry + wave_scan64(x, lane);
            if (t < tiles) sums[t] = x;
            carry = lane64(x, 63);
        }
    }
    __syncthreads();
    const double total = sums[tiles - 1];
    double x[WORDS];
    int last = 0;  // tile with a weight
#pragma unroll
    for (int k = 0; k < WORDS; ++k) {
        const uint64_t word = weighted[k];  // (the same for the wave: in scalar registers, and with it the tiles' numbers)
        const uint64_t some = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(word >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)word);
        x[k] = some >> lane & 1 ? sums[k * 64 + lane] : -INFINITY;
        if (some) last = k * 64 + 63 - __clzll(some);
    }
    constexpr int AT_ONCE = 4;  // draws of a wave whose tiles are read together
    for (int d0 = wave * AT_ONCE; d0 < a.draws; d0 += WAVES * AT_ONCE) {
        const int n = min(AT_ONCE, a.draws - d0);
        const double own = lane < n ? unit_number(a.u[row * a.draws + d0 + lane]) * total : 0.0;
        Quad<DT> quad[AT_ONCE];
        int tile[AT_ONCE];
#pragma unroll
        for (int d = 0; d < AT_ONCE; ++d) {
            const double want = lane64(own, d);
            int at = 0;  // the first tile with a weight whose running sum exceeds `want`, the last one with a weight where none does
#pragma unroll
            for (int k = WORDS - 1; k >= 0; --k) {
                const uint64_t past = __ballot(x[k] > want) | (last / 64 == k ? (uint64_t)1 << (last & 63) : 0);
                at = past ? k * 64 + __builtin_ctzll(past) : at;
            }
            tile[d] = at;
            quad[d].load(s, (int64_t)tile[d] * 256 + lane * 4, a.in.n);
        }
        uint32_t missed = 0;  // a bit per draw
#pragma unroll
        for (int d = 0; d < AT_ONCE; ++d) {
            if (d >= n) break;
            int64_t id = -1;
            double weight = 0.0;
            draw_in_tile<DT, false>(quad[d], (int64_t)tile[d] * 256, a.in.n, kept, weights, 0u, tile[d] > 0 ? sums[tile[d] - 1] : 0.0, lane64(own, d), lane, id, weight);
            if (tile_best && id < 0) missed |= 1u << d;
            if (lane == 0) {
                a.ids[row * a.draws + d0 + d] = id;
                if (a.logp) a.logp[row * a.draws + d0 + d] = (float)log(weight / total);
            }
        }
        if (!tile_best) continue;
        for (; missed; missed &= missed - 1) {
            const int d = __ffs((int)missed) - 1;
            int from = tile[0];
#pragma unroll
            for (int k = 1; k < AT_ONCE; ++k) from = d == k ? tile[k] : from;
            int64_t id = -1;
            double weight = 0.0;
#pragma unroll 1
            for (int j = 1; j < 4 && id < 0; ++j) {
                const int t = other_of_four(from, j);
                if (t >= tiles) continue;
                quad[0].load(s, (int64_t)t * 256 + lane * 4, a.in.n);
                draw_in_tile<DT, false>(quad[0], (int64_t)t * 256, a.in.n, kept, weights, 0u, t > 0 ? sums[t - 1] : 0.0, lane64(own, d), lane, id, weight);
            }
            if (lane == 0) {
                a.ids[row * a.draws + d0 + d] = id;
                if (a.logp) a.logp[row * a.draws + d0 + d] = (float)log(weight / total);
            }
        }
    }
}

// Rows of which nothing is left out: a wave works through its tiles, each relative to its own best score.
template <int DT, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void k_draw_whole(DrawArgs a) {
    constexpr int TILES = KGE_ROW_RESIDENT / 256;
    __shared__ double sums[TILES];
    __shared__ float bests[TILES], maxima[WAVES];
    const int64_t row = flat_block();
    if (row >= a.in.rows) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), tiles = (int)((a.in.n + 255) / 256);
    const auto* s = static_cast<const typename Score<DT>::type*>(a.in.p) + row * a.in.ld;
    const Scale scale(a.inv_t);
    float most = -INFINITY;
    Quad<DT> x[4];
    auto load = [&](int t0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i].load(s, (int64_t)(t0 + i) * 256 + lane * 4, a.in.n);
    };
    load(wave * 4);
    for (int t0 = wave * 4; t0 < tiles; t0 += 4 * WAVES) {
        float v[16];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i].values((int64_t)(t0 + i) * 256, a.in.n, v + 4 * i);
        if (t0 + 4 * WAVES < tiles) load(t0 + 4 * WAVES);  // (arrives while these are worked on)
        const float best = best_of(v);
        const Weights w(best, scale);
        const double z = sum_of_tiles(v, w, score_below(w.floor));
        const int tile = t0 + tile_of_row(lane >> 4);
        if ((lane & 15) == 15 && tile < tiles) { sums[tile] = z; bests[tile] = best; most = fmaxf(most, best); }
    }
    most = block_max<WAVES>(most, maxima);
    if (!(most > -INFINITY)) { write_empty<WAVES * 64>(a, row); return; }
    const Weights weights(most, scale);
    const Kept kept = {score_below(weights.floor), __uint_as_float(0x7FC00000u), 0u, 0u};
    draw_from_tiles<DT, WAVES, TILES>(a, row, s, tiles, sums, bests, kept, weights);
}

// ---------------------------------------------------------------------------------------------------------
// Where the weights of a row reach top-p.  The scores are counted into bins by what their weights sum to; the bin in which the running
// sum, from the best score down, reaches the target becomes the interval for the next round, until its scores are few enough
// to be put in order one by one or are all equal.  First round: bins of equal width between the best score and the lowest that matters
// (40 T below it, or the lowest there is); then of equal numbers of keys.
// Sums in bins are whole numbers (any order of the additions gives the same): p * 2^(n + bits - e) of a weight p * 2^n, with e the exponent at the
// bin's (in later rounds: the interval's) upper end, so that a sum is as exact in the far bins as in the first.
// ---------------------------------------------------------------------------------------------------------
template <int LOG_BINS> struct BinRule {
    static constexpr int BINS = 1 << LOG_BINS;
    uint32_t lo, hi;   // interval of keys
    int shift;         // keys per bin: 2^shift; negative: bins of equal width
    float unit, best;  // scores are taken times this power of two, the best one already is
    float per;         // bins per one of these
    float drop;        // exponents per bin
    int top;           // exponent at the interval's upper end
    __device__ __forceinline__ float place(float s) const { return fmaf(s, -unit, best) * per; }  // (the sum is exact but for its last bit)
    __device__ __forceinline__ int bin(float s) const {
        if (shift < 0) {
            const float x = place(s);  // (NaN: both are +inf)
            return x < (float)(BINS - 1) ? (int)x : x >= 0.f ? BINS - 1 : 0;
        }
        return (int)((hi - order_key(s)) >> shift);
    }
    __device__ __forceinline__ bool in(float s) const { return s >= key_score(lo) && s <= key_score(hi); }
    __device__ __forceinline__ int exponent(int b) const { return shift < 0 ? (int)floorf(-(float)b * drop) : top; }
};

// Rule of the first round.
template <int LOG_BINS> __device__ __forceinline__ BinRule<LOG_BINS> first_bins(float best, float worst, double inv_t) {
    constexpr int BINS = 1 << LOG_BINS;
    BinRule<LOG_BINS> r;
    r.lo = LOWEST_KEY; r.hi = order_key(best);
    r.shift = -1;
    // The unit keeps differences finite and the bins per unit a normal number: 1 unless scores are further apart than the type's largest value, or
    // those that matter are closer than 2^-60.  (Then either the best is below 2^-20, or all others are too far from it to matter.)
    float range = fminf(best - worst, (float)fmin(40.0 / inv_t, 3.4e38));
    r.unit = best - worst == INFINITY ? 0.5f : range < 0x1p-60f && fabsf(best) < 0x1p-20f ? 0x1p60f : 1.f;
    r.best = best * r.unit;
    range = fminf(fmaf(worst, -r.unit, r.best), (float)fmin(40.0 / inv_t * (double)r.unit, 3.4e38));
    r.per = range > 0.f ? fminf((float)BINS * (1.f - 0x1p-12f) / range, 1e38f) : 0.f;  // (the lowest score is inside the last bin)
    r.drop = r.per > 0.f ? (float)(inv_t * 1.4426950408889634 / ((double)r.per * (double)r.unit)) : 0.f;
    r.top = 0;
    return r;
}
// Rule of the round that follows, for bin b.
template <int LOG_BINS> __device__ __forceinline__ BinRule<LOG_BINS> next_bins(const BinRule<LOG_BINS>& r, int b, const Weights& w) {
    BinRule<LOG_BINS> x = r;
    if (r.shift < 0) {  // the keys whose bin is b: a larger key never has a larger bin
        x.lo = lowest_key(r.lo, r.hi, [&](uint32_t key) { return r.bin(key_score(key)) <= b; });
        x.hi = b > 0 ? lowest_key(r.lo, r.hi, [&](uint32_t key) { return r.bin(key_score(key)) < b; }) - 1 : r.hi;
    } else {
        x.hi = r.hi - ((uint32_t)b << r.shift);
        const uint32_t last = ((uint32_t)1 << r.shift) - 1;
        x.lo = x.hi >= last && x.hi - last > r.lo ? x.hi - last : r.lo;
        // (no score has the key of -0, but an interval that ends with it would hold +0, which the bin in front has counted)
        if (x.hi == NEGATIVE_ZERO_KEY && x.hi > x.lo) --x.hi;
    }
    x.shift = x.hi > x.lo ? max(0, 32 - __clz(x.hi - x.lo) - LOG_BINS) : 0;
    double p;
    w.split(key_score(x.hi), p, x.top);
    return x;
}

__device__ __forceinline__ uint64_t whole_weight(const Weights& w, float s, int exponent, int bits) {
    double p;
    int n;
    w.split(s, p, n);
    const int up = n - exponent + bits;
    if (!(s >= w.floor) || up < -2) return 0;
    return (uint64_t)__double_as_longlong(Weights::scaled(p, up) + 0x1p52) & (((uint64_t)1 << 52) - 1);
}

// Running sums of the bins' weights, from the best down, by THREADS threads of BINS / THREADS neighbours each: the first bin at which `above` plus
// the sum reaches the target (first: target = top_p times the whole sum, which is returned in it).  The last bin with
// anything in it where rounding leaves none.  `above` becomes the sum in front of the bin.
template <int THREADS, int LOG_BINS>
__device__ __forceinline__ int find_bin(const uint64_t* bins, const BinRule<LOG_BINS>& r, int bits, bool first, double top_p, double& target, double& above,
                                        double* part /* [THREADS / 64 + 1] */, uint32_t* found /* [2] */) {
    constexpr int BINS = 1 << LOG_BINS, PER = BINS / THREADS, WAVES = THREADS / 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (threadIdx.x < 2) found[threadIdx.x] = threadIdx.x ? 0 : BINS;
    double x[PER], sum = 0.0;
#pragma unroll
    for (int q = 0; q < PER; ++q) {
        const int b = threadIdx.x * PER + q;
        x[q] = ldexp((double)bins[b], r.exponent(b) - bits);
        sum += x[q];
    }
    const double incl = wave_scan64(sum, lane);
    if (lane == 63) part[wave] = incl;
    __syncthreads();
    double before = 0.0, all = 0.0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        if (w < wave) before += part[w];
        all += part[w];
    }
    if (first) target = top_p * all;
    double run = above + (before + (incl - sum)), front[PER];
    int mine = BINS, last = -1;
#pragma unroll
    for (int q = 0; q < PER; ++q) {
        front[q] = run;
        run += x[q];
        if (x[q] > 0.0) {
            last = threadIdx.x * PER + q;
            if (mine == BINS && run >= target) mine = last;
        }
    }
    if (mine < BINS) atomicMin(&found[0], (uint32_t)mine);
    if (last >= 0) atomicMax(&found[1], (uint32_t)last);
    __syncthreads();
    const int b = found[0] < BINS ? (int)found[0] : (int)found[1];
    if (b / PER == (int)threadIdx.x) {
#pragma unroll
        for (int q = 0; q < PER; ++q) if (q == b % PER) part[WAVES] = front[q];
    }
    __syncthreads();
    above = part[WAVES];
    return b;
}

template <int WAVES, int TPW> struct CutScratch {
    static constexpr int ROOM = WAVES * TPW * 256 < 1024 ? WAVES * TPW * 256 : 1024, LOG_BINS = WAVES * TPW <= 4 ? 8 : 10, BINS = 1 << LOG_BINS;
    uint64_t bins[BINS > ROOM ? BINS : ROOM];  // then the list
    uint64_t sorted[256];
    double sums[ROOM], part[WAVES + 1];
    uint32_t slots[2 * WAVES], rank[256], found[2], count;
    uint64_t more[WAVES * TPW];
};

// The bins in which the weights of a row reach top-p, as an interval of keys, from weights in 32 bits: a score's is that at its bin's upper end
// times a whole number of 32768ths, by two terms of the exponential (a bin has at most 0.04 T).  Sums of these are off by less than a
// 16,000th: 2^-16 from rounding, 1e-5 from the third term, 5e-6 from a score's place, 5e-6 from the bins' exponents; and 2^15 scores
// 40 T below the best, which are left out, have 2e-13.  A sum reaches top_p of the whole where what is behind it is at most the rest of 1: the closer
// of the two bounds is taken.
constexpr double ENCLOSE = 1.0 / 16000.0, LEFT_OUT = 2e-13;
template <int WAVES, int TPW>
__device__ __forceinline__ void enclose(const float v[TPW * 4], int64_t n, float best, float worst, double inv_t, double top_p, CutScratch<WAVES, TPW>& s, uint32_t& lo, uint32_t& hi) {
    constexpr int THREADS = WAVES * 64, LOG_BINS = CutScratch<WAVES, TPW>::LOG_BINS, BINS = 1 << LOG_BINS, PER = BINS / THREADS;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const BinRule<LOG_BINS> r = first_bins<LOG_BINS>(best, worst, inv_t);
    uint32_t* bins = reinterpret_cast<uint32_t*>(s.bins);
    for (int b = threadIdx.x; b < BINS; b += THREADS) bins[b] = 0;
    if (threadIdx.x < 2) s.found[threadIdx.x] = BINS;
    __syncthreads();
    const bool infinite = best == INFINITY;
    const float top = infinite ? 0.f : r.best, y = r.drop * 0.69314718f, c1 = -y * 32768.f, c2 = 0.5f * y * y * 32768.f;
#pragma unroll
    for (int q = 0; q < TPW * 4; ++q) {
        if (q % 16 == 0 && q > 0 && q * WAVES * 64 >= n) break;
        const float x = infinite ? (v[q] == INFINITY ? 0.f : -INFINITY) : v[q], at = fmaf(x, -r.unit, top) * r.per, part = __builtin_amdgcn_fractf(at);
        const uint32_t number = (uint32_t)fmaf(part, fmaf(part, c2, c1), 32768.5f);
        const bool counts = at < (float)BINS;  // neither masked nor too far; the others add 0, at places that do not collide
        atomicAdd(&bins[counts ? (int)at : lane], counts ? number : 0u);
        if (q % 4 == 3) __builtin_amdgcn_sched_barrier(0);
    }
    __syncthreads();
    double x[PER], sum = 0.0;
#pragma unroll
    for (int q = 0; q < PER; ++q) {
        const float e = (float)(threadIdx.x * PER + q) * r.drop, whole = floorf(e);
        x[q] = ldexp((double)bins[threadIdx.x * PER + q] * (double)__builtin_amdgcn_exp2f(whole - e), -(int)whole);
        sum += x[q];
    }
    const double incl = wave_scan64(sum, lane);
    if (lane == 63) s.part[wave] = incl;
    __syncthreads();
    double run = incl - sum, all = 0.0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        if (w < wave) run += s.part[w];
        all += s.part[w];
    }
    const double reach = top_p * all, behind = (1.0 - top_p) * all, off = 2.0 * ENCLOSE, left = LEFT_OUT * all;
    int first = BINS, last = BINS;
#pragma unroll
    for (int q = 0; q < PER; ++q) {
        run += x[q];
        if (!(x[q] > 0.0)) continue;
        const double rest = all - run;
        const int b = threadIdx.x * PER + q;
        if (first == BINS && run >= reach * (1.0 - off) && rest <= behind * (1.0 + off) + left) first = b;
        if (last == BINS && (run >= reach * (1.0 + off) || rest <= behind * (1.0 - off) - left)) last = b;
    }
    if (first < BINS) atomicMin(&s.found[0], (uint32_t)first);
    if (last < BINS) atomicMin(&s.found[1], (uint32_t)last);
    __syncthreads();
    if (wave == 0) {  // (one wave for all; a larger key never has a larger bin; no bin: all that is left)
        const int from = min((int)s.found[0], BINS - 1), to = min((int)s.found[1], BINS - 1);
        const uint32_t low = order_key(worst), high = order_key(best);
        lo = lowest_key(low, high, [&](uint32_t key) { return r.bin(key_score(key)) <= to; });
        hi = from > 0 ? lowest_key(low, high, [&](uint32_t key) { return r.bin(key_score(key)) < from; }) - 1 : high;
        if (lane == 0) { s.slots[0] = lo; s.slots[1] = hi; s.count = 0; }
    }
    for (int t = threadIdx.x; t < WAVES * TPW; t += THREADS) s.more[t] = 0;
    __syncthreads();
    lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)s.slots[0]);
    hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)s.slots[1]);
}

// The first entry of a list in LDS at which `above` and the sum of the weights reach the target, and what that keeps.
template <int WAVES, int TPW>
__device__ __forceinline__ Kept cut_list(int count, double target, double above, const Weights& w, CutScratch<WAVES, TPW>& s) {
    constexpr int THREADS = WAVES * 64;
    const int lane = threadIdx.x & 63;
    const uint64_t* list = order_list<THREADS>(s.bins, s.sorted, s.rank, count);
    for (int e = threadIdx.x; e < count; e += THREADS) s.sums[e] = w.of(key_score((uint32_t)(list[e] >> 32)));
    __syncthreads();
    if (threadIdx.x < 64) {
        double carry = above;
        int cut = count - 1;
        for (int e0 = 0; e0 < count; e0 += 64) {
            const double x = carry + wave_scan64(e0 + lane < count ? s.sums[e0 + lane] : 0.0, lane);
            const uint64_t there = __ballot(e0 + lane < count && x >= target);
            if (there) { cut = e0 + __ffsll((unsigned long long)there) - 1; break; }
            carry = lane64(x, 63);
        }
        if (lane == 0) {  // (no other score like it behind the cut: all of them are kept)
            s.found[0] = (uint32_t)(list[cut] >> 32);
            s.found[1] = cut + 1 < count && (uint32_t)(list[cut + 1] >> 32) == s.found[0] ? (uint32_t)list[cut] : 0u;
        }
    }
    __syncthreads();
    const float t = key_score(s.found[0]);
    return {s.found[1] == 0 ? score_below(t) : t, t, s.found[1], 0u};
}

// What top-p keeps of a workgroup's scores.
template <int WAVES, int TPW, typename L>
__device__ __forceinline__ Kept cut_by_weight(float v[TPW * 4], const L& low, float best, float worst, const Weights& w, double inv_t, double top_p,
                                              CutScratch<WAVES, TPW>& s) {
    constexpr int N = TPW * 4, THREADS = WAVES * 64, BITS = 46;  // 2^15 scores of up to 2^47.5
    constexpr int ROOM = CutScratch<WAVES, TPW>::ROOM, LOG_BINS = CutScratch<WAVES, TPW>::LOG_BINS, BINS = 1 << LOG_BINS;
    BinRule<LOG_BINS> r = first_bins<LOG_BINS>(best, worst, inv_t);
    double target = 0.0, above = 0.0;
    int count = 0;
    for (int round = 0;; ++round) {
        __syncthreads();
        for (int b = threadIdx.x; b < BINS; b += THREADS) s.bins[b] = 0;
        __syncthreads();
        forget<N>(v);
#pragma unroll
        for (int q = 0; q < N; ++q) {
            if (round == 0 ? v[q] > -INFINITY : r.in(v[q])) {
                const int b = r.bin(v[q]);
                const uint64_t x = whole_weight(w, v[q], r.exponent(b), BITS);
                if (x) atomicAdd(reinterpret_cast<unsigned long long*>(&s.bins[b]), (unsigned long long)x);
            }
        }
        __syncthreads();
        const int b = find_bin<THREADS, LOG_BINS>(s.bins, r, BITS, round == 0, top_p, target, above, s.part, s.found);
        r = next_bins(r, b, w);
        const float t0 = key_score(r.lo), t1 = key_score(r.hi);
        int c = 0;
#pragma unroll
        for (int q = 0; q < N; ++q) c += __popcll(__ballot(v[q] >= t0 && v[q] <= t1));
        __syncthreads();
        count = block_count<WAVES>(c, s.slots);
        if (count <= ROOM || r.lo == r.hi) break;
    }
    Kept kept = {key_score(r.hi), key_score(r.hi), 0u, 0u};
    __syncthreads();
    if (count > ROOM) {  // all equal: as many as it takes, the first ones
        const double need = ceil((target - above) / w.of(kept.t));
        if (need < count) kept.least = select_equal<WAVES, N>(v, kept.t, low, need < 1.0 ? 1 : (int)need, s.slots);
        else kept.over = score_below(kept.t);
        return kept;
    }
    if (threadIdx.x == 0) s.count = 0;
    __syncthreads();
    const float t0 = key_score(r.lo), t1 = key_score(r.hi);
    uint32_t marked = 0;
#pragma unroll
    for (int q = 0; q < N; ++q) marked |= (uint32_t)(v[q] >= t0 && v[q] <= t1) << q;
    append_marked<N>(v, marked, low, s.bins, ROOM, &s.count);
    __syncthreads();
    return cut_list(count, target, above, w, s);
}

// The cut and the tiles' sums of what it keeps in one pass with weights in 64 bits, once few scores are left between those that are surely kept and
// those that are not; false where too many are left (equal scores, top-p close to 1).
template <int DT, int WAVES, int TPW, typename L>
__device__ __forceinline__ bool cut_enclosed(float v[TPW * 4], const L& low, float best, float worst, const Weights& w, const DrawArgs& a,
                                             CutScratch<WAVES, TPW>& s, double* sums, Kept& kept) {
    constexpr int N = TPW * 4, THREADS = WAVES * 64, TILES = WAVES * TPW, BITS = 46;
    constexpr int ROOM = CutScratch<WAVES, TPW>::ROOM;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t lo, hi;
    enclose<WAVES, TPW>(v, a.in.n, best, worst, a.inv_t, a.top_p, s, lo, hi);
    forget<N>(v);
    const float from = key_score(lo), to = key_score(hi);
    kept = {to, __uint_as_float(0x7FC00000u), 0u, 0u};
    keep_from_min_p(kept, w, best, a.min_p);
    const bool refine = !(kept.over > to);  // (else min-p leaves less than top-p)
    uint32_t marked = 0;
    double all = 0.0;
#pragma unroll
    for (int i = 0; i < TPW; i += 4) {
        if (i > 0 && i * WAVES * 256 >= a.in.n) {
            if ((lane & 15) == 15) sums[(i + tile_of_row(lane >> 4)) * WAVES + wave] = 0.0;
            continue;
        }
        double z[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            z[k] = 0.0;
            double sum = 0.0;
#pragma unroll
            for (int q = 4 * (i + k); q < 4 * (i + k) + 4; ++q) {
                const double y = best == INFINITY ? (v[q] == INFINITY ? 1.0 : 0.0) : w.loose(v[q], v[q] >= w.floor);
                sum += y;
                z[k] += __hiloint2double(v[q] > kept.over ? __double2hiint(y) : 0, __double2loint(y));
                marked |= (uint32_t)(v[q] >= from && v[q] <= to) << q;
            }
            all += sum;
        }
        const double sum = Weights::some_weight(sum_four(z));
        if ((lane & 15) == 15) sums[(i + tile_of_row(lane >> 4)) * WAVES + wave] = sum;
        __builtin_amdgcn_sched_barrier(0);
    }
    all = wave_sum64(all);
    if (lane == 0) s.part[wave] = all;
    if (!refine) { __syncthreads(); return true; }
    append_marked<N>(v, marked, low, s.bins, ROOM, &s.count);
    __syncthreads();
    const int count = (int)s.count;
    if (count > ROOM || count == 0) return false;
    all = wave_sum64(lane < WAVES ? s.part[lane] : 0.0);
    double above = lane < TILES ? sums[lane] : 0.0;
#pragma unroll
    for (int t = 64; t < TILES; t += 64) above += sums[t + lane];
    above = wave_sum64(above);
    kept = cut_list<WAVES, TPW>(count, a.top_p * all, above, w, s);
    keep_from_min_p(kept, w, best, a.min_p);
    int top;
    double p;
    w.split(to, p, top);
    const uint64_t* list = by_counting<THREADS>(count) ? s.sorted : s.bins;
    for (int e = threadIdx.x; e < count; e += THREADS) {
        const float x = key_score((uint32_t)(list[e] >> 32));
        const uint32_t position = ~(uint32_t)list[e];
        if (x > kept.over || (x == kept.t && (uint32_t)list[e] >= kept.least))
            atomicAdd(reinterpret_cast<unsigned long long*>(&s.more[position / 256]), (unsigned long long)whole_weight(w, x, top, BITS));
    }
    __syncthreads();
    for (int t = threadIdx.x; t < TILES; t += THREADS) sums[t] += ldexp((double)s.more[t], top - BITS);
    return true;
}

enum { CUT_MIN, CUT_WEIGHT, CUT_LIST };  // min-p alone; top-p and min-p; top-k and what follows it

template <int DT, int WAVES, int TPW, int CUT>
__global__ __launch_bounds__(WAVES * 64, WAVES == 8 && TPW == 8 ? (CUT == CUT_WEIGHT ? 4 : 6) : 1) void k_draw_rows(DrawArgs a) {
    constexpr int THREADS = WAVES * 64, N = TPW * 4, TILES = WAVES * TPW;
    __shared__ float maxima[WAVES];
    const int64_t row = flat_block();
    if (row >= a.in.rows) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const auto* s = static_cast<const typename Score<DT>::type*>(a.in.p) + row * a.in.ld;
    auto low = [&](int q) { return ~(uint32_t)tile_position<WAVES>(q); };

    float v[N];
    const float mine = load_tiles<DT, WAVES, TPW>(s, 0, a.in.n, v), best = block_max<WAVES>(mine, maxima);
    if (!(best > -INFINITY)) { write_empty<THREADS>(a, row); return; }

    if constexpr (CUT == CUT_LIST) {
        __shared__ BestList<WAVES, TPW> b;
        __shared__ double sums[BestList<WAVES, TPW>::ROOM < KGE_TOP_MAX ? BestList<WAVES, TPW>::ROOM : KGE_TOP_MAX];
        __shared__ int kept_entries;
        const int count = collect_best<WAVES, TPW>(v, low, mine, order_key(best), a.top_k, b);
        uint64_t* list = order_list<THREADS>(b.list, b.sorted, b.rank, count);
        draw_from_list<THREADS>(a, row, list, list == b.sorted ? b.list : b.sorted, b.rank, min(count, a.top_k), sums, &kept_entries);
    } else {
        __shared__ double sums[TILES];
        const Scale scale(a.inv_t);
        const Weights weights(best, scale);
        Kept kept = {-INFINITY, __uint_as_float(0x7FC00000u), 0u, 0u};
        if constexpr (CUT == CUT_WEIGHT) {
            __shared__ CutScratch<WAVES, TPW> scratch;
            float worst = INFINITY;
#pragma unroll
            for (int q = 0; q < N; ++q) worst = v[q] > -INFINITY ? fminf(worst, v[q]) : worst;
            worst = -block_max<WAVES>(-worst, maxima);
            // us, bins of 64-bit weights alone -> this first, 1 / 1024 rows: of 2000 16.9 -> 16.2 / 26.2 -> 22.8, of 15,000 26 -> 22 / 72 -> 60, of 30,000
            // 39 -> 32 / 163 -> 138; about equal whatever top_p and the temperature.  (Rows of up to 1024 have 4 scores per thread: no pass to save.)
            if constexpr (TPW % 4 == 0) {
                if (cut_enclosed<DT, WAVES, TPW>(v, low, best, worst, weights, a, scratch, sums, kept)) {
                    draw_from_tiles<DT, WAVES, TILES>(a, row, s, TILES, sums, nullptr, kept, weights);
                    return;
                }
            }
            kept = cut_by_weight<WAVES, TPW>(v, low, best, worst, weights, a.inv_t, a.top_p, scratch);
            forget<N>(v);
        }
        keep_from_min_p(kept, weights, best, a.min_p);
        const bool some = CUT == CUT_WEIGHT && kept.least > 0;  // of the equal ones some are not kept
        if constexpr (TPW % 4 == 0) {
#pragma unroll
            for (int i = 0; i < TPW; i += 4) {
                const double z = i * WAVES * 256 < a.in.n ? sum_of_tiles(v + 4 * i, weights, kept.over) : 0.0;
                if ((lane & 15) == 15) sums[(i + tile_of_row(lane >> 4)) * WAVES + wave] = z;
            }
        } else {
            double z = 0.0;
#pragma unroll
            for (int q = 0; q < 4; ++q) z += weights.of(v[q], v[q] > kept.over);
            z = wave_sum64(z);
            if (lane == 0) sums[wave] = z;
        }
        if (some) {
            const double each = weights.of(kept.t);
#pragma unroll
            for (int i = 0; i < TPW; ++i) {
                int c = 0;
#pragma unroll
                for (int q = 4 * i; q < 4 * i + 4; ++q) c += __popcll(__ballot(v[q] == kept.t && low(q) >= kept.least));
                if (lane == 0) sums[i * WAVES + wave] += (double)c * each;
            }
        }
        draw_from_tiles<DT, WAVES, TILES>(a, row, s, TILES, sums, nullptr, kept, weights);
    }
}

// top-k of long rows: the draws from the lists that k_top leaves
__global__ __launch_bounds__(256) void k_draw_lists(DrawArgs a, const uint64_t* lists) {
    __shared__ uint64_t list[KGE_TOP_MAX], spare[256];
    __shared__ double sums[KGE_TOP_MAX];
    __shared__ uint32_t filled, rank[256];
    __shared__ int kept_entries;
    const int64_t row = flat_block();
    if (row >= a.in.rows) return;
    if (threadIdx.x == 0) filled = 0;
    __syncthreads();
    for (int e0 = 0; e0 < a.top_k; e0 += 256) {
        const int e = e0 + threadIdx.x;
        const uint64_t x = e < a.top_k ? lists[row * a.top_k + e] : 0;
        if (e < a.top_k) list[e] = x;
        if (x) atomicMax(&filled, (uint32_t)(e + 1));
    }
    __syncthreads();
    draw_from_list<256>(a, row, list, spare, rank, (int)filled, sums, &kept_entries);
}

// ---------------------------------------------------------------------------------------------------------
// Long rows: groups of GROUP scores = GROUP_TILES tiles.  Sums per tile and group by k_tiles (nothing cut) or k_draw_sums (what is kept), running
// sums over the groups, then a wave per draw.
// top-p: rounds of bins over the whole row, each a launch; a launch finds the bin of the round before it by itself.  From the second round on few
// scores are left: the workgroups note those of their part of the row, and later rounds read the notes.
// ---------------------------------------------------------------------------------------------------------
constexpr int LOG_BINS = 11, BINS = 1 << LOG_BINS;
constexpr int ROUNDS = 4;  // bins of equal width, then 2^32 keys in three rounds
constexpr int PART_GROUPS = 4, NOTES = 1024;  // groups per workgroup of k_draw_bins (16: 178 us for 2 x 10 M where 4 took 148), scores that it can note

struct RowCut {
    BinRule<LOG_BINS> rule;
    double target, above;
    float best;
    uint32_t equal;    // scores of the interval, where it is a single key
    Kept kept;         // the result
};

struct LongArgs {
    DrawArgs d;
    int64_t groups, parts;  // of a row
    int bits;
    int by_weight;
    float* tile_best;       // [rows][groups][GROUP_TILES] what the tile's sum is relative to
    double* tile_sum;
    uint32_t* tile_ties;    // equal to the threshold
    float* group_best;      // [rows][groups]
    float* group_worst;
    double* group_sum;      // then running sums
    uint32_t* group_ties;   // then the number in front
    uint64_t* bins;         // [rows][ROUNDS][BINS]
    RowCut* cuts;           // [ROUNDS + 1][rows]: before each round, and the result
    uint32_t* notes;        // [rows][parts]: how many, more than NOTES: not noted
    float* noted;           // [rows][parts][NOTES]
};

// The row's cut before round `round` (ROUNDS: the result), by a workgroup of 256 threads.
__device__ __forceinline__ RowCut cut_before(const LongArgs& a, int64_t row, int round, float* maxima /* [4] */, double* part /* [5] */, uint32_t* found /* [2] */) {
    if (round == 0) {
        RowCut c = {};
        float best = -INFINITY, lowest = -INFINITY;
        for (int64_t g = threadIdx.x; g < a.groups; g += 256) {
            best = fmaxf(best, a.group_best[row * a.groups + g]);
            lowest = fmaxf(lowest, -a.group_worst[row * a.groups + g]);
        }
        c.best = block_max<4>(best, maxima);
        lowest = block_max<4>(lowest, maxima);
        if (c.best > -INFINITY) c.rule = first_bins<LOG_BINS>(c.best, -lowest, a.d.inv_t);
        return c;
    }
    RowCut c = a.cuts[(round - 1) * a.d.in.rows + row];
    if (!(c.best > -INFINITY)) return c;
    const Scale scale(a.d.inv_t);
    const Weights w(c.best, scale);
    if (round == 1 || c.rule.hi > c.rule.lo) {
        const uint64_t* bins = a.bins + (row * ROUNDS + round - 1) * BINS;
        const int b = find_bin<256, LOG_BINS>(bins, c.rule, a.bits, round == 1, a.d.top_p, c.target, c.above, part, found);
        const int exponent = c.rule.exponent(b);
        c.rule = next_bins(c.rule, b, w);
        if (c.rule.hi == c.rule.lo) {  // every score added the same number
            const uint64_t each = whole_weight(w, key_score(c.rule.hi), exponent, a.bits);
            c.equal = each ? (uint32_t)((bins[b] + each / 2) / each) : 0u;
        }
    }
    if (round == ROUNDS) {
        const float t = key_score(c.rule.hi);
        const double need = ceil((c.target - c.above) / w.of(t));
        const bool all = need >= (double)c.equal;
        c.kept = {all ? score_below(t) : t, all ? __uint_as_float(0x7FC00000u) : t, 0u, all ? 0u : need < 1.0 ? 1u : (uint32_t)need};
    }
    return c;
}

template <int DT>
__global__ __launch_bounds__(256) void k_draw_bins(LongArgs a, int round) {
    __shared__ unsigned long long bins[BINS];
    __shared__ float maxima[4];
    __shared__ double found_sum[5];
    __shared__ uint32_t found[2], noted;
    const int64_t block = flat_block();
    if (block >= a.d.in.rows * a.parts) return;
    const int64_t row = block / a.parts, part = block - row * a.parts;
    const RowCut c = cut_before(a, row, round, maxima, found_sum, found);
    if (part == 0 && threadIdx.x == 0) a.cuts[round * a.d.in.rows + row] = c;
    if (!(c.best > -INFINITY) || (round > 0 && c.rule.hi == c.rule.lo)) return;
    const Scale scale(a.d.inv_t);
    const Weights w(c.best, scale);
    for (int b = threadIdx.x; b < BINS; b += 256) bins[b] = 0;
    if (threadIdx.x == 0) noted = 0;
    __syncthreads();
    auto add = [&](float s) {
        const int b = c.rule.bin(s);
        const uint64_t x = whole_weight(w, s, c.rule.exponent(b), a.bits);
        if (x) atomicAdd(&bins[b], (unsigned long long)x);
    };
    const uint32_t have = round > 1 ? a.notes[block] : NOTES + 1;
    if (have <= NOTES) {
        for (uint32_t e = threadIdx.x; e < have; e += 256) {
            const float s = a.noted[block * NOTES + e];
            if (c.rule.in(s)) add(s);
        }
    } else {
        const auto* s = static_cast<const typename Score<DT>::type*>(a.d.in.p) + row * a.d.in.ld;
        const int64_t last = min((part + 1) * PART_GROUPS, a.groups);
        for (int64_t g = part * PART_GROUPS; g < last; ++g) {
            float v[16];
            load_tiles<DT, 4, 4>(s, g * GROUP, a.d.in.n, v);
            if (round == 0 && c.best < INFINITY) {  // (as add, without a branch per score)
#pragma unroll
                for (int q = 0; q < 16; ++q) {
                    const float at = floorf(fminf(c.rule.place(v[q]), (float)(BINS - 1)));
                    const double d = (double)v[q] - w.best, shifted = fma(d, scale.per, 0x1.8p52), f = fma(d, scale.per, -(shifted - 0x1.8p52));
                    double p = scale.c[8];
#pragma unroll
                    for (int i = 7; i >= 0; --i) p = fma(p, f, scale.c[i]);
                    const int up = __double2loint(shifted) - (int)floorf(-at * c.rule.drop) + a.bits;
                    const double x = Weights::scaled(fma(p, f, 1.0), up) + 0x1p52;
                    const bool some = v[q] >= w.floor && up >= -2;  // the others add 0, at places that do not collide
                    atomicAdd(&bins[some ? (int)at : (int)(threadIdx.x & 63)],
                              some ? (unsigned long long)__double_as_longlong(x) & (((uint64_t)1 << 52) - 1) : 0ull);
                    if (q % 4 == 3) __builtin_amdgcn_sched_barrier(0);
                }
            } else if (round == 0) {
#pragma unroll
                for (int q = 0; q < 16; ++q) if (v[q] > -INFINITY) add(v[q]);
            } else {
#pragma unroll
                for (int q = 0; q < 16; ++q) {
                    const bool in = c.rule.in(v[q]);
                    const uint64_t who = __ballot(in);
                    if (!who) continue;
                    if (round == 1) {
                        uint32_t base = 0;
                        if ((threadIdx.x & 63) == 0) base = atomicAdd(&noted, (uint32_t)__popcll(who));
                        base = (uint32_t)__builtin_amdgcn_readfirstlane((int)base) + __popcll(who & (((uint64_t)1 << (threadIdx.x & 63)) - 1));
                        if (in && base < NOTES) a.noted[block * NOTES + base] = v[q];
                    }
                    if (in) add(v[q]);
                }
            }
        }
    }
    __syncthreads();
    unsigned long long* out = reinterpret_cast<unsigned long long*>(a.bins) + (row * ROUNDS + round) * BINS;
    for (int b = threadIdx.x; b < BINS; b += 256)
        if (bins[b]) atomicAdd(&out[b], bins[b]);
    if (round == 1 && threadIdx.x == 0) a.notes[block] = noted;
}

// Sums of what is kept, relative to the row's best score.  (Ranges of groups as in k_tiles.)
template <int DT>
__global__ __launch_bounds__(256) void k_draw_sums(LongArgs a, int64_t per) {
    __shared__ double sums[2][GROUP_TILES];
    __shared__ uint32_t ties[2][GROUP_TILES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t blocks = a.d.in.rows * a.groups, start = (int64_t)flat_block() * per, end = min(start + per, blocks);
    if (start >= blocks) return;
    int64_t row = start / a.groups, group = start - row * a.groups;
    const auto* scores = static_cast<const typename Score<DT>::type*>(a.d.in.p);
    Quad<DT> x[4];
    auto load = [&](int64_t r, int64_t g) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i].load(scores + r * a.d.in.ld, g * GROUP + (wave * 4 + i) * 256 + lane * 4, a.d.in.n);
    };
    load(row, group);
    const Scale scale(a.d.inv_t);
    float best = -INFINITY;
    Kept kept = {};
    for (int64_t block = start; block < end; ++block) {
        if (block == start || group == 0) {
            const RowCut& c = a.cuts[ROUNDS * a.d.in.rows + row];
            best = c.best;
            kept = c.kept;
        }
        float v[16];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i].values(group * GROUP + (wave * 4 + i) * 256, a.d.in.n, v + 4 * i);
        if (++group == a.groups) { group = 0; ++row; }
        if (block + 1 < end) load(row, group);
        const int half = (int)(block - start) & 1;
        const double sum = sum_of_tiles(v, Weights(best, scale), kept.over);
        if (kept.ties) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t e = 0;
#pragma unroll
                for (int q = 4 * i; q < 4 * i + 4; ++q) e += __popcll(__ballot(v[q] == kept.t));
                if (lane == 0) ties[half][wave * 4 + i] = e;
            }
        }
        if ((lane & 15) == 15) sums[half][wave * 4 + tile_of_row(lane >> 4)] = sum;
        __syncthreads();
        if (wave != (int)(block & 3)) continue;
        const double y = lane < GROUP_TILES ? sums[half][lane] : 0.0;
        uint32_t e = kept.ties && lane < GROUP_TILES ? ties[half][lane] : 0;
        if (lane < GROUP_TILES) {
            a.tile_best[block * GROUP_TILES + lane] = best;
            a.tile_sum[block * GROUP_TILES + lane] = y;
            a.tile_ties[block * GROUP_TILES + lane] = e;
        }
        const double all = wave_sum64(y);
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) e += __shfl_xor((int)e, o, 64);
        if (lane == 0) { a.group_best[block] = best; a.group_sum[block] = all; a.group_ties[block] = e; }
    }
}

// The result of the rounds, or with min-p alone the row's best score, once for all workgroups of k_draw_sums.
__global__ __launch_bounds__(256) void k_draw_cut(LongArgs a) {
    __shared__ float maxima[4];
    __shared__ double found_sum[5];
    __shared__ uint32_t found[2];
    const int64_t row = flat_block();
    if (row >= a.d.in.rows) return;
    RowCut c = cut_before(a, row, a.by_weight ? ROUNDS : 0, maxima, found_sum, found);
    if (!a.by_weight) c.kept = {-INFINITY, __uint_as_float(0x7FC00000u), 0u, 0u};
    if (c.best > -INFINITY) {
        const Scale scale(a.d.inv_t);
        keep_from_min_p(c.kept, Weights(c.best, scale), c.best, a.d.min_p);
        if (!(c.kept.t == c.kept.t)) c.kept.ties = 0;
    }
    if (threadIdx.x == 0) a.cuts[ROUNDS * a.d.in.rows + row] = c;
}

// Running sums over the groups of a row.
__global__ __launch_bounds__(1024) void k_draw_scan(LongArgs a, int cut) {
    __shared__ double part[16];
    __shared__ uint32_t tpart[16];
    __shared__ float maxima[16];
    const int64_t row = flat_block();
    if (row >= a.d.in.rows) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const float* bests = a.group_best + row * a.groups;
    double* sums = a.group_sum + row * a.groups;
    uint32_t* ties = a.group_ties + row * a.groups;
    float best = -INFINITY;
    for (int64_t g = threadIdx.x; g < a.groups; g += 1024) best = fmaxf(best, bests[g]);
    best = block_max<16>(best, maxima);
    const Scale scale(a.d.inv_t);
    const Weights weights(best, scale);
    uint32_t most = 0;
    double each = 0.0;
    if (cut) {
        const RowCut& c = a.cuts[ROUNDS * a.d.in.rows + row];
        most = c.kept.ties;
        if (most) each = weights.of(c.kept.t);
    } else if (threadIdx.x == 0) {
        RowCut c = {};
        c.best = best;
        c.kept = {score_below(weights.floor), __uint_as_float(0x7FC00000u), 0u, 0u};
        a.cuts[ROUNDS * a.d.in.rows + row] = c;
    }
    double carry = 0.0;
    uint32_t tcarry = 0;
    for (int64_t g0 = 0; g0 < a.groups; g0 += 1024) {
        const int64_t g = g0 + threadIdx.x;
        double v = 0.0;
        uint32_t e = 0;
        if (g < a.groups) {
            v = bests[g] > -INFINITY ? sums[g] * weights.of(bests[g]) : 0.0;
            if (most) e = ties[g];
        }
        const uint32_t es = wave_scan_u32(e);  // equal scores up to this group
        if (lane == 63) tpart[wave] = es;
        __syncthreads();
        uint32_t ebase = tcarry;
        for (int w = 0; w < 16; ++w) {
            if (w < wave) ebase += tpart[w];
            tcarry += tpart[w];
        }
        const uint32_t before = ebase + es - e;
        if (before < most) v += each * (double)min(e, most - before);
        v = wave_scan64(v, lane);
        if (lane == 63) part[wave] = v;
        __syncthreads();
        double base = carry;
        for (int w = 0; w < 16; ++w) {
            if (w < wave) base += part[w];
            carry += part[w];
        }
        if (g < a.groups) {
            sums[g] = base + v;
            if (most) ties[g] = before;
        }
        __syncthreads();
    }
}

// One wave per draw: group, tile, position.
template <int DT>
__global__ __launch_bounds__(256) void k_draw_pick(LongArgs a) {
    const int lane = threadIdx.x & 63;
    const int64_t d = (int64_t)flat_block() * 4 + (threadIdx.x >> 6);
    if (d >= a.d.in.rows * a.d.draws) return;
    const int64_t row = d / a.d.draws;
    const auto* s = static_cast<const typename Score<DT>::type*>(a.d.in.p) + row * a.d.in.ld;
    const RowCut& c = a.cuts[ROUNDS * a.d.in.rows + row];
    const float best = c.best;
    const Kept kept = c.kept;
    const double* sums = a.group_sum + row * a.groups;
    const double total = sums[a.groups - 1];
    if (!(best > -INFINITY)) {
        if (lane == 0) {
            a.d.ids[d] = -1;
            if (a.d.logp) a.d.logp[d] = -INFINITY;
        }
        return;
    }
    const double want = unit_number(a.d.u[d]) * total;
    Probes groups = {0, a.groups - 1};  // the first group whose sum exceeds `want`
    while (groups.open()) {
        const uint64_t past = __ballot(sums[groups.at(lane)] > want);
        groups.narrow(past ? __ffsll((unsigned long long)past) - 1 : 63);
    }
    int64_t lo = groups.lo;
    const Scale scale(a.d.inv_t);
    const Weights weights(best, scale);
    double base, incl;
    uint32_t before;
    int tile;
    for (;; --lo) {  // (never a group without weight, whose running sum may be a rounding above the one before it)
        const int64_t group = row * a.groups + lo;
        base = lo > 0 ? sums[lo - 1] : 0.0;
        before = 0;
        double v = 0.0;
        uint32_t e = 0;
        if (lane < GROUP_TILES) {
            const float own = a.tile_best[group * GROUP_TILES + lane];
            v = own > -INFINITY ? a.tile_sum[group * GROUP_TILES + lane] * weights.of(own) : 0.0;
            if (kept.ties) e = a.tile_ties[group * GROUP_TILES + lane];
        }
        if (kept.ties) {
            before = a.group_ties[group] + wave_scan_u32(e) - e;
            if (before < kept.ties) v += weights.of(kept.t) * (double)min(e, kept.ties - before);
        }
        const uint64_t any = __ballot(v > 0.0);
        if (!any && lo > 0) continue;
        incl = base + wave_scan64(v, lane);
        const uint64_t past = __ballot(incl > want && v > 0.0);
        tile = past ? __ffsll((unsigned long long)past) - 1 : any ? 63 - __clzll(any) : 0;
        incl -= v;
        break;
    }
    int64_t id = -1;
    double weight = 0.0;
#pragma unroll 1
    for (int j = 0; j < 4 && id < 0; ++j) {
        const int t = j == 0 ? tile : other_of_four(tile, j);
        const int64_t first = lo * GROUP + (int64_t)t * 256;
        Quad<DT> x;
        x.load(s, first + lane * 4, a.d.in.n);
        draw_in_tile<DT, true>(x, first, a.d.in.n, kept, weights, (uint32_t)__shfl((int)before, t, 64), lane64(incl, t), want, lane, id, weight);
    }
    if (lane == 0) {
        a.d.ids[d] = id;
        if (a.d.logp) a.d.logp[d] = (float)log(weight / total);
    }
}

template <int DT, int CUT>
void launch_rows(const DrawArgs& a, hipStream_t st) {
    const int64_t n = a.in.n;
    const dim3 grid = flat_grid(a.in.rows);
    if (n <= 256) k_draw_rows<DT, 1, 1, CUT><<<grid, 64, 0, st>>>(a);
    else if (n <= 1024) k_draw_rows<DT, 4, 1, CUT><<<grid, 256, 0, st>>>(a);
    else if (n <= 4096) k_draw_rows<DT, 4, 4, CUT><<<grid, 256, 0, st>>>(a);
    // us, 16 / 1024 / 4096 rows of 5000, by the kernel for 16,384 -> by this: top-p 20 -> 17.6 / 48 -> 41 / 181 -> 154, min-p 7.9 -> 7.0 / 18.3 -> 16.2 /
    // 61 -> 52, top-k 50 12.0 -> 10.5 / 23.5 -> 20.5 / 70 -> 60
    else if (n <= 8192) k_draw_rows<DT, 8, 4, CUT><<<grid, 512, 0, st>>>(a);
    // (1024 threads of half as many scores are as fast up to 256 rows.  us, 512 / 4096 rows of 15,000, 1024 -> 512 threads: top-p 46 -> 32 / 360 -> 221,
    // min-p 17.3 -> 12.7 / 122 -> 73, top-k 50 22.6 -> 13.8 / 165 -> 72)
    else if (n <= 16384) k_draw_rows<DT, 8, 8, CUT><<<grid, 512, 0, st>>>(a);
    else k_draw_rows<DT, 16, 8, CUT><<<grid, 1024, 0, st>>>(a);
}

template <int DT>
void launch_whole(const DrawArgs& a, hipStream_t st) {
    const int64_t tiles = pieces(a.in.n, 256);
    const dim3 grid = flat_grid(a.in.rows);
    // us, 4 draws, 16 -> 4 waves: rows of 4000, 256 / 512 of them 7.8 -> 8.3 / 11.5 -> 8.2; rows of 15,000 9.9 -> 11.1 / 15.9 -> 14.2, 4096 of
    // them 95 -> 64; rows of 32,768 13.7 -> 16.9 / 26.7 -> 24.5
    if (tiles <= 4) k_draw_whole<DT, 1><<<grid, 64, 0, st>>>(a);
    else if (tiles <= 16 || a.in.rows > 256) k_draw_whole<DT, 4><<<grid, 256, 0, st>>>(a);
    else k_draw_whole<DT, 16><<<grid, 1024, 0, st>>>(a);
}

// The pieces of the workspace of long rows; returns its size.
int64_t carve(LongArgs* a, char* base, int64_t rows, int64_t n, bool by_weight) {
    const int64_t groups = pieces(n, GROUP), blocks = rows * groups, parts = pieces(groups, PART_GROUPS);
    int64_t off = 0;
    auto take = [&](int64_t bytes) { const int64_t o = off; off += up256(bytes); return base ? base + o : nullptr; };
    char* tile_best = take(blocks * GROUP_TILES * 4);
    char* tile_sum = take(blocks * GROUP_TILES * 8);
    char* tile_ties = take(blocks * GROUP_TILES * 4);
    char* group_best = take(blocks * 4);
    char* group_worst = take(blocks * 4);
    char* group_sum = take(blocks * 8);
    char* group_ties = take(blocks * 4);
    char* cuts = take((ROUNDS + 1) * rows * (int64_t)sizeof(RowCut));
    char* bins = by_weight ? take(rows * ROUNDS * BINS * 8) : nullptr;
    char* notes = by_weight ? take(rows * parts * 4) : nullptr;
    char* noted = by_weight ? take(rows * parts * NOTES * 4) : nullptr;
    if (a) {
        a->groups = groups;
        a->parts = parts;
        a->tile_best = reinterpret_cast<float*>(tile_best);
        a->tile_sum = reinterpret_cast<double*>(tile_sum);
        a->tile_ties = reinterpret_cast<uint32_t*>(tile_ties);
        a->group_best = reinterpret_cast<float*>(group_best);
        a->group_worst = reinterpret_cast<float*>(group_worst);
        a->group_sum = reinterpret_cast<double*>(group_sum);
        a->group_ties = reinterpret_cast<uint32_t*>(group_ties);
        a->cuts = reinterpret_cast<RowCut*>(cuts);
        a->bins = reinterpret_cast<uint64_t*>(bins);
        a->notes = reinterpret_cast<uint32_t*>(notes);
        a->noted = reinterpret_cast<float*>(noted);
    }
    return off;
}

template <int DT>
void launch(const DrawArgs& d, void* workspace, hipStream_t st) {
    const bool by_weight = d.top_k == 0 && d.top_p < 1.0;
    if (d.in.n <= KGE_ROW_RESIDENT) {
        if (d.top_k > 0) launch_rows<DT, CUT_LIST>(d, st);
        else if (by_weight) launch_rows<DT, CUT_WEIGHT>(d, st);
        else if (d.min_p > 0.0) launch_rows<DT, CUT_MIN>(d, st);
        else launch_whole<DT>(d, st);
        return;
    }
    LongArgs a = {};
    a.d = d;
    carve(&a, static_cast<char*>(workspace), d.in.rows, d.in.n, by_weight);
    a.by_weight = by_weight;
    const bool cut = by_weight || d.min_p > 0.0;
    a.bits = 50;  // n weights of up to 2^(bits + 1.5) in 64 bits
    while (((int64_t)1 << (61 - a.bits)) < d.in.n) --a.bits;
    TileArgs t = {};
    t.in = d.in; t.inv_t = d.inv_t; t.groups = a.groups;
    t.group_best = a.group_best;
    if (cut) t.group_worst = a.group_worst;
    else { t.tile_best = a.tile_best; t.tile_sum = a.tile_sum; t.group_sum = a.group_sum; }
    if (by_weight) { t.clear = a.bins; t.clear_words = ROUNDS * BINS; }
    kge_launch_tiles(t, cut ? TILES_RANGE : TILES_SUMS, st);
    const dim3 rows = flat_grid(d.in.rows);
    if (by_weight) {
        for (int round = 0; round < ROUNDS; ++round) k_draw_bins<DT><<<flat_grid(d.in.rows * a.parts), 256, 0, st>>>(a, round);
    }
    if (cut) {
        const int64_t blocks = d.in.rows * a.groups, per = groups_per_workgroup(blocks);
        k_draw_cut<<<rows, 256, 0, st>>>(a);
        k_draw_sums<DT><<<flat_grid(pieces(blocks, per)), 256, 0, st>>>(a, per);
    }
    k_draw_scan<<<rows, 1024, 0, st>>>(a, cut);
    k_draw_pick<DT><<<flat_grid(pieces(d.in.rows * d.draws, 4)), 256, 0, st>>>(a);
}

}  // namespace

int64_t kge_draw_workspace(int64_t rows, int64_t n, int top_k, float top_p) {
    if (n <= KGE_ROW_RESIDENT) return 0;
    if (top_k > 0) return kge_top_workspace(rows, n, top_k) + up256(rows * (int64_t)top_k * 8);
    return carve(nullptr, nullptr, rows, n, top_p < 1.f);
}

void kge_launch_draw(const RowScores& in, const double* u, int draws, float temperature, int top_k, float top_p, float min_p, int64_t* ids,
                     float* logp, void* workspace, hipStream_t st) {
    DrawArgs a = {};
    a.in = in; a.u = u; a.draws = draws; a.top_k = top_k;
    a.inv_t = 1.0 / (double)temperature; a.top_p = (double)top_p; a.min_p = (double)min_p;
    a.ids = ids; a.logp = logp;
    if (top_k > 0 && in.n > KGE_ROW_RESIDENT) {
        char* ws = static_cast<char*>(workspace);
        uint64_t* lists = reinterpret_cast<uint64_t*>(ws);
        const bool by_tiles = kge_top_by_tiles(in.n, top_k);
        kge_launch_top(in, top_k, 1.f, nullptr, nullptr, lists, nullptr, by_tiles ? &a : nullptr, ws + up256(in.rows * (int64_t)top_k * 8), st);
        if (!by_tiles) k_draw_lists<<<flat_grid(in.rows), 256, 0, st>>>(a, lists);
        return;
    }
    if (in.dtype == KGE_F32) launch<KGE_F32>(a, workspace, st);
    else if (in.dtype == KGE_BF16) launch<KGE_BF16>(a, workspace, st);
    else launch<KGE_F16>(a, workspace, st);
}
