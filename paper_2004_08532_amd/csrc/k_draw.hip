// Candidates drawn from rows of scores by given random numbers (kge_sample_scores).
//
// With w_j = exp((s_j - best) / T) the candidates kept are the first K in order of their scores: K the least of top-k, the number that
// top-p takes (the fewest whose w reach top_p times the sum over the first top_k) and the number with w_j >= min_p.  A number u in
// [0, 1) falls on the first position j at which the sum of the kept w up to j exceeds u times the whole sum.
//
// Sums are kept per tile of 256 scores; a draw is a wave that finds its tile among the sums and its position in the tile.  All sums are
// formed in 64 bits, in a fixed order or as whole numbers, so a draw depends on the row and its number alone.
#include "k_rows.h"

namespace {

struct DrawArgs {
    RowScores in;
    const double* u;  // [rows][draws]
    int draws, top_k;
    double inv_t, top_p, min_p;
    int64_t* ids;
    float* logp;
};

__device__ __forceinline__ double unit_number(double u) { return u > 0.0 ? u : 0.0; }  // (NaN: 0)

template <int THREADS> __device__ __forceinline__ void write_empty(const DrawArgs& a, int64_t row) {
    for (int d = threadIdx.x; d < a.draws; d += THREADS) {
        a.ids[row * a.draws + d] = -1;
        if (a.logp) a.logp[row * a.draws + d] = -INFINITY;
    }
}

// What is kept, of scores with a weight of at least min_p: those above t, and of those equal to it the ones whose inverted position is
// at least `least`, or the first `ties` of the row.
struct Kept {
    float t;
    uint32_t least, ties;
};

// Position in a tile (256 scores from `first` on) at which the sum passes `target`, `base` of it in front of the tile; the tile's
// last kept position where rounding leaves none.  COUNTED: equal scores are kept by `ties`, `ties_before` of them lie in front of the tile.
template <int DT, bool COUNTED>
__device__ __forceinline__ void draw_in_tile(const typename Score<DT>::type* s, int64_t first, int64_t n, const Kept& k, const Weights& weights, double min_p,
                                             uint32_t ties_before, double base, double target, int lane, int64_t& id, double& weight) {
    float v[4];
    load4<DT>(s, first + lane * 4, n, v);
    double w[4], sum = 0.0;
    uint32_t rank = ties_before;
    if constexpr (COUNTED) {
        const uint64_t below = ((uint64_t)1 << lane) - 1;
#pragma unroll
        for (int q = 0; q < 4; ++q) rank += __popcll(__ballot(v[q] == k.t) & below);
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        v[q] = fmaxf(v[q], -INFINITY);
        const bool equal = v[q] == k.t, in = v[q] > k.t || (equal && (COUNTED ? rank < k.ties : ~(uint32_t)(first + lane * 4 + q) >= k.least));
        w[q] = in ? weights.of(v[q]) : 0.0;
        rank += equal;
        if (!(w[q] >= min_p)) w[q] = 0.0;
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

// The draws from a sorted list of the row's best candidates.  list: LDS, KGE_TOP_MAX entries, the first `count` of them
// filled; sums: LDS, as many.
template <int THREADS>
__device__ __forceinline__ void draw_from_list(const DrawArgs& a, int64_t row, uint64_t* list, int count, double* sums, int* kept) {
    if (count == 0) { write_empty<THREADS>(a, row); return; }
    const int lane = threadIdx.x & 63;
    const Weights weights(key_score((uint32_t)(list[0] >> 32)), a.inv_t);
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
    const int size = power_of_two(count);
    // into the order of positions; the key goes below the inverted position
    for (int e = threadIdx.x; e < size; e += THREADS) list[e] = e < count ? list[e] << 32 | list[e] >> 32 : 0;
    sort_descending<THREADS>(list, size);
    for (int e = threadIdx.x; e < count; e += THREADS) sums[e] = weights.of(key_score((uint32_t)list[e]));
    scan(count);
    const double total = sums[count - 1];
    for (int d = threadIdx.x; d < a.draws; d += THREADS) {
        const double want = unit_number(a.u[row * a.draws + d]) * total;
        int lo = 0, hi = count - 1;  // first entry whose running sum exceeds `want`, the last one where none does
        while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if (sums[mid] > want) hi = mid; else lo = mid + 1;
        }
        while (lo > 0 && !(sums[lo] > sums[lo - 1])) --lo;  // (an entry without weight is never drawn)
        a.ids[row * a.draws + d] = (int64_t)(uint32_t)~(uint32_t)(list[lo] >> 32);
        if (a.logp) a.logp[row * a.draws + d] = (float)log(weights.of(key_score((uint32_t)list[lo])) / total);
    }
}

enum { CUT_NONE, CUT_WEIGHT, CUT_LIST };  // whole row or min-p; top-p; top-k (and what follows it)

template <int DT, int WAVES, int TPW, int CUT>
__global__ __launch_bounds__(WAVES * 64) void k_draw_rows(DrawArgs a) {
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
        draw_from_list<THREADS>(a, row, list, min(count, a.top_k), sums, &kept_entries);
    } else {
        __shared__ double sums[TILES], part[2 * WAVES];
        __shared__ uint32_t slots[2 * WAVES];
        const Weights weights(best, a.inv_t);
        Kept kept = {-INFINITY, 0u, 0u};
        double w[N];
#pragma unroll
        for (int q = 0; q < N; ++q) w[q] = weights.of(v[q]);
        if constexpr (CUT == CUT_WEIGHT) {
            int round = 0;
            auto weight_from = [&](uint32_t key) {  // of the scores at or above a key's
                const float t = key_score(key);
                double z = 0.0;
#pragma unroll
                for (int q = 0; q < N; ++q) z += v[q] >= t ? w[q] : 0.0;
                z = wave_sum64(z);
                if constexpr (WAVES == 1) return z;
                double* p = part + (round++ & 1) * WAVES;
                if (lane == 0) p[wave] = z;
                __syncthreads();
                z = 0.0;
#pragma unroll
                for (int x = 0; x < WAVES; ++x) z += p[x];
                return z;
            };
            const double target = a.top_p * weight_from(LOWEST_KEY);
            uint32_t lo = LOWEST_KEY, hi = order_key(best);  // largest threshold that reaches the target
            while (lo < hi) {
                const uint32_t mid = lo + (hi - lo) / 2 + ((hi - lo) & 1);
                if (weight_from(mid) >= target) lo = mid; else hi = mid - 1;
            }
            kept.t = key_score(lo);
            int equal = 0;
#pragma unroll
            for (int q = 0; q < N; ++q) equal += __popcll(__ballot(v[q] == kept.t));
            __syncthreads();
            equal = block_count<WAVES>(equal, slots);
            const double above = lo < order_key(best) ? weight_from(lo + 1) : 0.0;
            const double need = ceil((target - above) / weights.of(kept.t));
            const int c = need >= equal ? equal : need < 1.0 ? 1 : (int)need;
            if (c < equal) kept.least = select_equal<WAVES, N>(v, kept.t, low, c, slots);
        }
#pragma unroll
        for (int i = 0; i < TPW; ++i) {
            double z = 0.0;
#pragma unroll
            for (int q = 4 * i; q < 4 * i + 4; ++q) {
                const bool in = CUT == CUT_NONE || v[q] > kept.t || (v[q] == kept.t && low(q) >= kept.least);
                z += in && w[q] >= a.min_p ? w[q] : 0.0;
            }
            z = wave_sum64(z);
            if (lane == 0) sums[i * WAVES + wave] = z;
        }
        __syncthreads();
        if (wave == 0) {
            double carry = 0.0;
#pragma unroll
            for (int t0 = 0; t0 < TILES; t0 += 64) {
                const double x = carry + wave_scan64(t0 + lane < TILES ? sums[t0 + lane] : 0.0, lane);
                if (t0 + lane < TILES) sums[t0 + lane] = x;
                carry = __shfl(x, 63, 64);
            }
        }
        __syncthreads();
        const double total = sums[TILES - 1];
        for (int d = wave; d < a.draws; d += WAVES) {
            const double want = unit_number(a.u[row * a.draws + d]) * total;
            int tile = -1, fallback = 0;
#pragma unroll
            for (int t0 = 0; t0 < TILES; t0 += 64) {
                const bool there = t0 + lane < TILES;
                const double x = there ? sums[t0 + lane] : 0.0, before = t0 + lane > 0 && there ? sums[t0 + lane - 1] : 0.0;
                const uint64_t past = __ballot(there && x > want), some = __ballot(there && x > before);
                if (tile < 0 && past) tile = t0 + __ffsll((unsigned long long)past) - 1;
                if (some) fallback = t0 + 63 - __clzll(some);
            }
            if (tile < 0) tile = fallback;
            int64_t id = -1;
            double weight = 0.0;
            draw_in_tile<DT, false>(s, (int64_t)tile * 256, a.in.n, kept, weights, a.min_p, 0u, tile > 0 ? sums[tile - 1] : 0.0, want, lane, id, weight);
            if (lane == 0) {
                a.ids[row * a.draws + d] = id;
                if (a.logp) a.logp[row * a.draws + d] = (float)log(weight / total);
            }
        }
    }
}

// top-k of long rows: the draws from the lists that k_top leaves
__global__ __launch_bounds__(256) void k_draw_lists(DrawArgs a, const uint64_t* lists) {
    __shared__ uint64_t list[KGE_TOP_MAX];
    __shared__ double sums[KGE_TOP_MAX];
    __shared__ uint32_t filled;
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
    draw_from_list<256>(a, row, list, (int)filled, sums, &kept_entries);
}

// ---------------------------------------------------------------------------------------------------------
// Long rows, segments of KGE_ROW_SEGMENT scores = SEG_TILES tiles.
// Weights as whole numbers, for sums whose order is not fixed: w * 2^bits, and the next `bits` bits behind the point in a word of their
// own; bits is such that the sum of either word over a row stays below 2^63.
// ---------------------------------------------------------------------------------------------------------
constexpr int SEG_WAVES = 16, SEG_TPW = 4, SEG_TILES = SEG_WAVES * SEG_TPW, BINS = 2048, LEVELS = 3;

struct RowCut {
    uint32_t lo, hi;      // the threshold's key is in lo .. hi
    uint32_t t, ties;     // the result
    uint64_t above[2];    // weights of the keys above hi
    double target;        // in units of the second word
    float best;
    int pad;
};

struct LongArgs {
    DrawArgs d;
    int segments, bits, cut;  // cut: anything is left out
    double* parts;        // [rows][segments][2] best score and sum of a segment, then running sums over the segments
    double* tiles;        // [rows][segments][SEG_TILES] sums
    uint32_t* tile_ties;  // [rows][segments][SEG_TILES] keys equal to the threshold
    uint32_t* seg_ties;   // [rows][segments]
    uint64_t* bins;       // [LEVELS][rows][BINS][2]
    RowCut* rows;
};

// Sums per tile.  First pass (PASS 0): relative to the segment's own best score, which it notes.  PASS 1: what is kept, relative to
// the row's.
template <int DT, int PASS>
__global__ __launch_bounds__(SEG_WAVES * 64) void k_draw_sums(LongArgs a) {
    __shared__ uint32_t slots[SEG_WAVES];
    __shared__ float maxima[SEG_WAVES];
    __shared__ double sums[SEG_WAVES];
    const int64_t block = flat_block();
    if (block >= a.d.in.rows * a.segments) return;
    const int64_t row = block / a.segments, seg = block - row * a.segments;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const auto* s = static_cast<const typename Score<DT>::type*>(a.d.in.p) + row * a.d.in.ld;
    float v[SEG_TPW * 4];
    const float mine = load_tiles<DT, SEG_WAVES, SEG_TPW>(s, seg * KGE_ROW_SEGMENT, a.d.in.n, v);
    float t = -INFINITY, best;
    if constexpr (PASS == 0) {
        best = block_max<SEG_WAVES>(mine, maxima);
        if (a.bins) {  // clear the row's bins
            const int64_t words = 2 * BINS;
            for (int level = 0; level < LEVELS; ++level)
                for (int64_t x = seg * 1024 + threadIdx.x; x < words; x += a.segments * 1024)
                    a.bins[((int64_t)level * a.d.in.rows + row) * words + x] = 0;
        }
    } else {
        best = a.rows[row].best;
        if (a.rows[row].t) t = key_score(a.rows[row].t);
    }
    const Weights weights(best, a.d.inv_t);
    const double min_p = PASS == 0 ? 0.0 : a.d.min_p;
    double all = 0.0;
    uint32_t equal = 0;
#pragma unroll
    for (int i = 0; i < SEG_TPW; ++i) {
        double z = 0.0;
        uint32_t e = 0;
#pragma unroll
        for (int q = 4 * i; q < 4 * i + 4; ++q) {
            const double w = v[q] > t ? weights.of(v[q]) : 0.0;
            z += w >= min_p ? w : 0.0;
            if constexpr (PASS == 1) e += t > -INFINITY ? __popcll(__ballot(v[q] == t)) : 0;
        }
        z = wave_sum64(z);
        all += z;
        equal += e;
        if (lane == 0) {
            const int64_t tile = block * SEG_TILES + i * SEG_WAVES + wave;
            a.tiles[tile] = z;
            if constexpr (PASS == 1) a.tile_ties[tile] = e;
        }
    }
    if (lane == 0) { sums[wave] = all; slots[wave] = equal; }
    __syncthreads();
    if (threadIdx.x == 0) {
        double z = 0.0;
        uint32_t e = 0;
        for (int w = 0; w < SEG_WAVES; ++w) { z += sums[w]; e += slots[w]; }
        a.parts[2 * block] = best;
        a.parts[2 * block + 1] = z;
        if constexpr (PASS == 1) a.seg_ties[block] = e;
    }
}

// The row's best score; with top-p the interval in which its threshold is looked for.
__global__ __launch_bounds__(256) void k_draw_begin(LongArgs a) {
    __shared__ float maxima[4];
    const int64_t row = flat_block();
    if (row >= a.d.in.rows) return;
    float best = -INFINITY;
    for (int64_t g = threadIdx.x; g < a.segments; g += 256) best = fmaxf(best, (float)a.parts[2 * (row * a.segments + g)]);
    best = block_max<4>(best, maxima);
    if (threadIdx.x == 0) {
        RowCut r = {};
        r.best = best;
        r.lo = LOWEST_KEY; r.hi = order_key(best);
        a.rows[row] = r;
    }
}

__device__ __forceinline__ int bin_shift(uint32_t lo, uint32_t hi) { return max(0, 32 - __clz(hi - lo) - 11); }  // hi > lo

// Weights of the keys in the row's interval, by bin.
template <int DT>
__global__ __launch_bounds__(SEG_WAVES * 64) void k_draw_bins(LongArgs a, int level) {
    __shared__ unsigned long long bins[BINS * 2];
    const int64_t block = flat_block();
    if (block >= a.d.in.rows * a.segments) return;
    const int64_t row = block / a.segments, seg = block - row * a.segments;
    const RowCut r = a.rows[row];
    const auto* s = static_cast<const typename Score<DT>::type*>(a.d.in.p) + row * a.d.in.ld;
    for (int x = threadIdx.x; x < BINS * 2; x += 1024) bins[x] = 0;
    float v[SEG_TPW * 4];
    load_tiles<DT, SEG_WAVES, SEG_TPW>(s, seg * KGE_ROW_SEGMENT, a.d.in.n, v);
    __syncthreads();
    const Weights weights(r.best, a.d.inv_t);
    const int shift = r.hi > r.lo ? bin_shift(r.lo, r.hi) : 0;
    const double unit = (double)((uint64_t)1 << a.bits);
#pragma unroll
    for (int q = 0; q < SEG_TPW * 4; ++q) {
        const uint32_t key = order_key(v[q]);
        if (key >= r.lo && key <= r.hi) {
            const int bin = (int)((r.hi - key) >> shift);
            const double w = weights.of(v[q]) * unit, whole = floor(w);
            const uint64_t x = (uint64_t)whole, y = (uint64_t)((w - whole) * unit);
            if (x) atomicAdd(&bins[2 * bin], (unsigned long long)x);
            if (y) atomicAdd(&bins[2 * bin + 1], (unsigned long long)y);
        }
    }
    __syncthreads();
    unsigned long long* out = reinterpret_cast<unsigned long long*>(a.bins) + ((int64_t)level * a.d.in.rows + row) * BINS * 2;
    for (int x = threadIdx.x; x < BINS * 2; x += 1024)
        if (bins[x]) atomicAdd(&out[x], bins[x]);
}

// The bin in which the running sum, from the best key down, reaches the target becomes the interval.
__global__ __launch_bounds__(256) void k_draw_narrow(LongArgs a, int level) {
    constexpr int PER = BINS / 256;
    __shared__ uint64_t wave_part[2][4];
    __shared__ uint32_t found;
    const int64_t row = flat_block();
    if (row >= a.d.in.rows) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    RowCut r = a.rows[row];
    if (!(r.best > -INFINITY)) return;  // no candidate
    const uint64_t* bins = a.bins + ((int64_t)level * a.d.in.rows + row) * BINS * 2 + threadIdx.x * PER * 2;
    uint64_t x[PER][2], sum[2] = {0, 0};
#pragma unroll
    for (int q = 0; q < PER; ++q)
#pragma unroll
        for (int h = 0; h < 2; ++h) { x[q][h] = bins[2 * q + h]; sum[h] += x[q][h]; }
    uint64_t before[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint64_t v = sum[h];
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const uint64_t y = __shfl_up((unsigned long long)v, o, 64);
            if (lane >= o) v += y;
        }
        if (lane == 63) wave_part[h][wave] = v;
        before[h] = v - sum[h];
    }
    if (threadIdx.x == 0) found = BINS;
    __syncthreads();
    const double unit = (double)((uint64_t)1 << a.bits);
    uint64_t all[2] = {0, 0};
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            if (w < wave) before[h] += wave_part[h][w];
            all[h] += wave_part[h][w];
        }
    auto whole = [&](const uint64_t v[2]) { return ((unsigned __int128)v[0] << a.bits) + v[1]; };
    auto number = [&](double v) {  // to a whole number, v >= 0 and below 2^126
        const double high = floor(v * 0x1p-63);
        return ((unsigned __int128)(uint64_t)high << 63) + (uint64_t)(v - high * 0x1p63);
    };
    if (level == 0) {
        const unsigned __int128 z = whole(all);
        r.target = a.d.top_p * ((double)(uint64_t)(z >> 63) * 0x1p63 + (double)(uint64_t)(z & (((unsigned __int128)1 << 63) - 1)));
    }
    const unsigned __int128 want = number(r.target);
    uint64_t run[2] = {r.above[0] + before[0], r.above[1] + before[1]};
    uint64_t above[PER][2];
    int mine = BINS;
#pragma unroll
    for (int q = 0; q < PER; ++q) {
        above[q][0] = run[0]; above[q][1] = run[1];
        run[0] += x[q][0]; run[1] += x[q][1];
        if (mine == BINS && (x[q][0] | x[q][1]) && whole(run) >= want) mine = threadIdx.x * PER + q;
    }
    if (mine < BINS) atomicMin(&found, (uint32_t)mine);
    __syncthreads();
    // rounding of the target may leave no bin: the last one that holds anything
    if (found == BINS) {
        int last = -1;
#pragma unroll
        for (int q = 0; q < PER; ++q) if (x[q][0] | x[q][1]) last = threadIdx.x * PER + q;
        __syncthreads();
        if (threadIdx.x == 0) found = 0;
        __syncthreads();
        if (last >= 0) atomicMax(&found, (uint32_t)last);
        __syncthreads();
    }
    if ((int)(found / PER) == (int)threadIdx.x) {
        const int q = found % PER;
        const int shift = r.hi > r.lo ? bin_shift(r.lo, r.hi) : 0;
        uint64_t over[2] = {0, 0};
#pragma unroll
        for (int v = 0; v < PER; ++v) if (v == q) { over[0] = above[v][0]; over[1] = above[v][1]; }
        r.above[0] = over[0]; r.above[1] = over[1];
        const uint32_t top = r.hi - ((uint32_t)found << shift), width = (uint32_t)1 << shift;
        r.hi = top;
        r.lo = top >= width && top - width + 1 > r.lo ? top - width + 1 : r.lo;
        if (level == LEVELS - 1) {
            r.t = r.hi;
            const double w = Weights(r.best, a.d.inv_t).of(key_score(r.t)) * unit, down = floor(w);
            const uint64_t one[2] = {(uint64_t)down, (uint64_t)((w - down) * unit)};
            const unsigned __int128 each = whole(one), have = whole(r.above);
            unsigned __int128 c = 1;
            if (want > have && each > 0) c = (want - have + each - 1) / each;
            r.ties = c < 1 ? 1 : c > 0xFFFFFFFFu ? 0xFFFFFFFFu : (uint32_t)c;
        }
        a.rows[row] = r;
    }
}

// Running sums over the segments of a row.
__global__ __launch_bounds__(1024) void k_draw_scan(LongArgs a) {
    __shared__ double part[16];
    __shared__ uint32_t tpart[16];
    __shared__ float maxima[16];
    const int64_t row = flat_block();
    if (row >= a.d.in.rows) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    double* parts = a.parts + 2 * row * a.segments;
    float best = -INFINITY;
    for (int64_t g = threadIdx.x; g < a.segments; g += 1024) best = fmaxf(best, (float)parts[2 * g]);
    best = block_max<16>(best, maxima);
    const Weights weights(best, a.d.inv_t);
    uint32_t t = 0, most = 0;
    double each = 0.0;
    if (a.cut) {
        const RowCut r = a.rows[row];
        t = r.t; most = r.ties;
        if (t) {
            each = weights.of(key_score(t));
            if (!(each >= a.d.min_p)) each = 0.0;
        }
    } else if (threadIdx.x == 0) {
        RowCut r = {};
        r.best = best;
        a.rows[row] = r;
    }
    double carry = 0.0;
    uint32_t tcarry = 0;
    for (int64_t g0 = 0; g0 < a.segments; g0 += 1024) {
        const int64_t g = g0 + threadIdx.x;
        double v = 0.0;
        uint32_t e = 0;
        if (g < a.segments) {
            const float own = (float)parts[2 * g];
            v = own > -INFINITY ? parts[2 * g + 1] * weights.of(own) : 0.0;
            if (t) e = a.seg_ties[row * a.segments + g];
        }
        uint32_t es = e;  // equal keys up to this segment
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const uint32_t y = __shfl_up((int)es, o, 64);
            if (lane >= o) es += y;
        }
        if (lane == 63) tpart[wave] = es;
        __syncthreads();
        uint32_t ebase = tcarry;
        for (int w = 0; w < 16; ++w) {
            if (w < wave) ebase += tpart[w];
            tcarry += tpart[w];
        }
        const uint32_t before = ebase + es - e;
        if (t && before < most) v += each * (double)min(e, most - before);
        v = wave_scan64(v, lane);
        if (lane == 63) part[wave] = v;
        __syncthreads();
        double base = carry;
        for (int w = 0; w < 16; ++w) {
            if (w < wave) base += part[w];
            carry += part[w];
        }
        if (g < a.segments) {
            parts[2 * g + 1] = base + v;
            if (t) a.seg_ties[row * a.segments + g] = before;
        }
        __syncthreads();
    }
}

// One wave per draw: segment, tile, position.
template <int DT>
__global__ __launch_bounds__(256) void k_draw_pick(LongArgs a) {
    const int lane = threadIdx.x & 63;
    const int64_t d = (int64_t)flat_block() * 4 + (threadIdx.x >> 6);
    if (d >= a.d.in.rows * a.d.draws) return;
    const int64_t row = d / a.d.draws;
    const auto* s = static_cast<const typename Score<DT>::type*>(a.d.in.p) + row * a.d.in.ld;
    const RowCut r = a.rows[row];
    const double* parts = a.parts + 2 * row * a.segments;
    const double total = parts[2 * (a.segments - 1) + 1];
    if (!(r.best > -INFINITY)) {
        if (lane == 0) {
            a.d.ids[d] = -1;
            if (a.d.logp) a.d.logp[d] = -INFINITY;
        }
        return;
    }
    const double want = unit_number(a.d.u[d]) * total;
    int64_t lo = 0, hi = a.segments - 1;
    while (lo < hi) {
        const int64_t mid = (lo + hi) / 2;
        if (parts[2 * mid + 1] > want) hi = mid; else lo = mid + 1;
    }
    while (lo > 0 && !(parts[2 * lo + 1] > parts[2 * lo - 1])) --lo;  // (never a segment without weight)
    const int64_t block = row * a.segments + lo;
    const float own = (float)parts[2 * lo];
    const Weights weights(r.best, a.d.inv_t);
    double base = lo > 0 ? parts[2 * lo - 1] : 0.0;
    double v = a.tiles[block * SEG_TILES + lane] * weights.of(own);
    uint32_t before = 0;
    if (r.t) {
        const uint32_t e = a.tile_ties[block * SEG_TILES + lane];
        uint32_t es = e;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const uint32_t y = __shfl_up((int)es, o, 64);
            if (lane >= o) es += y;
        }
        before = a.seg_ties[block] + es - e;
        const double each = weights.of(key_score(r.t));
        if (before < r.ties && each >= a.d.min_p) v += each * (double)min(e, r.ties - before);
    }
    const double incl = base + wave_scan64(v, lane);
    const uint64_t past = __ballot(incl > want && v > 0.0), any = __ballot(v > 0.0);
    const int tile = past ? __ffsll((unsigned long long)past) - 1 : any ? 63 - __clzll(any) : 0;
    base = __shfl(incl - v, tile, 64);
    before = __shfl((int)before, tile, 64);
    const Kept kept = {r.t ? key_score(r.t) : -INFINITY, 0u, r.ties};
    int64_t id = -1;
    double weight = 0.0;
    draw_in_tile<DT, true>(s, lo * KGE_ROW_SEGMENT + (int64_t)tile * 256, a.d.in.n, kept, weights, a.d.min_p, before, base, want, lane, id, weight);
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
    else if (n <= 16384) k_draw_rows<DT, 16, 4, CUT><<<grid, 1024, 0, st>>>(a);
    else k_draw_rows<DT, 16, 8, CUT><<<grid, 1024, 0, st>>>(a);
}

// The pieces of the workspace of long rows; returns its size.
int64_t carve(LongArgs* a, char* base, int64_t rows, int64_t n, bool weight_cut) {
    const int64_t segments = pieces(n, KGE_ROW_SEGMENT), blocks = rows * segments;
    int64_t off = 0;
    auto take = [&](int64_t bytes) { const int64_t o = off; off += up256(bytes); return base ? base + o : nullptr; };
    char* parts = take(blocks * 16);
    char* tiles = take(blocks * SEG_TILES * 8);
    char* tile_ties = take(blocks * SEG_TILES * 4);
    char* seg_ties = take(blocks * 4);
    char* cuts = take(rows * (int64_t)sizeof(RowCut));
    char* bins = weight_cut ? take(rows * LEVELS * BINS * 16) : nullptr;
    if (a) {
        a->segments = (int)segments;
        a->parts = reinterpret_cast<double*>(parts);
        a->tiles = reinterpret_cast<double*>(tiles);
        a->tile_ties = reinterpret_cast<uint32_t*>(tile_ties);
        a->seg_ties = reinterpret_cast<uint32_t*>(seg_ties);
        a->rows = reinterpret_cast<RowCut*>(cuts);
        a->bins = reinterpret_cast<uint64_t*>(bins);
    }
    return off;
}

template <int DT>
void launch(const DrawArgs& d, void* workspace, hipStream_t st) {
    const bool weight_cut = d.top_k == 0 && d.top_p < 1.0;
    if (d.in.n <= KGE_ROW_RESIDENT) {
        if (d.top_k > 0) launch_rows<DT, CUT_LIST>(d, st);
        else if (weight_cut) launch_rows<DT, CUT_WEIGHT>(d, st);
        else launch_rows<DT, CUT_NONE>(d, st);
        return;
    }
    LongArgs a = {};
    a.d = d;
    carve(&a, static_cast<char*>(workspace), d.in.rows, d.in.n, weight_cut);
    a.cut = weight_cut || d.min_p > 0.0;
    a.bits = 62;
    while (((int64_t)1 << (62 - a.bits)) < d.in.n) --a.bits;
    const dim3 segs = flat_grid(d.in.rows * a.segments), rows = flat_grid(d.in.rows);
    k_draw_sums<DT, 0><<<segs, SEG_WAVES * 64, 0, st>>>(a);
    if (a.cut) {
        k_draw_begin<<<rows, 256, 0, st>>>(a);
        for (int level = 0; weight_cut && level < LEVELS; ++level) {
            k_draw_bins<DT><<<segs, SEG_WAVES * 64, 0, st>>>(a, level);
            k_draw_narrow<<<rows, 256, 0, st>>>(a, level);
        }
        k_draw_sums<DT, 1><<<segs, SEG_WAVES * 64, 0, st>>>(a);
    }
    k_draw_scan<<<rows, 1024, 0, st>>>(a);
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
        kge_launch_top(in, top_k, 1.f, nullptr, nullptr, lists, nullptr, ws + up256(in.rows * (int64_t)top_k * 8), st);
        k_draw_lists<<<flat_grid(in.rows), 256, 0, st>>>(a, lists);
        return;
    }
    if (in.dtype == KGE_F32) launch<KGE_F32>(a, workspace, st);
    else if (in.dtype == KGE_BF16) launch<KGE_BF16>(a, workspace, st);
    else launch<KGE_F16>(a, workspace, st);
}
