// The best candidates of every row of scores, and its log-sum-exp (kge_top_scores).
//
// One workgroup holds a row, or a segment of a long one, in registers, collects the few candidates that its best m are among and
// puts them in order in LDS (collect_best, order_list).  Of a row in segments every workgroup leaves its candidates, at least
// its best m; they are collected and ordered in the same way, level by level, until one list is left.  Long rows of short lists: k_tiles has the best
// score of every tile, and one workgroup per row reads again the few tiles that can hold one of the best m.
// log-sum-exp: the weights exp((s - best) / T) of a segment are summed in 64 bits beside it.
//
// Best 64 and log-sum-exp of 1024 rows of 14,951 fp32: 34 us (a large copy reads them in 12): 11.4 M wave instructions, 23 us of the vector units, half
// of them the weights.  Best 100 of 16 rows of 2.5 M bf16: k_tiles 15 us (5.3 TB/s), k_top_finish 16, a chain of steps in 16 workgroups.  Best 10
// of 256 rows of 64: 4.3 us in the kernel, 6.2 per call on the host.
#include "k_draw_list.h"

namespace {

struct TopArgs {
    RowScores in;
    int m, segments;
    double inv_t;
    int want_lse;
    uint64_t* lists;      // [rows][segments][m], rows in several segments
    double* parts;        // [rows][segments][2]: best score, sum of weights relative to it
    int64_t* ids;
    float* scores;
    float* lse;
};

template <int THREADS>
__device__ __forceinline__ void write_list(const uint64_t* list, int count, int m, int64_t* ids, float* scores) {
    for (int e = threadIdx.x; e < m; e += THREADS) {
        const uint64_t x = e < count ? list[e] : 0;
        ids[e] = x ? entry_position(x) : -1;
        scores[e] = x ? key_score((uint32_t)(x >> 32)) : -INFINITY;
    }
}

__device__ __forceinline__ float lse_of(double best, double sum, double inv_t) {
    return sum > 0.0 ? (float)(best * inv_t + log(sum)) : -INFINITY;
}

template <int DT, int WAVES, int TPW>
__global__ __launch_bounds__(WAVES * 64, WAVES == 8 ? 8 : 1) void k_top_rows(TopArgs a) {
    constexpr int CAP = WAVES * TPW * 256, THREADS = WAVES * 64;
    __shared__ BestList<WAVES, TPW> s;
    __shared__ double sums[WAVES];
    __shared__ float maxima[WAVES];
    const int64_t block = flat_block();
    if (block >= a.in.rows * a.segments) return;
    const int64_t row = block / a.segments, seg = block - row * a.segments, first = seg * CAP;
    const auto* scores = static_cast<const typename Score<DT>::type*>(a.in.p) + row * a.in.ld;

    float v[TPW * 4];
    const float mine = load_tiles<DT, WAVES, TPW>(scores, first, a.in.n, v), best = block_max<WAVES>(mine, maxima);
    const bool empty = !(best > -INFINITY);
    if (a.want_lse) {
        double z = 0.0;
        if (!empty) {
            const Scale scale(a.inv_t);
            const Weights w(best, scale);
            if (best == INFINITY) {
                z = 1.0;
            } else {
#pragma unroll
                for (int q = 0; q < TPW * 4; ++q) {
                    z += w.loose(v[q], v[q] >= w.floor);
                    if (q % 8 == 7) __builtin_amdgcn_sched_barrier(0);
                }
            }
            z = block_sum64<WAVES>(z, sums);
        }
        if (threadIdx.x == 0) {
            if (a.segments == 1) a.lse[row] = lse_of(best, z, a.inv_t);
            else { a.parts[2 * block] = best; a.parts[2 * block + 1] = z; }
        }
    }
    const int count = empty ? 0 :
        collect_best<WAVES, TPW>(v, [&](int q) { return ~(uint32_t)(first + tile_position<WAVES>(q)); }, mine, order_key(best), a.m, s);
    const uint64_t* list = s.list;
    // the candidates of a segment: in order only where they are more than its share of the lists
    if (a.segments == 1 || count > a.m) list = order_list<THREADS>(s.list, s.sorted, s.rank, count);
    if (a.segments == 1) {
        write_list<THREADS>(list, count, a.m, a.ids + row * a.m, a.scores + row * a.m);
    } else {
        for (int e = threadIdx.x; e < a.m; e += THREADS) a.lists[block * a.m + e] = e < count ? list[e] : 0;
    }
}

struct MergeArgs {
    const uint64_t* in;   // [rows][entries]
    int64_t rows, entries;
    int m, groups;        // groups of KGE_ROW_SEGMENT entries per row
    uint64_t* out;        // [rows][groups][m], several groups
    int64_t* ids;
    float* scores;
    const double* parts;  // [rows][segments][2], null: no log-sum-exp
    int segments;
    double inv_t;
    float* lse;
};

// Lists of a row -> one list of its group.
template <int WAVES, int TPW>
__global__ __launch_bounds__(WAVES * 64) void k_top_merge(MergeArgs a) {
    constexpr int CAP = WAVES * TPW * 256, N = TPW * 4, THREADS = WAVES * 64;
    __shared__ BestList<WAVES, TPW> s;
    __shared__ double sums[WAVES];
    __shared__ float maxima[WAVES];
    const int64_t block = flat_block();
    if (block >= a.rows * a.groups) return;
    const int64_t row = block / a.groups, first = (block - row * a.groups) * CAP;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const uint64_t* in = a.in + row * a.entries;
    const int n = (int)min((int64_t)CAP, a.entries - first);

    float v[N], mine = -INFINITY;
    uint32_t low[N];  // inverted positions
#pragma unroll
    for (int q = 0; q < N; ++q) {
        const int at = (q * WAVES + wave) * 64 + lane;
        const uint64_t x = at < n ? in[first + at] : 0;
        v[q] = x ? key_score((uint32_t)(x >> 32)) : -INFINITY;
        low[q] = (uint32_t)x;
        mine = fmaxf(mine, v[q]);
    }
    const float best = block_max<WAVES>(mine, maxima);
    const int count = best > -INFINITY ? collect_best<WAVES, TPW>(v, [&](int q) { return low[q]; }, mine, order_key(best), a.m, s) : 0;
    const uint64_t* list = order_list<THREADS>(s.list, s.sorted, s.rank, count);
    if (a.groups > 1 || !a.ids) {
        for (int e = threadIdx.x; e < a.m; e += THREADS) a.out[block * a.m + e] = e < count ? list[e] : 0;
        return;
    }
    write_list<THREADS>(list, count, a.m, a.ids + row * a.m, a.scores + row * a.m);
    if (a.parts) {
        const double* p = a.parts + 2 * row * a.segments;
        const Scale scale(a.inv_t);
        const Weights w(best, scale);
        double z = 0.0;
        for (int g = threadIdx.x; g < a.segments; g += THREADS)
            if (p[2 * g + 1] > 0.0) z += p[2 * g + 1] * w.of((float)p[2 * g]);
        z = block_sum64<WAVES>(z, sums);
        if (threadIdx.x == 0) a.lse[row] = lse_of(best, z, a.inv_t);
    }
}

// ---------------------------------------------------------------------------------------------------------
// Long rows of which every tile's best score is known (k_tiles): a score that m groups of tiles reach with their best bounds the list, so that
// only the few tiles which reach it are read again, by one workgroup per row.  (100 best of 2.5 M: about 103 tiles of 9766.)
// ---------------------------------------------------------------------------------------------------------
struct FinishArgs {
    RowScores in;
    int m;
    int64_t tiles;            // of a row, and the distance of two rows' in tile_best
    int64_t pitch;
    const float* tile_best;
    const float* group_best;  // log-sum-exp: groups of pitch / GROUP_TILES
    const double* group_sum;
    double inv_t;
    int64_t* ids;
    float* scores;
    float* lse;               // null: none
};

template <int DT, int PER, bool DRAW>  // PER: groups of tiles per thread, m <= PER * 512
__global__ __launch_bounds__(1024) void k_top_finish(FinishArgs a, DrawArgs draw) {
    constexpr int THREADS = 1024, WAVES = 16, ROOM = BEST_ROOM, TILE_ROOM = 4096;
    __shared__ uint64_t list[ROOM], sorted[256], masks[WAVES];
    __shared__ float most[PER * THREADS], maxima[WAVES];
    __shared__ uint32_t tile_list[TILE_ROOM], rank[256], slots[2 * WAVES], count, n_tiles, shared_bound;
    __shared__ double sums[DRAW ? KGE_TOP_MAX : WAVES];
    __shared__ int kept_entries;
    const int64_t row = flat_block();
    if (row >= a.in.rows) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const auto* s = static_cast<const typename Score<DT>::type*>(a.in.p) + row * a.in.ld;
    const float* bests = a.tile_best + row * a.pitch;

    float mine[PER], best = -INFINITY;
#pragma unroll
    for (int g = 0; g < PER; ++g) mine[g] = -INFINITY;
    constexpr int READS = 8;  // of a thread at once
    for (int64_t t0 = threadIdx.x; t0 < a.tiles; t0 += READS * THREADS) {
        float x[READS];
#pragma unroll
        for (int k = 0; k < READS; ++k) x[k] = bests[min(t0 + k * THREADS, a.tiles - 1)];
#pragma unroll
        for (int k = 0; k < READS; ++k) mine[k % PER] = fmaxf(mine[k % PER], t0 + k * THREADS < a.tiles ? x[k] : -INFINITY);
    }
#pragma unroll
    for (int g = 0; g < PER; ++g) {
        most[g * THREADS + threadIdx.x] = mine[g];
        best = fmaxf(best, mine[g]);
    }
    if (threadIdx.x == 0) { count = 0; n_tiles = 0; }
    best = block_max<WAVES>(best, maxima);
    if (!(best > -INFINITY)) {
        if constexpr (DRAW) write_empty<THREADS>(draw, row);
        else write_list<THREADS>(list, 0, a.m, a.ids + row * a.m, a.scores + row * a.m);
        if (!DRAW && a.lse && threadIdx.x == 0) a.lse[row] = -INFINITY;
        return;
    }
    if (wave == 0) {
        float x[PER * WAVES];
#pragma unroll
        for (int w = 0; w < PER * WAVES; ++w) x[w] = most[w * 64 + lane];
        const uint32_t b = wave_bound<PER * WAVES>(x, order_key(best), a.m);
        if (lane == 0) shared_bound = b;
    }
    __syncthreads();
    float t = key_score(shared_bound);
    for (int64_t i0 = threadIdx.x; i0 < a.tiles; i0 += READS * THREADS) {
        float x[READS];
#pragma unroll
        for (int k = 0; k < READS; ++k) x[k] = bests[min(i0 + k * THREADS, a.tiles - 1)];
#pragma unroll
        for (int k = 0; k < READS; ++k) {
            const int64_t i = i0 + k * THREADS;
            if (i < a.tiles && x[k] >= t) {  // (few)
                const uint32_t at = atomicAdd(&n_tiles, 1u);
                if (at < TILE_ROOM) tile_list[at] = (uint32_t)i;
            }
        }
    }
    __syncthreads();
    const uint32_t found = n_tiles;
    if (found <= TILE_ROOM) {
        constexpr int AT_ONCE = 4;
        for (uint32_t e0 = wave * AT_ONCE; e0 < found; e0 += WAVES * AT_ONCE) {
            Quad<DT> x[AT_ONCE];
            int64_t first[AT_ONCE];
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) {
                first[k] = (int64_t)tile_list[min(e0 + k, found - 1)] * 256;
                x[k].load(s, first[k] + lane * 4, a.in.n);
            }
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) {
                if (e0 + k >= found) break;
                float v[4];
                x[k].values(first[k], a.in.n, v);
                uint32_t marked = 0;
#pragma unroll
                for (int q = 0; q < 4; ++q) marked |= (uint32_t)(v[q] >= t) << q;
                append_marked<4>(v, marked, [&](int q) { return ~(uint32_t)(first[k] + lane * 4 + q); }, list, ROOM, &count);
            }
        }
        __syncthreads();
    }
    int have = (int)count;
    if (found > TILE_ROOM || have > ROOM) {
        // Too many scores reach the bound (many equal ones): the tiles in their order, four at a time, into a list that is cut to its best m where it
        // gets full; from then on only what is above its last entry can enter, since equal scores count by position.
        bool above = false;
        have = 0;
        for (int64_t i0 = 0; i0 < a.tiles; i0 += THREADS) {
            const int64_t i = i0 + threadIdx.x;
            const float b = i < a.tiles ? bests[i] : -INFINITY;
            const uint64_t who = __ballot(above ? b > t : b >= t);
            __syncthreads();
            if (lane == 0) masks[wave] = who;
            __syncthreads();
            for (int w = 0; w < WAVES; ++w) {
                uint64_t left = masks[w];
                while (left) {
                    int64_t tile = -1;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        if (!left) break;
                        const int b2 = __ffsll((unsigned long long)left) - 1;
                        left &= left - 1;
                        if (wave / 4 == k) tile = i0 + w * 64 + b2;
                    }
                    const int64_t j = tile * 256 + (threadIdx.x & 255);
                    float v = tile >= 0 && j < a.in.n ? widen<DT>(s[j]) : -INFINITY;
                    v = fmaxf(v, -INFINITY);
                    bool in = above ? v > t : v >= t;
                    if (threadIdx.x == 0) count = have;
                    int c = block_count<WAVES>(__popcll(__ballot(in)), slots);
                    if (have + c > ROOM) {
                        __syncthreads();
                        uint64_t* sl = order_list<THREADS>(list, sorted, rank, have);
                        t = key_score((uint32_t)(sl[a.m - 1] >> 32));
                        above = true;
                        have = a.m;
                        in = v > t;
                        if (threadIdx.x == 0) count = have;
                        c = block_count<WAVES>(__popcll(__ballot(in)), slots + WAVES);
                    }
                    append_marked<1>(&v, in, [&](int) { return ~(uint32_t)j; }, list, ROOM, &count);
                    have += c;
                    __syncthreads();
                }
            }
        }
    }
    uint64_t* in_order = order_list<THREADS>(list, sorted, rank, have);
    if constexpr (DRAW) {
        draw_from_list<THREADS>(draw, row, in_order, in_order == sorted ? list : sorted, rank, min(have, a.m), sums, &kept_entries);
    } else {
        write_list<THREADS>(in_order, have, a.m, a.ids + row * a.m, a.scores + row * a.m);
        if (a.lse) {
            const int64_t groups = a.pitch / GROUP_TILES;
            const Scale scale(a.inv_t);
            const Weights w(best, scale);
            double z = 0.0;
            for (int64_t g = threadIdx.x; g < groups; g += THREADS) {
                const float b = a.group_best[row * groups + g];
                if (b > -INFINITY) z += a.group_sum[row * groups + g] * w.of(b);
            }
            z = block_sum64<WAVES>(z, sums);
            if (threadIdx.x == 0) a.lse[row] = lse_of(best, z, a.inv_t);
        }
    }
}

template <int DT>
void launch_finish(const FinishArgs& f, const DrawArgs* draw, hipStream_t st) {
    const dim3 grid = flat_grid(f.in.rows);
    if (draw) {
        if (f.m <= 512) k_top_finish<DT, 1, true><<<grid, 1024, 0, st>>>(f, *draw);
        else k_top_finish<DT, 2, true><<<grid, 1024, 0, st>>>(f, *draw);
    } else {
        if (f.m <= 512) k_top_finish<DT, 1, false><<<grid, 1024, 0, st>>>(f, DrawArgs());
        else k_top_finish<DT, 2, false><<<grid, 1024, 0, st>>>(f, DrawArgs());
    }
}

template <int DT>
void launch_rows(const TopArgs& a, hipStream_t st) {
    const int64_t n = a.in.n, blocks = a.in.rows * a.segments;
    if (a.segments > 1) k_top_rows<DT, 16, 4><<<flat_grid(blocks), 1024, 0, st>>>(a);
    else if (n <= 256) k_top_rows<DT, 1, 1><<<flat_grid(blocks), 64, 0, st>>>(a);
    else if (n <= 1024) k_top_rows<DT, 4, 1><<<flat_grid(blocks), 256, 0, st>>>(a);
    else if (n <= 4096) k_top_rows<DT, 4, 4><<<flat_grid(blocks), 256, 0, st>>>(a);
    // us, best 64 of 5000, by the kernels for 16,384 -> by this: 16 / 1024 / 4096 rows 9.0 -> 7.8 / 18.9 -> 11.8 / 63 -> 38.5
    else if (n <= 8192) k_top_rows<DT, 8, 4><<<flat_grid(blocks), 512, 0, st>>>(a);
    // 16,384 scores in 1024 threads, or in 512 where a CU would get more than one row.  us, best 64, 1024 -> 512 threads: 256 rows of 5000 / 15,000
    // 9.4 -> 11.1 / 9.5 -> 11.1, 512 rows 17.0 -> 14.5 / 17.1 -> 17.0, 4096 rows 122 -> 63 / 125 -> 82
    else if (n <= 16384 && blocks > 256) k_top_rows<DT, 8, 8><<<flat_grid(blocks), 512, 0, st>>>(a);
    else if (n <= 16384) k_top_rows<DT, 16, 4><<<flat_grid(blocks), 1024, 0, st>>>(a);
    else k_top_rows<DT, 16, 8><<<flat_grid(blocks), 1024, 0, st>>>(a);
}

}  // namespace

// The best tiles bound the scores from below only where there are more than enough of them.  us, segment by segment -> by tiles, at m = n / 512: n = 40,943,
// 4 / 256 rows 17.3 -> 14.6 / 35 -> 22; n = 300,000 54 -> 51 / 503 -> 112; at m = n / 2000: 16.9 -> 11.5 / 32.6 -> 17.3 and 22 -> 20 / 206 -> 73.  At m = n / 300 the
// candidates do not fit the list: 21 -> 73 / 41 -> 85.
bool kge_top_by_tiles(int64_t n, int m) { return n > KGE_ROW_RESIDENT && n >= 512ll * m; }

int64_t kge_top_workspace(int64_t rows, int64_t n, int m) {
    if (n <= KGE_ROW_RESIDENT) return 0;
    if (kge_top_by_tiles(n, m)) {
        const int64_t groups = rows * pieces(n, GROUP);
        return up256(groups * GROUP_TILES * 4) + up256(groups * 4) + up256(groups * 8);
    }
    const int64_t segments = pieces(n, KGE_ROW_SEGMENT), second = pieces(segments * m, KGE_ROW_SEGMENT);
    return up256(rows * segments * m * 8) + up256(rows * second * m * 8) + up256(rows * segments * 16);
}

void kge_launch_top(const RowScores& in, int m, float temperature, int64_t* ids, float* scores, uint64_t* entries, float* lse,
                    const DrawArgs* draw, void* workspace, hipStream_t st) {
    if (kge_top_by_tiles(in.n, m)) {
        TileArgs t = {};
        t.in = in; t.inv_t = 1.0 / (double)temperature; t.groups = pieces(in.n, GROUP);
        char* ws = static_cast<char*>(workspace);
        t.tile_best = reinterpret_cast<float*>(ws);
        ws += up256(in.rows * t.groups * GROUP_TILES * 4);
        t.group_best = reinterpret_cast<float*>(ws);
        t.group_sum = reinterpret_cast<double*>(ws + up256(in.rows * t.groups * 4));
        kge_launch_tiles(t, lse ? TILES_BEST_SUMS : TILES_BEST, st);
        FinishArgs f = {};
        f.in = in; f.m = m; f.tiles = pieces(in.n, 256); f.pitch = t.groups * GROUP_TILES;
        f.tile_best = t.tile_best; f.group_best = t.group_best; f.group_sum = t.group_sum;
        f.inv_t = t.inv_t; f.ids = ids; f.scores = scores; f.lse = lse;
        if (in.dtype == KGE_F32) launch_finish<KGE_F32>(f, draw, st);
        else if (in.dtype == KGE_BF16) launch_finish<KGE_BF16>(f, draw, st);
        else launch_finish<KGE_F16>(f, draw, st);
        return;
    }
    TopArgs a = {};
    a.in = in; a.m = m; a.inv_t = 1.0 / (double)temperature; a.want_lse = lse != nullptr;
    a.ids = ids; a.scores = scores; a.lse = lse;
    a.segments = in.n <= KGE_ROW_RESIDENT ? 1 : (int)pieces(in.n, KGE_ROW_SEGMENT);
    char* ws = static_cast<char*>(workspace);
    uint64_t* lists[2] = {};
    if (a.segments > 1) {
        lists[0] = reinterpret_cast<uint64_t*>(ws);
        ws += up256(in.rows * a.segments * m * 8);
        lists[1] = reinterpret_cast<uint64_t*>(ws);
        ws += up256(in.rows * pieces((int64_t)a.segments * m, KGE_ROW_SEGMENT) * m * 8);
        a.lists = lists[0];
        a.parts = reinterpret_cast<double*>(ws);
    }
    if (in.dtype == KGE_F32) launch_rows<KGE_F32>(a, st);
    else if (in.dtype == KGE_BF16) launch_rows<KGE_BF16>(a, st);
    else launch_rows<KGE_F16>(a, st);
    if (a.segments == 1) return;
    int64_t per_row = a.segments;
    for (int level = 0;; ++level) {
        MergeArgs g = {};
        g.in = lists[level & 1]; g.rows = in.rows; g.entries = per_row * m; g.m = m;
        g.groups = (int)pieces(g.entries, KGE_ROW_SEGMENT);
        const bool final = g.groups == 1;
        g.out = final ? entries : lists[(level + 1) & 1];
        if (final) {
            g.ids = ids; g.scores = scores; g.lse = lse;
            g.parts = lse ? a.parts : nullptr;
            g.segments = a.segments; g.inv_t = a.inv_t;
        }
        k_top_merge<16, 4><<<flat_grid(in.rows * g.groups), 1024, 0, st>>>(g);
        if (final) return;
        per_row = g.groups;
    }
}
