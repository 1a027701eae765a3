// The best candidates of every row of scores, and its log-sum-exp (kge_top_scores).
//
// One workgroup holds a row, or a segment of a long one, in registers, collects the few candidates that its best m are among and
// puts them in order in LDS (collect_best, order_list).  Of a row in segments every workgroup leaves its candidates, at least
// its best m; they are collected and ordered in the same way, level by level, until one list is left.
// log-sum-exp: the weights exp((s - best) / T) of a segment are summed in 64 bits beside it.
#include "k_rows.h"

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
__global__ __launch_bounds__(WAVES * 64) void k_top_rows(TopArgs a) {
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
#pragma unroll
            for (int q = 0; q < TPW * 4; ++q) z += w.of(v[q]);
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

template <int DT>
void launch_rows(const TopArgs& a, hipStream_t st) {
    const int64_t n = a.in.n, blocks = a.in.rows * a.segments;
    if (a.segments > 1) k_top_rows<DT, 16, 4><<<flat_grid(blocks), 1024, 0, st>>>(a);
    else if (n <= 256) k_top_rows<DT, 1, 1><<<flat_grid(blocks), 64, 0, st>>>(a);
    else if (n <= 1024) k_top_rows<DT, 4, 1><<<flat_grid(blocks), 256, 0, st>>>(a);
    else if (n <= 4096) k_top_rows<DT, 4, 4><<<flat_grid(blocks), 256, 0, st>>>(a);
    else if (n <= 16384) k_top_rows<DT, 16, 4><<<flat_grid(blocks), 1024, 0, st>>>(a);
    else k_top_rows<DT, 16, 8><<<flat_grid(blocks), 1024, 0, st>>>(a);
}

}  // namespace

int64_t kge_top_workspace(int64_t rows, int64_t n, int m) {
    if (n <= KGE_ROW_RESIDENT) return 0;
    const int64_t segments = pieces(n, KGE_ROW_SEGMENT), second = pieces(segments * m, KGE_ROW_SEGMENT);
    return up256(rows * segments * m * 8) + up256(rows * second * m * 8) + up256(rows * segments * 16);
}

void kge_launch_top(const RowScores& in, int m, float temperature, int64_t* ids, float* scores, uint64_t* entries, float* lse,
                    void* workspace, hipStream_t st) {
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
