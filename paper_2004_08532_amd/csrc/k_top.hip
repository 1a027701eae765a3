// The best candidates of every row of scores, and its log-sum-exp (kge_top_scores).
//
// One workgroup holds a row, or a segment of a long one, in registers and finds the score that exactly its m best reach by
// halving the interval of keys.  The entries at or above it are sorted in LDS.  The lists of a row's segments are joined by
// the same selection over (key, position) entries, level by level, until one list is left.
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
__device__ __forceinline__ void write_list(const uint64_t* list, int m, int64_t* ids, float* scores) {
    for (int e = threadIdx.x; e < m; e += THREADS) {
        const uint64_t x = list[e];
        ids[e] = x ? entry_position(x) : -1;
        scores[e] = x ? key_score((uint32_t)(x >> 32)) : -INFINITY;
    }
}

__device__ __forceinline__ float lse_of(double best, double sum, double inv_t) {
    return sum > 0.0 ? (float)(best * inv_t + log(sum)) : -INFINITY;
}

template <int DT, int WAVES, int TPW>
__global__ __launch_bounds__(WAVES * 64) void k_top_rows(TopArgs a) {
    constexpr int CAP = WAVES * TPW * 256, LIST = CAP < KGE_TOP_MAX ? CAP : KGE_TOP_MAX;
    __shared__ uint64_t list[LIST];
    __shared__ uint32_t slots[2 * WAVES], ties[WAVES * TPW + 1], count;
    __shared__ double sums[WAVES];
    const int64_t block = flat_block();
    if (block >= a.in.rows * a.segments) return;
    const int64_t row = block / a.segments, seg = block - row * a.segments, first = seg * CAP;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const auto* s = static_cast<const typename Score<DT>::type*>(a.in.p) + row * a.in.ld;

    uint32_t key[TPW * 4];
    load_keys<DT, WAVES, TPW>(s, first, a.in.n, key);
    uint32_t best = 0;
#pragma unroll
    for (int q = 0; q < TPW * 4; ++q) best = max(best, key[q]);
    best = block_max_u32<WAVES>(best, slots);

    if (a.want_lse) {
        double z = 0.0;
        const float top = key_score(best);
#pragma unroll
        for (int q = 0; q < TPW * 4; ++q) z += key[q] ? weight64(key_score(key[q]), top, a.inv_t) : 0.0;
        z = block_sum64<WAVES>(z, sums);
        if (threadIdx.x == 0) {
            if (a.segments == 1) a.lse[row] = lse_of(top, best ? z : 0.0, a.inv_t);
            else { a.parts[2 * block] = best ? top : -INFINITY; a.parts[2 * block + 1] = best ? z : 0.0; }
        }
    }

    const int m = min(a.m, LIST), size = power_of_two(m);
    for (int e = threadIdx.x; e < size; e += WAVES * 64) list[e] = 0;
    if (threadIdx.x == 0) count = 0;
    int reach = 0, last = CAP;
    const uint32_t t = best ? select_threshold<WAVES, TPW * 4, uint32_t>(key, best, m, slots, reach) : 1;
    if (reach > m) {  // more than m reach it: equal scores, of which the first ones count
        int above = 0;
#pragma unroll
        for (int q = 0; q < TPW * 4; ++q) above += __popcll(__ballot(key[q] > t));
        __syncthreads();
        if (lane == 0) slots[wave] = above;
        __syncthreads();
        above = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) above += slots[w];
        last = nth_equal<WAVES, TPW>(key, t, m - above, ties);
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < TPW * 4; ++q) {
        const int at = ((q / 4) * WAVES + wave) * 256 + lane * 4 + q % 4;
        append_entry(key[q] > t || (key[q] == t && at <= last), order_entry(key[q], first + at), list, &count);
    }
    sort_descending<WAVES * 64>(list, size);
    if (a.segments == 1) {
        write_list<WAVES * 64>(list, m, a.ids + row * a.m, a.scores + row * a.m);
        for (int e = m + threadIdx.x; e < a.m; e += WAVES * 64) { a.ids[row * a.m + e] = -1; a.scores[row * a.m + e] = -INFINITY; }
    } else {
        for (int e = threadIdx.x; e < a.m; e += WAVES * 64) a.lists[block * a.m + e] = e < m ? list[e] : 0;
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
    constexpr int CAP = WAVES * TPW * 256;
    __shared__ uint64_t list[KGE_TOP_MAX], bests[WAVES];
    __shared__ uint32_t slots[2 * WAVES], count;
    __shared__ double sums[WAVES];
    const int64_t block = flat_block();
    if (block >= a.rows * a.groups) return;
    const int64_t row = block / a.groups, first = (block - row * a.groups) * CAP;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint64_t* in = a.in + row * a.entries;
    const int n = (int)min((int64_t)CAP, a.entries - first);

    uint64_t key[TPW * 4], best = 0;
#pragma unroll
    for (int q = 0; q < TPW * 4; ++q) {
        const int at = (q * WAVES + wave) * 64 + lane;
        key[q] = at < n ? in[first + at] : 0;
        best = key[q] > best ? key[q] : best;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        const uint64_t v = __shfl_xor((unsigned long long)best, o, 64);
        best = v > best ? v : best;
    }
    if (lane == 0) bests[wave] = best;
    const int size = power_of_two(a.m);
    for (int e = threadIdx.x; e < size; e += WAVES * 64) list[e] = 0;
    if (threadIdx.x == 0) count = 0;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) best = bests[w] > best ? bests[w] : best;

    int reach = 0;
    const uint64_t t = best ? select_threshold<WAVES, TPW * 4, uint64_t>(key, best, a.m, slots, reach) : 1;
    __syncthreads();
#pragma unroll
    for (int q = 0; q < TPW * 4; ++q) append_entry(key[q] >= t, key[q], list, &count);
    sort_descending<WAVES * 64>(list, size);
    if (a.groups > 1) {
        for (int e = threadIdx.x; e < a.m; e += WAVES * 64) a.out[block * a.m + e] = list[e];
        return;
    }
    if (a.ids) write_list<WAVES * 64>(list, a.m, a.ids + row * a.m, a.scores + row * a.m);
    else for (int e = threadIdx.x; e < a.m; e += WAVES * 64) a.out[row * a.m + e] = list[e];
    if (a.parts) {
        const double* p = a.parts + 2 * row * a.segments;
        const float top = key_score((uint32_t)(list[0] >> 32));
        double z = 0.0;
        for (int g = threadIdx.x; g < a.segments; g += WAVES * 64)
            if (p[2 * g + 1] > 0.0) z += p[2 * g + 1] * weight64((float)p[2 * g], top, a.inv_t);
        z = block_sum64<WAVES>(z, sums);
        if (threadIdx.x == 0) a.lse[row] = lse_of(top, list[0] ? z : 0.0, a.inv_t);
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
