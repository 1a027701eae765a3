// Rows of scores as distributions over candidates: what k_top.hip, k_draw.hip and k_distill.hip share.
//
// A row is cut into tiles of 256 consecutive scores, 4 per lane of a wave.  A workgroup of WAVES waves holds up to TPW tiles per
// wave in registers (tile t belongs to wave t % WAVES), so a row of up to WAVES * TPW * 256 scores is read once whatever is
// done with it; longer rows are cut into segments of that size, a workgroup each.
//
// Order of candidates: higher score first, equal scores by their position.  -inf and NaN are masked: no candidate.  A score
// becomes an unsigned key of the same order (0: masked; -0 counts as +0), and key and position together a 64-bit number
// that is unique in its row.
#pragma once
#include "kge_common.h"

constexpr int KGE_TOP_MAX = 1024;           // longest list of best candidates
constexpr int KGE_ROW_SEGMENT = 16384;      // scores per workgroup of a row that is cut (16 waves of 4 tiles)
constexpr int KGE_ROW_RESIDENT = 32768;     // longest row that one workgroup holds (16 waves of 8 tiles)

struct RowScores {
    const void* p;
    int dtype;  // kge_dtype
    int64_t rows, n, ld;
};

inline int64_t pieces(int64_t n, int64_t of) { return (n + of - 1) / of; }
inline int64_t up256(int64_t x) { return (x + 255) & ~(int64_t)255; }

int64_t kge_top_workspace(int64_t rows, int64_t n, int m);
// (ids and scores, or the sorted entries alone; lse may be null)
void kge_launch_top(const RowScores& in, int m, float temperature, int64_t* ids, float* scores, uint64_t* entries, float* lse,
                    void* workspace, hipStream_t st);
int64_t kge_draw_workspace(int64_t rows, int64_t n, int top_k, float top_p);
void kge_launch_draw(const RowScores& in, const double* u, int draws, float temperature, int top_k, float top_p, float min_p, int64_t* ids,
                     float* logp, void* workspace, hipStream_t st);
// A teacher's lists of m candidates per row.  step != null: the scores are those of a training step in its workspace, rows of up to
// KGE_ROW_RESIDENT, and become its coefficients W in place
struct TeacherLists {
    const int64_t* ids;
    const float* scores;
    const float* lse;  // null: the lists are all there is
    int m;
    float temperature;
};
struct StepRows {
    kge_ctx* c;
    float gamma;
    int is_dist, bf16;  // S holds distances, score = gamma - S; W is rounded to bf16
    float* cpos;        // [b] zeroed: the positives' own scores have no part in this loss
};
int64_t kge_distill_workspace(int64_t rows, int64_t n);
void kge_launch_distill(const RowScores& in, const TeacherLists& t, float grad_scale, float loss_scale, float* loss, void* grad, int64_t ld_grad,
                        const StepRows* step, void* workspace, hipStream_t st);

#ifdef __HIPCC__
namespace {

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned short u16x4u __attribute__((ext_vector_type(4), aligned(2)));

template <int DT> struct Score { using type = unsigned short; };
template <> struct Score<KGE_F32> { using type = float; };

template <int DT> __device__ __forceinline__ float widen(typename Score<DT>::type v) {
    if constexpr (DT == KGE_F32) return v;
    else if constexpr (DT == KGE_BF16) return __uint_as_float((uint32_t)v << 16);
    else return (float)__builtin_bit_cast(_Float16, v);
}
template <int DT> __device__ __forceinline__ typename Score<DT>::type narrow(float v) {  // to nearest, ties to even
    if constexpr (DT == KGE_F32) return v;
    else if constexpr (DT == KGE_BF16) return __builtin_bit_cast(unsigned short, (__bf16)v);
    else return __builtin_bit_cast(unsigned short, (_Float16)v);
}

// Scores j .. j + 3 of a row of n, -inf behind its end.  (Rows start at any multiple of a score's size.)
template <int DT> __device__ __forceinline__ void load4(const typename Score<DT>::type* row, int64_t j, int64_t n, float v[4]) {
    if (j + 4 <= n) {
        if constexpr (DT == KGE_F32) {
            const f32x4u x = *reinterpret_cast<const f32x4u*>(row + j);
            v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
        } else {
            const u16x4u x = *reinterpret_cast<const u16x4u*>(row + j);
            v[0] = widen<DT>(x.x); v[1] = widen<DT>(x.y); v[2] = widen<DT>(x.z); v[3] = widen<DT>(x.w);
        }
    } else {
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = j + q < n ? widen<DT>(row[j + q]) : -INFINITY;
    }
}

__device__ __forceinline__ uint32_t order_key(float s) {
    const uint32_t u = __float_as_uint(s + 0.f);  // -0 -> +0
    const uint32_t k = u >> 31 ? ~u : u | 0x80000000u;
    return s > -INFINITY ? k : 0u;  // (false for NaN)
}
__device__ __forceinline__ float key_score(uint32_t k) {  // of a key that is not 0
    return __uint_as_float(k >> 31 ? k & 0x7FFFFFFFu : ~k);
}
__device__ __forceinline__ uint64_t order_entry(uint32_t key, int64_t j) { return key ? (uint64_t)key << 32 | (uint32_t)~(uint32_t)j : 0; }
__device__ __forceinline__ int64_t entry_position(uint64_t e) { return (int64_t)(uint32_t)~(uint32_t)e; }

// exp((s - best) / T) of a score that is not masked.  In 64 bits: which candidate a random number falls on is decided by sums
// of these, and the sums of 32-bit weights would move thousands of borders by more than the numbers' spacing.
__device__ __forceinline__ double weight64(float s, float best, double inv_t) {
    return s == best ? 1.0 : exp(((double)s - (double)best) * inv_t);
}

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}
__device__ __forceinline__ double wave_scan64(double v, int lane) {  // sum over lanes 0 .. lane
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const double w = __shfl_up(v, o, 64);
        if (lane >= o) v += w;
    }
    return v;
}
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o, 64));
    return v;
}

// Reductions over a workgroup of WAVES waves; `slot` is LDS of WAVES values that is free again after the next barrier.
template <int WAVES> __device__ __forceinline__ double block_sum64(double v, double* slot) {
    v = wave_sum64(v);
    if constexpr (WAVES == 1) return v;
    if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = v;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) s += slot[w];
    __syncthreads();
    return s;
}
template <int WAVES> __device__ __forceinline__ uint32_t block_max_u32(uint32_t v, uint32_t* slot) {
    v = wave_max_u32(v);
    if constexpr (WAVES == 1) return v;
    if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = v;
    __syncthreads();
    uint32_t m = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) m = max(m, slot[w]);
    __syncthreads();
    return m;
}

// The tiles of a workgroup in registers, as keys.
template <int DT, int WAVES, int TPW>
__device__ __forceinline__ void load_keys(const typename Score<DT>::type* row, int64_t first, int64_t n, uint32_t key[TPW * 4]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int i = 0; i < TPW; ++i) {
        float v[4];
        load4<DT>(row, first + (int64_t)(i * WAVES + wave) * 256 + lane * 4, n, v);
#pragma unroll
        for (int q = 0; q < 4; ++q) key[4 * i + q] = order_key(v[q]);
    }
}

// Largest threshold that at least m of the workgroup's keys reach, by halving the interval of keys: every round counts the keys
// at or above its middle.  Ends early where exactly m do.  `reach`: how many reach the result.  Fewer than m candidates: 1.
template <int WAVES, int N, typename K>
__device__ __forceinline__ K select_threshold(const K key[N], K best, int m, uint32_t* slots /* [2 * WAVES] */, int& reach) {
    K lo = 1, hi = best;  // count(>= lo) >= m, count(> hi) < m
    int round = 0;
    auto count = [&](K t) {
        int c = 0;
#pragma unroll
        for (int q = 0; q < N; ++q) c += __popcll(__ballot(key[q] >= t));
        if constexpr (WAVES == 1) return c;
        uint32_t* s = slots + (round++ & 1) * WAVES;
        if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = c;
        __syncthreads();
        c = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) c += s[w];
        return c;
    };
    reach = count(lo);
    if (reach <= m) return lo;
    while (lo < hi) {
        const K mid = lo + (hi - lo) / 2 + ((hi - lo) & 1);  // lo < mid <= hi
        const int c = count(mid);
        if (c >= m) {
            lo = mid;
            reach = c;
            if (c == m) break;
        } else {
            hi = mid - 1;
        }
    }
    return lo;
}

// Position (within the workgroup's tiles) of the c-th key that equals t, c >= 1 and at most their number.
template <int WAVES, int TPW>
__device__ __forceinline__ int nth_equal(const uint32_t key[TPW * 4], uint32_t t, int c, uint32_t* tile_count /* [WAVES * TPW + 1] */) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint64_t below = ((uint64_t)1 << lane) - 1;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < TPW; ++i) {
        int s = 0;
#pragma unroll
        for (int q = 0; q < 4; ++q) s += __popcll(__ballot(key[4 * i + q] == t));
        if (lane == 0) tile_count[i * WAVES + wave] = s;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < TPW; ++i) {
        const int tile = i * WAVES + wave;
        int before = 0;
        for (int u = 0; u < tile; ++u) before += tile_count[u];
        if (before >= c || before + (int)tile_count[tile] < c) continue;
        int at = before;
        uint64_t eq[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            eq[q] = __ballot(key[4 * i + q] == t);
            at += __popcll(eq[q] & below);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (eq[q] >> lane & 1) {
                if (++at == c) tile_count[WAVES * TPW] = tile * 256 + lane * 4 + q;
            }
        }
    }
    __syncthreads();
    return (int)tile_count[WAVES * TPW];
}

// Appends the entries that `take` says to a list in LDS (in any order); *n starts at 0 and ends at their number.
__device__ __forceinline__ void append_entry(bool take, uint64_t entry, uint64_t* list, uint32_t* n) {
    const int lane = threadIdx.x & 63;
    const uint64_t who = __ballot(take);
    if (!who) return;
    uint32_t base = 0;
    if (lane == 0) base = atomicAdd(n, (uint32_t)__popcll(who));
    base = __shfl((int)base, 0, 64);
    if (take) list[base + __popcll(who & (((uint64_t)1 << lane) - 1))] = entry;
}

// Sorts the first `size` (a power of two) entries of a list in LDS, the largest first.
template <int THREADS> __device__ __forceinline__ void sort_descending(uint64_t* list, int size) {
    for (int k = 2; k <= size; k *= 2) {
        for (int j = k / 2; j > 0; j /= 2) {
            __syncthreads();
            for (int p = threadIdx.x; p < size / 2; p += THREADS) {
                const int x = 2 * p - (p & (j - 1)), y = x + j;
                const uint64_t a = list[x], b = list[y];
                if ((a < b) == ((x & k) == 0)) { list[x] = b; list[y] = a; }
            }
        }
    }
    __syncthreads();
}

__device__ __forceinline__ int power_of_two(int x) { return x <= 1 ? 1 : 1 << (32 - __clz(x - 1)); }

}  // namespace
#endif
