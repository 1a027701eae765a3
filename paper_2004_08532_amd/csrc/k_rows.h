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
#include <type_traits>

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

constexpr int GROUP_TILES = 16, GROUP = GROUP_TILES * 256;  // scores of long rows that a workgroup of k_tiles takes
enum TileMode {
    TILES_SUMS,       // sums of tiles and groups
    TILES_RANGE,      // best and lowest score of groups
    TILES_BEST,       // best score of every tile
    TILES_BEST_SUMS,  // the same, and sums of groups
};
struct TileArgs {
    RowScores in;
    double inv_t;
    int64_t groups;       // of a row
    float* tile_best;     // [rows][groups][GROUP_TILES]; TILES_SUMS: what the tile's sum is relative to
    double* tile_sum;
    float* group_best;    // [rows][groups]; not TILES_BEST
    double* group_sum;    // relative to the group's best
    float* group_worst;   // of the scores that are not masked, +inf without one
    uint64_t* clear;      // [rows][clear_words] that the pass sets to 0, may be null
    int64_t clear_words;
    int64_t per;          // groups of a workgroup (set by the launcher)
};
// Groups in a row for each of the workgroups of 256 threads that fill the chip, 8 per CU.
inline int64_t groups_per_workgroup(int64_t groups) { return pieces(groups, 2048); }
void kge_launch_tiles(TileArgs a, TileMode mode, hipStream_t st);

int64_t kge_top_workspace(int64_t rows, int64_t n, int m);
// Long rows whose lists are found among the tiles' best scores, and not segment by segment
bool kge_top_by_tiles(int64_t n, int m);
struct DrawArgs;  // (k_draw_list.h)
// (ids and scores, or with by_tiles the draws of `draw`, or else the sorted entries alone; lse may be null)
void kge_launch_top(const RowScores& in, int m, float temperature, int64_t* ids, float* scores, uint64_t* entries, float* lse,
                    const DrawArgs* draw, void* workspace, hipStream_t st);
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

// The 4 scores of a lane from position j of a row of n on, -inf behind its end.  (Rows start at any multiple of a score's
// size.)  The load is the same whatever the position, so that many are in flight: a lane at or behind the end reads the row's last four
// scores, and those of the tile that the row ends in are moved into place when the values are used.
template <int DT> struct Quad {
    using Vec = typename std::conditional<DT == KGE_F32, f32x4u, u16x4u>::type;
    Vec raw;
    __device__ __forceinline__ void load(const typename Score<DT>::type* row, int64_t j, int64_t n) {
        if (n >= 4) {
            raw = *reinterpret_cast<const Vec*>(row + min(j, n - 4));
        } else {  // (the positions of a row this short are 0 .. 3; what is behind its end is not used)
            raw.x = row[0];
            raw.y = row[min((int64_t)1, n - 1)];
            raw.z = row[n - 1];
            raw.w = row[n - 1];
        }
    }
    // first: of the tile, 256 scores that the wave holds.  MASK: NaN becomes -inf
    template <bool MASK = true> __device__ __forceinline__ void values(int64_t first, int64_t n, float v[4]) const {
        v[0] = widen<DT>(raw.x); v[1] = widen<DT>(raw.y); v[2] = widen<DT>(raw.z); v[3] = widen<DT>(raw.w);
        if (first + 256 > n) {
            const int64_t j = first + (threadIdx.x & 63) * 4, beyond = n >= 4 ? j - (n - 4) : 0;
#pragma unroll
            for (int k = 1; k <= 4; ++k) {
                if (beyond >= k) { v[0] = v[1]; v[1] = v[2]; v[2] = v[3]; v[3] = -INFINITY; }
            }
            if (n < 4) {
#pragma unroll
                for (int q = 0; q < 4; ++q) if (j + q >= n) v[q] = -INFINITY;
            }
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) if (MASK) v[q] = fmaxf(v[q], -INFINITY);
    }
};

constexpr uint32_t LOWEST_KEY = 0x00800000u;  // of the lowest finite number
constexpr uint32_t NEGATIVE_ZERO_KEY = 0x7FFFFFFFu;  // below that of +0; of no score
__device__ __forceinline__ uint32_t order_key(float s) {
    const uint32_t u = __float_as_uint(s + 0.f);  // -0 -> +0
    const uint32_t k = u >> 31 ? ~u : u | 0x80000000u;
    return s > -INFINITY ? k : 0u;  // (false for NaN)
}
__device__ __forceinline__ float key_score(uint32_t k) {  // of a key that is not 0
    return __uint_as_float(k >> 31 ? k & 0x7FFFFFFFu : ~k);
}
__device__ __forceinline__ int64_t entry_position(uint64_t e) { return (int64_t)(uint32_t)~(uint32_t)e; }

// exp((s - best) / T) in 64 bits, 0 of a masked score (-inf): which candidate a random number falls on is decided by sums of these, and
// the sums of 32-bit weights would move thousands of borders by more than the numbers' spacing.  As p * 2^n: n the whole number nearest to
// the exponent of 2 (its low bits appear where 1.5 * 2^52 is added), p the polynomial of degree 9 that interpolates exp2 on
// [-1/2, 1/2] at the Chebyshev nodes, off by 4e-14.  About 20 instructions where the library's exp takes twice as many; of the
// kernels that form a weight per score they are what bounds it beside the reads: 64 scores take a SIMD some 90 cycles.
struct Scale {  // what all weights of a kernel have in common
    double per, c[9];  // log2(e) / T; coefficients
    double far;        // a weight 2^-1000 lies that far below the best score
    __device__ __forceinline__ explicit Scale(double inv_t) : per(inv_t * 1.4426950408889634),
        c{0x1.62e42fefa39f7p-1, 0x1.ebfbdff8149f2p-3, 0x1.c6b08d7044119p-5, 0x1.3b2ab72b175eep-7, 0x1.5d87fe908f88ap-10, 0x1.43088e257f341p-13,
          0x1.ffcb76789860fp-17, 0x1.63ef969a64d3cp-20, 0x1.b6571de2f2351p-24}, far(1000.0 / per) {
        // (in scalar registers: a coefficient in a vector register is copied for every step, the instruction adds to its own output)
#pragma unroll
        for (int i = 0; i < 9; ++i) asm("" : "+s"(c[i]));
    }
};
struct Weights {
    const Scale& scale;
    double best;
    float floor;  // scores below have a weight of 0: 2^-1000 and less, or that of no number between the floor and the best
    __device__ __forceinline__ Weights(float b, const Scale& s) : scale(s) {
        const double f = (double)b - s.far;
        floor = fmaxf(fminf(b, (float)fma(fabs(f), 0x1p-22, f)), -3.402823466e38f);  // (rounded up; b = +inf: above every number)
        best = (double)fminf(b, 3.402823466e38f);
    }
    // (of a score at or above the floor; something else below it)
    __device__ __forceinline__ void split(float s, double& p, int& n) const {
        const double d = (double)__builtin_amdgcn_fmed3f(s, -3.402823466e38f, 3.402823466e38f) - best, shifted = fma(d, scale.per, 0x1.8p52);
        const double f = fma(d, scale.per, -(shifted - 0x1.8p52));
        n = __double2loint(shifted);
        p = scale.c[8];
#pragma unroll
        for (int i = 7; i >= 0; --i) p = fma(p, f, scale.c[i]);
        p = fma(p, f, 1.0);
    }
    static __device__ __forceinline__ double scaled(double p, int n) {  // p * 2^n, p and the result normal numbers
        return __hiloint2double(__double2hiint(p) + (n << 20), __double2loint(p));
    }
    // 0 where `keep`, which implies that s is at or above the floor, does not hold.  (Masked by its bits: a choice between the weight
    // and 0 would become a branch around every weight.)
    __device__ __forceinline__ double of(float s, bool keep) const {
        double p;
        int n;
        split(s, p, n);
        const int mask = keep ? -1 : 0;
        p = scaled(p, n);
        return __hiloint2double(__double2hiint(p) & mask, __double2loint(p) & mask);
    }
    __device__ __forceinline__ double of(float s) const { return of(s, s >= floor); }
    // For sums of many, of scores of a row whose best is finite: less than 2^-1040 instead of 0 (see some_weight).
    __device__ __forceinline__ double loose(float s, bool keep) const {
        const double d = (double)s - best, shifted = fma(d, scale.per, 0x1.8p52), f = fma(d, scale.per, -(shifted - 0x1.8p52));
        double p = scale.c[8];
#pragma unroll
        for (int i = 7; i >= 0; --i) p = fma(p, f, scale.c[i]);
        p = scaled(fma(p, f, 1.0), __double2loint(shifted));
        return __hiloint2double(keep ? __double2hiint(p) : 0, __double2loint(p));
    }
    // The sum of up to 2^10 loose weights, 0 where none of them is one.
    static __device__ __forceinline__ double some_weight(double z) { return z < 0x1p-1025 ? 0.0 : z; }
};

// The lowest key in lo .. hi for which `yes` holds, asked by a wave for 64 keys at a time; it holds for hi and for every key above one for
// which it holds.
template <typename F> __device__ __forceinline__ uint32_t lowest_key(uint32_t lo, uint32_t hi, const F& yes) {
    while (lo < hi) {
        const uint32_t step = (hi - lo) / 64 + 1;
        const uint64_t at = (uint64_t)lo + (uint64_t)((threadIdx.x & 63) + 1) * step - 1;
        const uint64_t who = __ballot(at >= hi || yes((uint32_t)at));
        const uint32_t first = (uint32_t)__ffsll((unsigned long long)who) - 1;
        hi = (uint32_t)min((uint64_t)hi, (uint64_t)lo + (uint64_t)(first + 1) * step - 1);
        lo += first * step;
    }
    return lo;
}
// The next lower score (of 0 the negative number next to it, not -0): -inf below the lowest number.
__device__ __forceinline__ float score_below(float s) {
    const uint32_t k = order_key(s);
    return k <= LOWEST_KEY ? -INFINITY : key_score(k - (k == 0x80000000u ? 2 : 1));
}

// Sums and maxima of a wave by moves within rows of 16 lanes and from row to row: no LDS on the way.
template <int CTRL, int ROWS> __device__ __forceinline__ double moved64(double v) {  // lanes without a source: 0
    const int lo = __builtin_amdgcn_update_dpp(0, __double2loint(v), CTRL, ROWS, 0xf, ROWS == 0xf);
    const int hi = __builtin_amdgcn_update_dpp(0, __double2hiint(v), CTRL, ROWS, 0xf, ROWS == 0xf);
    return __hiloint2double(hi, lo);
}
constexpr int ROW_SHR = 0x110, BCAST_15 = 0x142, BCAST_31 = 0x143;
__device__ __forceinline__ double wave_scan64(double v, int) {  // sum over lanes 0 .. own
    v += moved64<ROW_SHR + 1, 0xf>(v);
    v += moved64<ROW_SHR + 2, 0xf>(v);
    v += moved64<ROW_SHR + 4, 0xf>(v);
    v += moved64<ROW_SHR + 8, 0xf>(v);
    v += moved64<BCAST_15, 0xa>(v);
    v += moved64<BCAST_31, 0xc>(v);
    return v;
}
template <int CTRL, int ROWS> __device__ __forceinline__ uint32_t moved32(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false); }
__device__ __forceinline__ uint32_t wave_scan_u32(uint32_t v) {
    v += moved32<ROW_SHR + 1, 0xf>(v);
    v += moved32<ROW_SHR + 2, 0xf>(v);
    v += moved32<ROW_SHR + 4, 0xf>(v);
    v += moved32<ROW_SHR + 8, 0xf>(v);
    v += moved32<BCAST_15, 0xa>(v);
    v += moved32<BCAST_31, 0xc>(v);
    return v;
}
__device__ __forceinline__ double lane64(double v, int lane) {  // of one lane, the same for all
    return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), lane), __builtin_amdgcn_readlane(__double2loint(v), lane));
}
__device__ __forceinline__ double wave_sum64(double v) { return lane64(wave_scan64(v, 0), 63); }
// Of four tiles at once: the halves of two tiles' values are joined in one register, then the quarters of four, so that the steps within a row of 16
// lanes serve all.  Lane 15 of row k ends with the tile k = 0, 2, 1, 3.
__device__ __forceinline__ void swap32(int& a, int& b) {
    const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
    a = r[0]; b = r[1];
}
__device__ __forceinline__ void swap16(int& a, int& b) {
    const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
    a = r[0]; b = r[1];
}
template <bool HALVES> __device__ __forceinline__ double join64(double a, double b) {
    int al = __double2loint(a), ah = __double2hiint(a), bl = __double2loint(b), bh = __double2hiint(b);
    if (HALVES) { swap32(al, bl); swap32(ah, bh); }
    else { swap16(al, bl); swap16(ah, bh); }
    return __hiloint2double(ah, al) + __hiloint2double(bh, bl);
}
__device__ __forceinline__ double sum_four(const double z[4]) {
    double v = join64<false>(join64<true>(z[0], z[1]), join64<true>(z[2], z[3]));
    v += moved64<ROW_SHR + 1, 0xf>(v);
    v += moved64<ROW_SHR + 2, 0xf>(v);
    v += moved64<ROW_SHR + 4, 0xf>(v);
    v += moved64<ROW_SHR + 8, 0xf>(v);
    return v;
}
template <int CTRL, int ROWS> __device__ __forceinline__ float max_moved(float v) {
    return fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(-INFINITY), __float_as_int(v), CTRL, ROWS, 0xf, false)));
}
__device__ __forceinline__ float max_four(const float z[4]) {  // (in the lanes of sum_four)
    auto join = [](float a, float b, auto swap) {
        int x = __float_as_int(a), y = __float_as_int(b);
        swap(x, y);
        return fmaxf(__int_as_float(x), __int_as_float(y));
    };
    float v = join(join(z[0], z[1], swap32), join(z[2], z[3], swap32), swap16);
    v = max_moved<ROW_SHR + 1, 0xf>(v);
    v = max_moved<ROW_SHR + 2, 0xf>(v);
    v = max_moved<ROW_SHR + 4, 0xf>(v);
    return max_moved<ROW_SHR + 8, 0xf>(v);
}
__device__ __forceinline__ float wave_most(float v) {
    v = max_moved<ROW_SHR + 1, 0xf>(v);
    v = max_moved<ROW_SHR + 2, 0xf>(v);
    v = max_moved<ROW_SHR + 4, 0xf>(v);
    v = max_moved<ROW_SHR + 8, 0xf>(v);
    v = max_moved<BCAST_15, 0xa>(v);
    v = max_moved<BCAST_31, 0xc>(v);
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
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
template <int WAVES> __device__ __forceinline__ float block_max(float v, float* slot) {
    v = wave_most(v);
    if constexpr (WAVES == 1) return v;
    if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = v;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) v = fmaxf(v, slot[w]);
    __syncthreads();
    return v;
}

// What has been formed from these is formed again, and not kept in registers from one place to the other.
template <int N> __device__ __forceinline__ void forget(float v[N]) {
#pragma unroll
    for (int q = 0; q < N; ++q) asm volatile("" : "+v"(v[q]));
}

// The tiles of a workgroup in registers; returns this thread's largest score.
template <int DT, int WAVES, int TPW>
__device__ __forceinline__ float load_tiles(const typename Score<DT>::type* row, int64_t first, int64_t n, float v[TPW * 4]) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Quad<DT> x[TPW];
#pragma unroll
    for (int i = 0; i < TPW; ++i) x[i].load(row, first + (i * WAVES + wave) * 256 + lane * 4, n);
    float best = -INFINITY;
#pragma unroll
    for (int i = 0; i < TPW; ++i) {
        x[i].values(first + (i * WAVES + wave) * 256, n, v + 4 * i);
        best = fmaxf(best, fmaxf(fmaxf(v[4 * i], v[4 * i + 1]), fmaxf(v[4 * i + 2], v[4 * i + 3])));
    }
    return best;
}

// Sums of the weights of four tiles that a wave holds, relative to the best score among them; of scores above `over`.  The sums are in lane 15 of
// the rows, see sum_four.
__device__ __forceinline__ float best_of(const float v[16]) {
    float m = v[0];
#pragma unroll
    for (int q = 1; q < 16; ++q) m = fmaxf(m, v[q]);
    return wave_most(m);
}
__device__ __forceinline__ double sum_of_tiles(const float v[16], const Weights& w, float over) {
    double z[4];
    if (w.floor == INFINITY) {  // (the best is +inf: the same for the wave)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            z[i] = 0.0;
#pragma unroll
            for (int q = 4 * i; q < 4 * i + 4; ++q) z[i] += v[q] == INFINITY && v[q] > over ? 1.0 : 0.0;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            z[i] = (w.loose(v[4 * i], v[4 * i] > over) + w.loose(v[4 * i + 1], v[4 * i + 1] > over)) +
                   (w.loose(v[4 * i + 2], v[4 * i + 2] > over) + w.loose(v[4 * i + 3], v[4 * i + 3] > over));
    }
    return Weights::some_weight(sum_four(z));
}
__device__ __forceinline__ int tile_of_row(int row) { return row == 1 ? 2 : row == 2 ? 1 : row; }

template <int WAVES> __device__ __forceinline__ int tile_position(int q) {  // of register q, in the workgroup's tiles
    return ((q / 4) * WAVES + (int)(threadIdx.x >> 6)) * 256 + (int)(threadIdx.x & 63) * 4 + q % 4;
}

template <int WAVES> __device__ __forceinline__ int block_count(int c, uint32_t* slot) {  // c: of a wave
    if constexpr (WAVES == 1) return c;
    if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = c;
    __syncthreads();
    c = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) c += slot[w];
    return c;
}

// Key of the largest score that at least m of the workgroup's scores reach, by halving the interval of keys: every round
// counts the scores at or above its middle.  Ends early where exactly m do.  `reach`: how many reach the result.  Fewer than m
// candidates: the lowest key.
template <int WAVES, int N>
__device__ __forceinline__ uint32_t select_threshold(const float v[N], uint32_t best, int m, uint32_t* slots /* [2 * WAVES] */, int& reach) {
    uint32_t lo = LOWEST_KEY, hi = best;  // count(>= lo) >= m, count(> hi) < m
    int round = 0;
    auto count = [&](uint32_t key) {
        const float t = key_score(key);
        int c = 0;
#pragma unroll
        for (int q = 0; q < N; ++q) c += __popcll(__ballot(v[q] >= t));
        return block_count<WAVES>(c, slots + (round++ & 1) * WAVES);
    };
    reach = count(lo);
    if (reach <= m) return lo;
    while (lo < hi) {
        const uint32_t mid = lo + (hi - lo) / 2 + ((hi - lo) & 1);  // lo < mid <= hi
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

// Of the scores that equal t: the largest bound that c of their inverted positions reach, 1 <= c <= their number.
template <int WAVES, int N, typename L>
__device__ __forceinline__ uint32_t select_equal(const float v[N], float t, const L& low, int c, uint32_t* slots /* [2 * WAVES] */) {
    uint32_t lo = 0, hi = 0xFFFFFFFFu;
    int round = 0;
    __syncthreads();
    while (lo < hi) {
        const uint32_t mid = lo + (hi - lo) / 2 + ((hi - lo) & 1);
        int n = 0;
#pragma unroll
        for (int q = 0; q < N; ++q) n += __popcll(__ballot(v[q] == t && low(q) >= mid));
        if (block_count<WAVES>(n, slots + (round++ & 1) * WAVES) >= c) lo = mid; else hi = mid - 1;
    }
    __syncthreads();
    return lo;
}

// Appends a thread's scores whose bit is set, as entries, to a list in LDS (in any order) that has room for `room`; *n starts at 0 and ends at the
// number of those that there are.
template <int N, typename L>
__device__ __forceinline__ void append_marked(const float v[N], uint32_t marked, const L& low, uint64_t* list, uint32_t room, uint32_t* n) {
    static_assert(N <= 32, "a bit per score");
    if (!__ballot(marked != 0)) return;
    const uint32_t own = (uint32_t)__popc(marked), upto = wave_scan_u32(own);
    uint32_t at = 0;
    if ((threadIdx.x & 63) == 63) at = atomicAdd(n, upto);
    at = (uint32_t)__builtin_amdgcn_readlane((int)at, 63) + upto - own;
#pragma unroll
    for (int q = 0; q < N; ++q) {
        if (marked >> q & 1) {
            if (at < room) list[at] = (uint64_t)order_key(v[q]) << 32 | low(q);
            ++at;
        }
    }
}

// Sorts the first `size` entries (a power of two, 128 or more) of a list in LDS, the largest first.
template <int THREADS> __device__ __forceinline__ void sort_descending(uint64_t* list, int size) {
    constexpr int PAIRS = THREADS == 64 ? 2 : 1024 / THREADS;  // of a thread (one wave: lists of up to 256)
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x & ~63u), lane = threadIdx.x & 63;
    for (int k = 2; k <= size; k *= 2) {
        for (int j = k / 2; j > 0; j /= 2) {
            __syncthreads();
            uint64_t a[PAIRS], b[PAIRS];
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) {  // (all reads at once)
                const int p = wave + i * THREADS + lane, x = 2 * p - (p & (j - 1));
                if (wave + i * THREADS < size / 2) { a[i] = list[x]; b[i] = list[x + j]; }
            }
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) {
                const int p = wave + i * THREADS + lane, x = 2 * p - (p & (j - 1));
                if (wave + i * THREADS < size / 2 && (a[i] < b[i]) == ((x & k) == 0)) { list[x] = b[i]; list[x + j] = a[i]; }
            }
        }
    }
    __syncthreads();
}

__device__ __forceinline__ int power_of_two(int x) { return x <= 1 ? 1 : 1 << (32 - __clz(x - 1)); }

// The best of a workgroup's scores, as entries in an LDS list, best first.  A score that at least m of the workgroup's groups (its
// threads, or the threads' vectors of 4) reach with their largest is reached by at least m scores, and by few more than m if
// not many more groups reach it: -groups ln(1 - m / groups) where scores lie as they come, 1.4 m at m = groups / 2.  So it is enough
// to look for such a score among the groups' largest, 1024 instead of 16,384, and only until at most a quarter too many reach it; the
// candidates are then put in order.  Where they do not fit the list (equal scores, orders made for it) the threshold is found among all scores.
constexpr int BEST_ROOM = 2048;
template <int WAVES, int TPW> struct BestList {
    static constexpr int ROOM = WAVES * TPW * 256 < BEST_ROOM ? WAVES * TPW * 256 : BEST_ROOM;
    uint64_t list[ROOM];
    uint64_t sorted[256];
    float most[WAVES * 64];
    uint32_t slots[2 * WAVES], rank[256];
    uint32_t count, bound;
};

// A key that at least m, and if it is found in time at most m + m / 4 + 2, of a wave's PER values per lane reach.
template <int PER> __device__ __forceinline__ uint32_t wave_bound(const float v[PER], uint32_t best, int m) {
    uint32_t lo = LOWEST_KEY, hi = best;
    while (lo < hi) {
        const uint32_t mid = lo + (hi - lo) / 2 + ((hi - lo) & 1);
        const float t = key_score(mid);
        int c = 0;
#pragma unroll
        for (int q = 0; q < PER; ++q) c += __popcll(__ballot(v[q] >= t));
        if (c >= m) {
            lo = mid;
            if (c <= m + m / 4 + 2) break;
        } else {
            hi = mid - 1;
        }
    }
    return lo;
}

// Whether a list is put in order by counting for each entry those above it, count^2 comparisons in few steps, or by a sorting network, which has
// log^2 steps with a barrier each.  us, best m of 1565 scores (256 threads), 14 / 1024 rows, by the network -> by counting: m = 80 11.2 -> 6.9 /
// 14.2 -> 9.7, m = 150 14.5 -> 10.7 / 19.7 -> 16.5; of 6000 (512 threads): m = 60 10.5 -> 7.4 / 16.0 -> 11.4, m = 150 12.2 -> 9.4 / 17.8 -> 15.4; of 15,000
// (1024 threads, 14 rows): m = 60 12.4 -> 8.8, m = 150 14.0 -> 10.2.  One wave, of 250 scores: m = 100 (all 250 are candidates) 9.2 -> 20.  (The
// lists have up to m / 4 entries more.)
template <int THREADS> __device__ __forceinline__ bool by_counting(int count) { return count <= (THREADS == 64 ? 64 : 256); }

// Sorts the list's first `count` entries, the largest first; returns where they are.
template <int THREADS> __device__ __forceinline__ uint64_t* order_list(uint64_t* list, uint64_t* sorted, uint32_t* rank, int count) {
    if (by_counting<THREADS>(count)) {
        const int width = count <= 64 ? 64 : power_of_two(count), parts = THREADS > width ? THREADS / width : 1;
        for (int e = threadIdx.x; e < width; e += THREADS) rank[e] = 0;
        __syncthreads();
        for (int e0 = threadIdx.x; e0 < width * parts; e0 += THREADS) {
            const int e = e0 & (width - 1), part = e0 / width;
            if (e < count) {
                const uint64_t own = list[e];
                uint32_t above = 0;
                int j = part;
                for (; j + 7 * parts < count; j += 8 * parts) {
                    uint64_t y[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) y[i] = list[j + i * parts];  // (all reads at once)
#pragma unroll
                    for (int i = 0; i < 8; ++i) above += y[i] > own;
                }
                for (; j < count; j += parts) above += list[j] > own;
                if (parts > 1) atomicAdd(&rank[e], above);
                else rank[e] = above;
            }
        }
        __syncthreads();
        for (int e = threadIdx.x; e < count; e += THREADS) sorted[rank[e]] = list[e];
        __syncthreads();
        return sorted;
    }
    const int size = power_of_two(max(count, 128));
    for (int e = count + threadIdx.x; e < size; e += THREADS) list[e] = 0;
    sort_descending<THREADS>(list, size);
    return list;
}

// v: the workgroup's scores, low(q): their inverted positions in the row, `mine` this thread's largest score, `best` the key of the largest
// (not 0).  Fills the list with candidates that the best m are among (any order, list[0 .. count - 1]) and returns their number.
template <int WAVES, int TPW, typename L>
__device__ __forceinline__ int collect_best(const float v[TPW * 4], const L& low, float mine, uint32_t best, int m, BestList<WAVES, TPW>& s) {
    constexpr int N = TPW * 4, THREADS = WAVES * 64, CAP = WAVES * TPW * 256, ROOM = BestList<WAVES, TPW>::ROOM;
    uint32_t bound = LOWEST_KEY;
    if (threadIdx.x == 0) s.count = 0;
    if (m <= THREADS / 2) {
        if constexpr (WAVES == 1) {
            bound = wave_bound<1>(&mine, best, m);
        } else {
            s.most[threadIdx.x] = mine;
            __syncthreads();
            if (threadIdx.x < 64) {
                float x[WAVES];
#pragma unroll
                for (int w = 0; w < WAVES; ++w) x[w] = s.most[w * 64 + threadIdx.x];
                bound = wave_bound<WAVES>(x, best, m);
                if (threadIdx.x == 0) s.bound = bound;
            }
            __syncthreads();
            bound = s.bound;
        }
    } else if (CAP > ROOM && m <= THREADS * TPW / 2) {
        float x[TPW];
#pragma unroll
        for (int i = 0; i < TPW; ++i) x[i] = fmaxf(fmaxf(v[4 * i], v[4 * i + 1]), fmaxf(v[4 * i + 2], v[4 * i + 3]));
        int reach;
        bound = select_threshold<WAVES, TPW>(x, best, m, s.slots, reach);
    }
    __syncthreads();
    float t = key_score(bound);
    uint32_t marked = 0;
#pragma unroll
    for (int q = 0; q < N; ++q) marked |= (uint32_t)(v[q] >= t) << q;
    append_marked<N>(v, marked, low, s.list, ROOM, &s.count);
    __syncthreads();
    if constexpr (CAP > ROOM) {
        if (s.count > ROOM) {  // (the same for all) too many: exactly those that count
            uint32_t least = 0;  // of the inverted positions of scores that equal t
            __syncthreads();
            if (threadIdx.x == 0) s.count = 0;
            int reach;
            t = key_score(select_threshold<WAVES, N>(v, best, m, s.slots, reach));
            if (reach > m) {  // more than m reach it: equal scores, of which the first ones count
                int above = 0;
#pragma unroll
                for (int q = 0; q < N; ++q) above += __popcll(__ballot(v[q] > t));
                __syncthreads();
                above = block_count<WAVES>(above, s.slots);
                least = select_equal<WAVES, N>(v, t, low, m - above, s.slots);
            }
            __syncthreads();
            marked = 0;
#pragma unroll
            for (int q = 0; q < N; ++q) marked |= (uint32_t)(v[q] > t || (v[q] == t && low(q) >= least)) << q;
            append_marked<N>(v, marked, low, s.list, ROOM, &s.count);
            __syncthreads();
        }
    }
    return (int)s.count;
}

}  // namespace
#endif
