// Divergence of rows of scores from a teacher's lists of best candidates, and its gradient (kge_distill_loss, kge_distill_step).
//
// With z = s / T, w_j = exp(z_j - max z), Z = sum w, q_j = w_j / Z and the teacher's p_e over the entries e of a row's list:
//     loss   = T^2 [ sum_e p_e log(p_e / q_{id_e})  +  p_r log(p_r / q_r) ]
//     grad_j = c T [ P q_j - sum_{e: id_e = j} p_e ]   listed candidates, and all where the lists are all there is
//     grad_j = c T [ P - p_r Z / Z_r ] q_j             candidates that are not listed, where there is a rest
// p_r = 1 - sum p is the mass that the teacher has outside of the list, q_r = Z_r / Z the student's, P = sum p + p_r.
// Z_r can be less than any number where the listed candidates lie far above the others.  So what is not listed has weights relative to its own best
// score u, w'_j = exp(z_j - u / T) and Z'_r = sum w' >= 1: the gradient of these is c T [ P exp((u - max) / T) / Z - p_r / Z'_r ] w'_j.
//
// A row that a workgroup holds is read once and its gradient written once: the weights stay in registers between the sum and the gradient.
// Long rows: a pass for the sums, one workgroup per row for what their gradients have in common, a second pass for the gradient.  Weights of listed
// candidates are formed in 64 bits (but for the sum of a long row without a rest); up to T = 4 those of the others in 32 bits from an argument in 64, four of them
// added in 32.  All other sums and logarithms are in 64.
//
// 1024 rows of 14,951 fp32, lists of 64 and a rest: 37 us, 3.3 TB/s read and written (a large copy: 24 us); the vector units work for 19, and the
// phases of a row (reads, sums, list, writes) overlap only with those of two other rows on the CU.  16 rows of 2.5 M bf16, lists of 256 and a
// rest: sums 33 us (2.4 TB/s; 11.9 M wave instructions, 25 us of the vector units), lists 10, gradient 32 (5 TB/s).  690 rows of 40,943 fp16, loss
// alone: sums 24, lists 7.  1024 rows of 256, lists of 16: 7.4 us.
#include "k_rows.h"

namespace {

// What the gradients of a row have in common: of listed candidates w_j * listed - p * unit, with w relative to the row's best score and p_e =
// exp(Teacher::log_p) * scale; of the others w_j * other, with w relative to `from`.
struct RowGrad {
    double from, scale, listed, unit;
    float other;
};

struct DistillArgs {
    RowScores in;
    TeacherLists t;
    double inv_t;
    double grad_scale, loss_scale;  // grad_scale: of the call times T; loss_scale: T^2, and 1 / b in a step
    float* loss;
    void* grad;
    int64_t ld_grad;
    StepRows step;
    // long rows
    int64_t groups, per;  // groups of a row, and of a workgroup
    double* sums;         // [rows][groups][2]: a score, the weights' sum relative to it; where there is a rest of those that are not listed
    RowGrad* rows;
};

__device__ __forceinline__ float largest(float a, float b, float c) {  // NaN if one of them is
    float r;
    asm("v_maximum3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// The same for all lanes: in a scalar register.
__device__ __forceinline__ float scalar(float v) { return __uint_as_float((uint32_t)__builtin_amdgcn_readfirstlane((int)__float_as_uint(v))); }

// Weights relative to `best`.  The argument of the exponential is formed in 64 bits and its fraction taken in 32, so the weight is off by
// the roundings of exp2 alone, whatever the distance.  Masked: 0.
struct Weight32 {
    double best, per, far;  // per: log2(e) / T; 2^1024 times less than the best's: 0
    __device__ __forceinline__ Weight32(float b, double p) : best(fabsf(b) < INFINITY ? (double)b : 0.0 /* no candidate */), per(p), far(-1024.0 / p) {}
    __device__ __forceinline__ float of(float s) const {
        const double d = fmax((double)s - best, far), shifted = fma(d, per, 0x1.8p52), f = fma(d, per, -(shifted - 0x1.8p52));
        return __builtin_amdgcn_ldexpf(__builtin_amdgcn_exp2f((float)f), __double2loint(shifted));
    }
};

template <int DT> struct RowAt {
    const typename Score<DT>::type* s;
    int64_t n;
    bool is_dist;
    float gamma;
    __device__ __forceinline__ float of(float raw) const { return is_dist ? gamma - raw : raw; }
    __device__ __forceinline__ float at(int64_t j) const { return of(widen<DT>(s[j])); }
};

// exp in 64 bits.  WIDE: the library's.  Else the polynomial of the draws' weights (k_rows.h), off by 4e-14: its coefficients are in scalar registers, those of
// the library's in vector registers for all the loops over a list together (rows of 8192: 88 registers instead of 73).
template <bool WIDE> struct Exp64 {
    __device__ __forceinline__ double operator()(double x) const { return exp(x); }
};
template <> struct Exp64<false> {
    Scale scale;
    __device__ __forceinline__ Exp64() : scale(1.0) {}
    __device__ __forceinline__ double operator()(double x) const {
        x = x < -800.0 ? -800.0 : x > 800.0 ? 800.0 : x;  // (NaN stays)
        const double shifted = fma(x, scale.per, 0x1.8p52), f = fma(x, scale.per, -(shifted - 0x1.8p52));
        double p = scale.c[8];
#pragma unroll
        for (int i = 7; i >= 0; --i) p = fma(p, f, scale.c[i]);
        return __builtin_ldexp(fma(p, f, 1.0), __double2loint(shifted));
    }
};

// An entry of a list: the candidate's position, -1 if the entry is not used.
template <int DT> __device__ __forceinline__ int64_t list_position(const DistillArgs& a, int64_t row, int e, int64_t n) {
    const int64_t id = a.t.ids[row * a.t.m + e];
    return id >= 0 && id < n && a.t.scores[row * a.t.m + e] != -INFINITY ? id : -1;
}

// log p of an entry before p is scaled: relative to the teacher's log-sum-exp, or to the largest score of the list.
struct Teacher {
    const float* scores;
    double inv_t, best, lse;
    __device__ __forceinline__ Teacher(const DistillArgs& a, int64_t row, float most)
        : scores(a.t.scores + row * a.t.m), inv_t(a.inv_t), best(a.t.lse || !(most > -INFINITY) ? 0.0 : (double)most), lse(a.t.lse ? (double)a.t.lse[row] : 0.0) {}
    __device__ __forceinline__ double log_p(int e) const { return ((double)scores[e] - best) * inv_t - lse; }
};

struct ListSums { double a, b, z; };  // sum of p before it is scaled, sum of p * (log p - (s - best) / T), MARKED: of the weights of the list's candidates

struct Entry { double p, w; };  // before p is scaled; the student's weight

// A thread's part of the list's sums.  stands(e): the first entry of its candidate.  `own` becomes the thread's first entry.
template <int DT, int THREADS, bool MARKED, typename X, typename S>
__device__ __forceinline__ ListSums sum_list(const DistillArgs& a, int64_t row, const RowAt<DT>& r, const Teacher& teacher, double best, const X& exp_of, const S& stands, Entry& own) {
    ListSums l = {0.0, 0.0, 0.0};
#pragma unroll 1
    for (int e = threadIdx.x; e < a.t.m; e += THREADS) {
        const int64_t id = list_position<DT>(a, row, e, r.n);
        if (id < 0) continue;
        const double lp = teacher.log_p(e), p = exp_of(lp), x = ((double)r.at(id) - best) * a.inv_t;
        l.a += p;
        if (p > 0.0 || p != p) l.b += p * (lp - x);
        if (!MARKED && !a.grad) continue;
        const double w = x < INFINITY ? exp_of(x) : __longlong_as_double(0x7FF8000000000000ll);  // (of +inf and NaN)
        if (MARKED && stands(e)) l.z += w;
        if (e == (int)threadIdx.x) own = {p, w};
    }
    return l;
}

// (What fp32 does not hold becomes its largest value: a weight of 0 times it is a gradient of 0.)
__device__ __forceinline__ float coefficient(double x) {
    const double most = 3.402823466e38;
    return (float)(x > most ? most : x < -most ? -most : x);
}

// Weights of a row: z = Z, relative to the row's best score; z_rest: of the candidates that are not listed (of all, where that makes no difference), relative
// to the score `from`, whose own weight is `shift`.
struct RowSums {
    double best, from, shift, z, z_rest;
};
template <typename X>
__device__ __forceinline__ RowSums row_sums(const DistillArgs& a, double best, double from, const ListSums& l, double z_rest, const X& exp_of) {
    const double shift = from == best ? 1.0 : exp_of((from - best) * a.inv_t);
    return {best, from, shift, z_rest > 0.0 ? l.z + z_rest * shift : l.z + z_rest, z_rest};
}
// From these and the sums of the row's list.
__device__ __forceinline__ RowGrad row_grad(const DistillArgs& a, const RowSums& s, const ListSums& l) {
    double mass = l.a, scale = 1.0, rest = 0.0;
    if (a.t.lse) {
        rest = fmax(1.0 - mass, 0.0);
        if (!(s.z_rest > 0.0)) rest = 0.0;  // no candidate that it could go to
    } else {
        scale = mass > 0.0 || mass != mass ? 1.0 / mass : 0.0;
        mass *= scale;
    }
    RowGrad g = {s.from, scale, 0.0, 0.0, 0.f};
    const double c = a.grad_scale;
    if (s.z != 0.0 && mass + rest != 0.0) {
        const double own = c * (mass + rest) / s.z;
        g.listed = own;
        g.other = rest > 0.0 ? coefficient(own * s.shift - c * rest / s.z_rest) : s.z_rest > 0.0 ? coefficient(own * s.shift) : coefficient(own);
        g.unit = c;
    }
    return g;
}
__device__ __forceinline__ double row_loss(const DistillArgs& a, const RowSums& s, const ListSums& l) {
    double mass = l.a, cross = l.b, rest = 0.0;
    if (a.t.lse) {
        rest = s.z_rest > 0.0 ? fmax(1.0 - mass, 0.0) : 0.0;
    } else if (mass > 0.0 || mass != mass) {  // log p has still to lose the logarithm of the sum
        cross = cross / mass - log(mass);
        mass /= mass;
    }
    if (s.z == 0.0 || mass + rest == 0.0) return 0.0;
    double loss = cross + mass * log(s.z);
    if (rest > 0.0) loss += rest * (log(rest * s.z / s.z_rest) - (s.from - s.best) * a.inv_t);
    return loss * a.loss_scale;
}

// Above T = 4 the weights of candidates that are not listed are formed in 64 bits, too.  An error e of their sum's logarithm is multiplied with |p_r - q_r|, which falls as
// 1 / T, and the divergence that T^2 multiplies falls as 1 / T^2 where student and teacher are near each other: the loss is off by e T of itself, and e is some 1e-8 in
// 32 bits.  The sums of p log(p / q), which are near 0, and of what is near 1 lose bits in the same way, so with delta_e = log(p_e / q_e), the same for the rest,
// and sums of p and of q that are both 1:
//     sum p delta = sum (p delta - p + q) = sum p (delta + expm1(-delta)),    P q - p = p expm1(-delta) + (P - 1) q
// whose terms are all small of themselves: an error of delta, 2^-53 times the size of the logarithms in it, is multiplied with |p - q|.
// Largest error of a loss beside the loss, 14,952 candidates, lists of 64 and a rest, 32 bits -> 64: T = 4 7e-8 (half a step of fp32 is 6e-8), T = 8 9e-8 -> 5e-8, T = 100
// 5e-7 -> 5e-8, T = 1000 8e-6 -> 5e-8.  us, 1024 rows of 256 / 14,951 with their gradient 8.0 -> 8.4 / 34 -> 43, 64 rows of 100,000 30 -> 33.
constexpr float WIDE_TEMPERATURE = 4.f;
struct WideRow {
    double log_z, log_mass;  // of the student's weights, of the list's p before they are scaled
    double excess, rest;     // P - 1; what the candidates that are not listed add to the loss / T^2
    int live;
};
// p log(p / q) - p + q
__device__ __forceinline__ double wide_term(double p, double delta, double q) {
    return fabs(delta) < 1.0 ? p * (delta + expm1(-delta)) : (p > 0.0 || p != p ? p * delta : 0.0) - p + q;
}
__device__ __forceinline__ WideRow wide_row(const DistillArgs& a, const RowSums& s, const ListSums& l, RowGrad& g) {
    WideRow w = {log(s.z), 0.0, 0.0, 0.0, 0};
    double rest = 0.0;
    if (a.t.lse) {
        if (s.z_rest > 0.0) rest = fmax(1.0 - l.a, 0.0);
        if (!(rest > 0.0)) w.excess = l.a - 1.0;
    } else {
        w.log_mass = log(l.a);
    }
    w.live = s.z != 0.0 && l.a + rest != 0.0;
    const double q = s.z_rest > 0.0 ? s.z_rest * s.shift / s.z : s.z_rest, c = a.grad_scale;
    g = {s.from, 1.0, 0.0, 0.0, 0.f};
    if (rest > 0.0) {
        const double delta = log(rest * s.z / s.z_rest) - (s.from - s.best) * a.inv_t;
        w.rest = wide_term(rest, delta, q);
        g.other = coefficient(fabs(delta) < 1.0 ? c * (rest / s.z_rest) * expm1(-delta) : c * (s.shift / s.z - rest / s.z_rest));
    } else {
        w.rest = w.excess + q;
        if (w.live) g.other = coefficient(c * (1.0 + w.excess) * s.shift / s.z);
    }
    return w;
}
struct WideEntry {
    double p, delta, q;
    __device__ __forceinline__ WideEntry(const Teacher& teacher, const WideRow& w, int e, double x /* (s - best) / T */) {
        const double lp = teacher.log_p(e) - w.log_mass;
        delta = lp - x + w.log_z;
        p = exp(lp);
        q = exp(x - w.log_z);
    }
    __device__ __forceinline__ double grad(double excess) const {
        return fabs(delta) < 1.0 ? p * expm1(-delta) + excess * q : (1.0 + excess) * q - p;
    }
};
// What a list adds to the loss / T^2: a thread's part.  position(e): of an entry's candidate, -1 if it is not used.  (The q of a candidate is counted once.)
template <int THREADS, typename R, typename P, typename S>
__device__ __forceinline__ double wide_list(const DistillArgs& a, const R& r, const Teacher& teacher, double best, const WideRow& w, const P& position, const S& stands) {
    double sum = 0.0;
#pragma unroll 1
    for (int e = threadIdx.x; e < a.t.m; e += THREADS) {
        const int64_t at = position(e);
        if (at < 0) continue;
        const WideEntry x(teacher, w, e, ((double)r.at(at) - best) * a.inv_t);
        sum += wide_term(x.p, x.delta, x.q) - (stands(e) ? 0.0 : x.q);
    }
    return sum;
}
// A listed candidate's gradient by its first entry e; repeated: there are more of them.
template <typename R, typename P>
__device__ __forceinline__ double wide_grad(const DistillArgs& a, const R& r, const Teacher& teacher, double best, const WideRow& w, const P& position, int e, int64_t at, bool repeated) {
    if (!w.live) return 0.0;
    const WideEntry x(teacher, w, e, ((double)r.at(at) - best) * a.inv_t);
    double sum = x.grad(w.excess);
    if (repeated)
        for (int y = e + 1; y < a.t.m; ++y) if (position(y) == at) sum -= exp(teacher.log_p(y) - w.log_mass);
    return a.grad_scale * sum;
}

// Gradients j .. j + 3 of a row of n, but those of candidates whose bit is set.
template <int DT>
__device__ __forceinline__ void store_unlisted(typename Score<DT>::type* row, int64_t j, int64_t n, const float v[4], uint32_t bits) {
    if (j + 4 <= n && bits == 0) {
        if constexpr (DT == KGE_F32) {
            f32x4u x;
            x.x = v[0]; x.y = v[1]; x.z = v[2]; x.w = v[3];
            *reinterpret_cast<f32x4u*>(row + j) = x;
        } else {
            u16x4u x;
            x.x = narrow<DT>(v[0]); x.y = narrow<DT>(v[1]); x.z = narrow<DT>(v[2]); x.w = narrow<DT>(v[3]);
            *reinterpret_cast<u16x4u*>(row + j) = x;
        }
    } else {
#pragma unroll
        for (int q = 0; q < 4; ++q) if (j + q < n && !(bits >> q & 1)) row[j + q] = narrow<DT>(v[q]);
    }
}

// (Workgroups of 512: 80 registers for three rows on a CU; of rows of 16,384, 9 are spilled.  us, 4096 rows of 15,000 at two rows -> at three 147 -> 116; of 5000,
// where nothing is spilled, 73 -> 58.)
template <int DT, int WAVES, int TPW, bool WIDE, bool STEP>
__global__ __launch_bounds__(WAVES * 64, WAVES != 8 ? 1 : !WIDE ? 6 : 4) void k_distill(DistillArgs a) {
    constexpr int CAP = WAVES * TPW * 256, THREADS = WAVES * 64, N = TPW * 4;
    __shared__ uint32_t listed[CAP / 32];  // a bit per candidate
    __shared__ int32_t list_at[KGE_TOP_MAX];
    __shared__ float maxima[3][WAVES];
    __shared__ double parts[4][WAVES];
    __shared__ RowGrad shared_grad;
    __shared__ WideRow shared_wide;
    __shared__ int twice;  // a candidate is listed more than once
    const int64_t row = flat_block();
    if (row >= a.in.rows) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    RowAt<DT> r;
    r.s = static_cast<const typename Score<DT>::type*>(a.in.p) + row * a.in.ld;
    r.n = a.in.n;
    r.is_dist = STEP && a.step.is_dist; r.gamma = STEP ? a.step.gamma : 0.f;

    for (int x = threadIdx.x; x < CAP / 32; x += THREADS) listed[x] = 0;
    if (threadIdx.x == 0) twice = 0;
    Quad<DT> x[TPW];
#pragma unroll
    for (int i = 0; i < TPW; ++i) x[i].load(r.s, (i * WAVES + wave) * 256 + lane * 4, r.n);
    __syncthreads();
    float list_best = -INFINITY, listed_best = -INFINITY;  // of the teacher's scores, of the student's
#pragma unroll 1
    for (int e = threadIdx.x; e < a.t.m; e += THREADS) {
        const int at = (int)list_position<DT>(a, row, e, r.n);
        list_at[e] = at;
        if (at >= 0) {
            const uint32_t bit = 1u << (at & 31);
            if (atomicOr(&listed[at >> 5], bit) & bit) twice = 1;
            list_best = fmaxf(list_best, a.t.scores[row * a.t.m + e]);
            listed_best = fmaxf(listed_best, r.at(at));
        }
    }
    __syncthreads();
    // The list's candidates have no part in the registers' weights, which are relative to the best of the others.
    float v[N], from = -INFINITY;
#pragma unroll
    for (int i = 0; i < TPW; ++i) {
        const int tile = (i * WAVES + wave) * 256, at = tile + lane * 4;
        const uint32_t bits = listed[at >> 5] >> (at & 31);
        x[i].template values<false>(tile, r.n, v + 4 * i);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if constexpr (STEP) if (at + q < r.n) v[4 * i + q] = r.of(v[4 * i + q]);
            const int mask = __builtin_amdgcn_sbfe((int)bits, q, 1);  // (-1: listed)
            v[4 * i + q] = __int_as_float((mask & (int)0xFF800000) | (~mask & __float_as_int(v[4 * i + q])));
        }
        from = largest(largest(from, v[4 * i], v[4 * i + 1]), v[4 * i + 2], v[4 * i + 3]);
    }
    const bool bad = __ballot(!(from < INFINITY)) != 0;  // NaN or +inf: the row's sums are NaN
    from = bad ? INFINITY : wave_most(from);
    list_best = wave_most(list_best);
    listed_best = wave_most(listed_best);
    if (lane == 0) { maxima[0][wave] = from; maxima[1][wave] = list_best; maxima[2][wave] = listed_best; }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        from = fmaxf(from, maxima[0][w]);
        list_best = fmaxf(list_best, maxima[1][w]);
        listed_best = fmaxf(listed_best, maxima[2][w]);
    }
    from = scalar(from);
    const float best = scalar(fmaxf(from, listed_best));
    const Teacher teacher(a, row, scalar(list_best));
    const double per = a.inv_t * 1.4426950408889634;
    const Weight32 relative(from, per);
    double z = 0.0;
    forget<N>(v);
    if constexpr (WIDE) {  // (the registers keep the scores)
        const Scale scale(a.inv_t);
        const Weights wide(from, scale);
#pragma unroll
        for (int q = 0; q < N; ++q) {
            z += wide.of(v[q]);
            if (q % 4 == 3) __builtin_amdgcn_sched_barrier(0);
        }
    } else {
#pragma unroll
        for (int i = 0; i < TPW; ++i) {
#pragma unroll
            for (int q = 4 * i; q < 4 * i + 4; ++q) v[q] = relative.of(v[q]);
            z += (double)((v[4 * i] + v[4 * i + 1]) + (v[4 * i + 2] + v[4 * i + 3]));
            __builtin_amdgcn_sched_barrier(0);  // (tile by tile: the 64-bit halves of all weights at once would not fit the registers)
        }
    }
    forget<N>(v);
    auto stands = [&](int e) {
        bool first = true;
        if (twice) for (int x = 0; x < e; ++x) first = first && list_at[x] != list_at[e];
        return first;
    };
    const double top = fabsf(best) < INFINITY ? (double)best : 0.0;
    ListSums l = {0.0, 0.0, 0.0};
    const Exp64<WIDE> exp_of;
    Entry own = {0.0, 0.0};  // (most lists have at most an entry per thread: nothing is formed twice)
    z = wave_sum64(z);
    if (wave * 64 < a.t.m) {
        l = sum_list<DT, THREADS, true>(a, row, r, teacher, top, exp_of, stands, own);
        l.a = wave_sum64(l.a);
        l.b = wave_sum64(l.b);
        l.z = wave_sum64(l.z);
    }
    if (lane == 0) { parts[0][wave] = z; parts[1][wave] = l.z; parts[2][wave] = l.a; parts[3][wave] = l.b; }
    __syncthreads();
    if (wave == 0) {  // (one wave for all: the divisions and logarithms of a row are as much work as a tile)
        double sum[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) sum[k] = wave_sum64(lane < WAVES ? parts[k][lane] : 0.0);
        l = {sum[2], sum[3], sum[1]};
        const RowSums sums = row_sums(a, top, relative.best, l, best == INFINITY ? __longlong_as_double(0x7FF8000000000000ll) : sum[0], exp_of);
        if (lane == 0) {
            if constexpr (WIDE) {
                shared_wide = wide_row(a, sums, l, shared_grad);
            } else {
                if (a.loss) a.loss[row] = (float)row_loss(a, sums, l);
                shared_grad = row_grad(a, sums, l);
            }
            if constexpr (STEP) a.step.cpos[row] = 0.f;
        }
    }
    auto position = [&](int e) { return (int64_t)list_at[e]; };
    if (WIDE && a.loss) {
        __syncthreads();
        const double sum = block_sum64<WAVES>(wide_list<THREADS>(a, r, teacher, top, shared_wide, position, stands), parts[0]);
        if (threadIdx.x == 0) a.loss[row] = shared_wide.live ? (float)((sum + shared_wide.rest) * a.loss_scale) : 0.f;
    }
    if (!a.grad) return;
    __syncthreads();
    const RowGrad g = shared_grad;
    auto* out = static_cast<typename Score<DT>::type*>(a.grad) + row * a.ld_grad;
    auto shape = [&](float x, float raw) {  // a gradient as the backward products of a step want it
        if constexpr (STEP) {
            if (r.is_dist) x = raw > 0.f ? x / raw : 0.f;
            if (a.step.bf16) x = round_bf16(x);
        }
        return x;
    };
    // The list's candidates are stored here and left out below, so that neither has to wait for the other.  The first entry of a candidate
    // stands for all of them.
#pragma unroll 1
    for (int e = threadIdx.x; e < a.t.m; e += THREADS) {
        const int at = list_at[e];
        if (at < 0) continue;
        if (!stands(e)) continue;
        const float raw = widen<DT>(r.s[at]);
        float x;
        if constexpr (WIDE) {
            x = (float)wide_grad(a, r, teacher, top, shared_wide, position, e, at, twice != 0);
        } else {
            if (e >= THREADS) own = {exp_of(teacher.log_p(e)), exp_of(((double)r.of(raw) - top) * a.inv_t)};
            double p = own.p;
            if (twice) {
                for (int y = e + 1; y < a.t.m; ++y) if (list_at[y] == at) p += exp_of(teacher.log_p(y));
            }
            x = (float)(own.w * g.listed - p * g.scale * g.unit);
        }
        out[at] = narrow<DT>(shape(x, raw));
    }
#pragma unroll
    for (int i = 0; i < TPW; ++i) {
        const int tile = (i * WAVES + wave) * 256, at = tile + lane * 4;
        float x[4], raw[4] = {};
        if constexpr (STEP) {
            Quad<DT> again;
            again.load(r.s, at, r.n);
            again.template values<false>(tile, r.n, raw);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) x[q] = shape((WIDE ? relative.of(v[4 * i + q]) : v[4 * i + q]) * g.other, raw[q]);
        if (at < r.n) store_unlisted<DT>(out, at, r.n, x, listed[at >> 5] >> (at & 31) & 15u);
        if constexpr (STEP) __builtin_amdgcn_sched_barrier(0);
    }
}

// ---------------------------------------------------------------------------------------------------------
// Long rows, groups of GROUP scores.  Workgroups go through ranges of groups as in k_tiles; the positions of a row's list stay in registers
// while they do (up to 4 per thread), and those in a group become bits in LDS.
// ---------------------------------------------------------------------------------------------------------
constexpr int LIST_PER = KGE_TOP_MAX / 256, GROUP_WORDS = GROUP / 32;

struct GroupWalk {
    int64_t row, group;
    __device__ __forceinline__ void step(int64_t groups) { if (++group == groups) { group = 0; ++row; } }
};

// The bits of the listed candidates of a group.  Three sets: this group's, the next one's, and one that is cleared for the group after that, so
// that one barrier per group is enough.
template <int DT> struct GroupMarks {
    int64_t pos[LIST_PER];
    __device__ __forceinline__ void load(const DistillArgs& a, int64_t row) {
#pragma unroll
        for (int k = 0; k < LIST_PER; ++k) {
            const int e = k * 256 + threadIdx.x;
            pos[k] = e < a.t.m ? list_position<DT>(a, row, e, a.in.n) : -1;
        }
    }
    __device__ __forceinline__ void set(const DistillArgs& a, int64_t group, uint32_t* bits) const {
#pragma unroll
        for (int k = 0; k < LIST_PER; ++k) {
            if (k * 256 >= a.t.m) break;
            const int64_t p = pos[k] - group * GROUP;
            if (pos[k] >= 0 && p >= 0 && p < GROUP) atomicOr(&bits[p >> 5], 1u << (p & 31));
        }
    }
};
__device__ __forceinline__ void clear_marks(uint32_t* bits) { if (threadIdx.x < GROUP_WORDS) bits[threadIdx.x] = 0; }
__device__ __forceinline__ uint32_t marks_of(const uint32_t* bits, int p) { return bits[p >> 5] >> (p & 31) & 15u; }

// Sums of the weights of a workgroup's part of a row, noted with its last group; its other groups note none.  A wave adds up relative to a score of
// its own, the best of the first scores it meets, and takes another one only when a score lies 2^40 above (in weights).
template <int DT, bool WIDE>
__global__ __launch_bounds__(256) void k_distill_sums(DistillArgs a) {
    __shared__ uint32_t listed[3][GROUP_WORDS];
    __shared__ double parts[2][4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t blocks = a.in.rows * a.groups, start = (int64_t)flat_block() * a.per, end = min(start + a.per, blocks);
    if (start >= blocks) return;
    GroupWalk at = {start / a.groups, 0};
    at.group = start - at.row * a.groups;
    const auto* scores = static_cast<const typename Score<DT>::type*>(a.in.p);
    const double per = a.inv_t * 1.4426950408889634;
    const bool rest = WIDE || a.t.lse;
    const Scale scale(a.inv_t);
    Quad<DT> x[4];
    auto load = [&](const GroupWalk& w) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i].load(scores + w.row * a.in.ld, w.group * GROUP + (wave * 4 + i) * 256 + lane * 4, a.in.n);
    };
    GroupMarks<DT> marks;
    load(at);
    if (rest) {
        marks.load(a, at.row);
        for (int k = 0; k < 3; ++k) clear_marks(listed[k]);
        __syncthreads();
        marks.set(a, at.group, listed[0]);
        __syncthreads();
    }
    float base = -INFINITY, limit = -INFINITY;
    double z = 0.0;  // of this lane
    Weight32 weight(base, per);
    int turn = 0;
    for (int64_t block = start; block < end; ++block) {
        const GroupWalk here = at;
        float v[16], best = -INFINITY;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i].template values<false>(here.group * GROUP + (wave * 4 + i) * 256, a.in.n, v + 4 * i);
            if (!rest) best = largest(largest(best, v[4 * i], v[4 * i + 1]), v[4 * i + 2], v[4 * i + 3]);
        }
        if (rest) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t bits = marks_of(listed[turn], (wave * 4 + i) * 256 + lane * 4);
                if (bits) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) if (bits >> q & 1) v[4 * i + q] = -INFINITY;
                }
                best = largest(largest(best, v[4 * i], v[4 * i + 1]), v[4 * i + 2], v[4 * i + 3]);
            }
        }
        at.step(a.groups);
        const int next = turn == 2 ? 0 : turn + 1;
        if (block + 1 < end) {
            load(at);  // (arrives while these are worked on)
            if (rest) {
                if (at.row != here.row) marks.load(a, at.row);
                marks.set(a, at.group, listed[next]);
                clear_marks(listed[next == 2 ? 0 : next + 1]);
            }
        }
        if (__ballot(!(best <= limit))) {  // far above what the sums are relative to, or NaN
            const bool bad = __ballot(!(best < INFINITY)) != 0;
            const float top = wave_most(best);
            if (bad) {
                z = __longlong_as_double(0x7FF8000000000000ll);
                limit = INFINITY;  // (NaN comes back here, and is NaN again)
            } else if (top > limit) {
                const double f = base > -INFINITY ? exp2(((double)base - (double)top) * per) : 0.0;
                z = f == 0.0 && !(z != z) ? 0.0 : z * f;
                base = top;
                limit = top + (float)fmin(40.0 / per, 3e38);
                weight = Weight32(base, per);
            }
        }
        if constexpr (WIDE) {
            const Weights wide(base, scale);
#pragma unroll
            for (int q = 0; q < 16; ++q) {
                z += wide.of(v[q]);
                if (q % 4 == 3) __builtin_amdgcn_sched_barrier(0);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float four = (weight.of(v[4 * i]) + weight.of(v[4 * i + 1])) + (weight.of(v[4 * i + 2]) + weight.of(v[4 * i + 3]));
                z += (double)four;
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        turn = next;
        const bool last = block + 1 == end || at.row != here.row;
        if (last) {
            z = wave_sum64(z);
            if (lane == 0) { parts[0][wave] = (double)base; parts[1][wave] = z; }
            base = limit = -INFINITY;
            z = 0.0;
        }
        if (last || rest) __syncthreads();
        if (threadIdx.x == 0) {
            double* p = a.sums + 2 * block;
            double top = -INFINITY, s = 0.0;
            if (last) {
#pragma unroll 1
                for (int w = 0; w < 4; ++w) top = fmax(top, parts[0][w]);
#pragma unroll 1
                for (int w = 0; w < 4; ++w) {
                    const double b = parts[0][w], f = b == top ? 1.0 : exp2((b - top) * per);
                    if (parts[1][w] != 0.0) s += parts[1][w] * f;
                }
            }
            p[0] = top; p[1] = s;
        }
        if (last) __syncthreads();
    }
}

// A row's loss, what its gradients have in common, and the gradients of its listed candidates: k_distill_grad leaves these out, and what it reads in
// their place (where gradients replace the scores) does not matter to it.
template <int DT, bool WIDE>
__global__ __launch_bounds__(256) void k_distill_finish(DistillArgs a) {
    constexpr int SLOTS = 2 * KGE_TOP_MAX;
    __shared__ double slot[4];
    __shared__ float maxima[4];
    __shared__ uint32_t key[SLOTS], first[SLOTS], times[SLOTS];  // candidates of the list, its first entry and their number
    __shared__ uint16_t entry_slot[KGE_TOP_MAX];
    __shared__ RowGrad shared_grad;
    __shared__ WideRow shared_wide;
    const int64_t row = flat_block();
    if (row >= a.in.rows) return;
    RowAt<DT> r;
    r.s = static_cast<const typename Score<DT>::type*>(a.in.p) + row * a.in.ld;
    r.n = a.in.n; r.is_dist = false; r.gamma = 0.f;
    const double* p = a.sums + 2 * row * a.groups;
    const double per = a.inv_t * 1.4426950408889634;
    const bool rest = WIDE || a.t.lse;
    constexpr uint32_t NONE = 0xFFFFFFFFu;  // (not a position: rows have fewer than 2^32 candidates)
    for (int x = threadIdx.x; x < SLOTS; x += 256) { key[x] = NONE; first[x] = NONE; times[x] = 0; }
    float from = -INFINITY, list_best = -INFINITY, listed_best = -INFINITY;  // best of what the sums are of, of the teacher's scores, of the student's in the list
    for (int64_t g = threadIdx.x; g < a.groups; g += 256) from = fmaxf(from, (float)p[2 * g]);
    __syncthreads();
    for (int e = threadIdx.x; e < a.t.m; e += 256) {
        const int64_t id = list_position<DT>(a, row, e, r.n);
        if (id < 0) { entry_slot[e] = 0xFFFF; continue; }
        list_best = fmaxf(list_best, a.t.scores[row * a.t.m + e]);
        if (rest) listed_best = fmaxf(listed_best, r.at(id));
        uint32_t x = ((uint32_t)id * 2654435761u) >> 21;  // (2^11 slots for up to 2^10 candidates: there is always a free one)
        while (true) {
            const uint32_t was = atomicCAS(&key[x], NONE, (uint32_t)id);
            if (was == NONE || was == (uint32_t)id) break;
            x = (x + 1) & (SLOTS - 1);
        }
        atomicMin(&first[x], (uint32_t)e);
        atomicAdd(&times[x], 1u);
        entry_slot[e] = (uint16_t)x;
    }
    from = block_max<4>(from, maxima);
    list_best = block_max<4>(list_best, maxima);
    if (rest) listed_best = block_max<4>(listed_best, maxima);
    const float best = fmaxf(from, listed_best);
    const double b = best > -INFINITY ? (double)best : 0.0;
    double z_rest = 0.0;
    for (int64_t g = threadIdx.x; g < a.groups; g += 256)
        if (p[2 * g + 1] != 0.0) z_rest += p[2 * g + 1] * (p[2 * g] == (double)from ? 1.0 : exp2((p[2 * g] - (double)from) * per));
    z_rest = block_sum64<4>(z_rest, slot);
    const Teacher teacher(a, row, list_best);
    auto stands = [&](int e) { return first[entry_slot[e]] == (uint32_t)e; };
    const Exp64<WIDE> exp_of;
    Entry own = {0.0, 0.0};
    ListSums l = rest ? sum_list<DT, 256, true>(a, row, r, teacher, b, exp_of, stands, own) : sum_list<DT, 256, false>(a, row, r, teacher, b, exp_of, stands, own);
    l.a = block_sum64<4>(l.a, slot);
    l.b = block_sum64<4>(l.b, slot);
    if (rest) l.z = block_sum64<4>(l.z, slot);
    const RowSums sums = row_sums(a, b, from > -INFINITY ? (double)from : b, l, z_rest, exp_of);
    if (threadIdx.x == 0) {
        if constexpr (WIDE) {
            shared_wide = wide_row(a, sums, l, shared_grad);
        } else {
            if (a.loss) a.loss[row] = (float)row_loss(a, sums, l);
            shared_grad = row_grad(a, sums, l);
        }
        a.rows[row] = shared_grad;
    }
    auto position = [&](int e) { return entry_slot[e] == 0xFFFF ? (int64_t)-1 : (int64_t)key[entry_slot[e]]; };
    if (WIDE && a.loss) {
        __syncthreads();
        const double sum = block_sum64<4>(wide_list<256>(a, r, teacher, b, shared_wide, position, stands), slot);
        if (threadIdx.x == 0) a.loss[row] = shared_wide.live ? (float)((sum + shared_wide.rest) * a.loss_scale) : 0.f;
    }
    __syncthreads();
    if (!a.grad) return;
    const RowGrad g = shared_grad;
    auto* out = static_cast<typename Score<DT>::type*>(a.grad) + row * a.ld_grad;
    for (int e = threadIdx.x; e < a.t.m; e += 256) {
        const uint32_t x = entry_slot[e];
        if (x == 0xFFFF || first[x] != (uint32_t)e) continue;
        if constexpr (WIDE) {
            out[key[x]] = narrow<DT>((float)wide_grad(a, r, teacher, b, shared_wide, position, e, key[x], times[x] > 1));
        } else {
            if (e >= 256) own = {exp_of(teacher.log_p(e)), exp_of(((double)r.at(key[x]) - b) * a.inv_t)};
            double sum = own.p;
            uint32_t left = times[x] - 1;
            for (int y = e + 1; left; ++y) {
                if (entry_slot[y] != x) continue;
                sum += exp_of(teacher.log_p(y));
                --left;
            }
            out[key[x]] = narrow<DT>((float)(own.w * g.listed - sum * g.scale * g.unit));
        }
    }
}

template <int DT>
__global__ __launch_bounds__(256) void k_distill_grad(DistillArgs a) {
    __shared__ uint32_t listed[3][GROUP_WORDS];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t blocks = a.in.rows * a.groups, start = (int64_t)flat_block() * a.per, end = min(start + a.per, blocks);
    if (start >= blocks) return;
    GroupWalk at = {start / a.groups, 0};
    at.group = start - at.row * a.groups;
    const auto* scores = static_cast<const typename Score<DT>::type*>(a.in.p);
    const double per = a.inv_t * 1.4426950408889634;
    Quad<DT> x[4];
    auto load = [&](const GroupWalk& w) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i].load(scores + w.row * a.in.ld, w.group * GROUP + (wave * 4 + i) * 256 + lane * 4, a.in.n);
    };
    GroupMarks<DT> marks;
    load(at);
    marks.load(a, at.row);
    for (int k = 0; k < 3; ++k) clear_marks(listed[k]);
    __syncthreads();
    marks.set(a, at.group, listed[0]);
    __syncthreads();
    Weight32 weight((float)a.rows[at.row].from, per);
    float other = a.rows[at.row].other;
    int turn = 0;
    for (int64_t block = start; block < end; ++block) {
        const GroupWalk here = at;
        float v[16];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i].template values<false>(here.group * GROUP + (wave * 4 + i) * 256, a.in.n, v + 4 * i);
        at.step(a.groups);
        const int next = turn == 2 ? 0 : turn + 1;
        if (block + 1 < end) {
            load(at);
            if (at.row != here.row) marks.load(a, at.row);
            marks.set(a, at.group, listed[next]);
            clear_marks(listed[next == 2 ? 0 : next + 1]);
        }
        auto* out = static_cast<typename Score<DT>::type*>(a.grad) + here.row * a.ld_grad;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int p = (wave * 4 + i) * 256 + lane * 4;
            const int64_t j = here.group * GROUP + p;
            float y[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) y[q] = weight.of(v[4 * i + q]) * other;
            if (j < a.in.n) store_unlisted<DT>(out, j, a.in.n, y, marks_of(listed[turn], p));
            __builtin_amdgcn_sched_barrier(0);
        }
        turn = next;
        if (block + 1 < end && at.row != here.row) {
            weight = Weight32((float)a.rows[at.row].from, per);
            other = a.rows[at.row].other;
        }
        __syncthreads();
    }
}

// c: the context of a training step, whose launches are timed; null otherwise
template <int DT, bool WIDE, bool STEP>
void launch_rows(kge_ctx* c, const DistillArgs& a, hipStream_t st) {
    const int64_t n = a.in.n;
    const dim3 grid = flat_grid(a.in.rows);
    auto go = [&](auto kernel, int threads) {
        if (c) KGE_LAUNCH(c, kernel, grid, dim3(threads), 0, st, a);
        else hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, st, a);
    };
    if (n <= 256) go(k_distill<DT, 1, 1, WIDE, STEP>, 64);
    else if (n <= 1024) go(k_distill<DT, 4, 1, WIDE, STEP>, 256);
    else if (n <= 4096) go(k_distill<DT, 4, 4, WIDE, STEP>, 256);
    // (us, 16 / 1024 / 4096 rows of 5000, by the kernel for 16,384 -> by this: 9.6 -> 8.1 / 24 -> 19 / 76 -> 58)
    else if (n <= 8192) go(k_distill<DT, 8, 4, WIDE, STEP>, 512);
    // (us, 16 / 256 / 4096 rows of 15,000, 1024 threads -> these 512: 9.2 -> 9.8 / 11.7 -> 12.0 / 198 -> 116)
    else if (n <= 16384) go(k_distill<DT, 8, 8, WIDE, STEP>, 512);
    else go(k_distill<DT, 16, 8, WIDE, STEP>, 1024);
}

template <int DT>
void launch(const DistillArgs& a, hipStream_t st) {
    const bool wide = a.t.temperature > WIDE_TEMPERATURE;
    if (a.groups == 0) {
        if (wide) launch_rows<DT, true, false>(nullptr, a, st);
        else launch_rows<DT, false, false>(nullptr, a, st);
        return;
    }
    const dim3 grid = flat_grid(pieces(a.in.rows * a.groups, a.per)), rows = flat_grid(a.in.rows);
    if (wide) {
        k_distill_sums<DT, true><<<grid, 256, 0, st>>>(a);
        k_distill_finish<DT, true><<<rows, 256, 0, st>>>(a);
    } else {
        k_distill_sums<DT, false><<<grid, 256, 0, st>>>(a);
        k_distill_finish<DT, false><<<rows, 256, 0, st>>>(a);
    }
    if (a.grad) k_distill_grad<DT><<<grid, 256, 0, st>>>(a);
}

}  // namespace

int64_t kge_distill_workspace(int64_t rows, int64_t n) {
    if (n <= KGE_ROW_RESIDENT) return 0;
    return up256(rows * pieces(n, GROUP) * 16) + up256(rows * (int64_t)sizeof(RowGrad));
}

void kge_launch_distill(const RowScores& in, const TeacherLists& t, float grad_scale, float loss_scale, float* loss, void* grad, int64_t ld_grad,
                        const StepRows* step, void* workspace, hipStream_t st) {
    DistillArgs a = {};
    a.in = in; a.t = t;
    a.inv_t = 1.0 / (double)t.temperature;
    a.grad_scale = (double)grad_scale * (double)t.temperature;
    a.loss_scale = (double)loss_scale * (double)t.temperature * (double)t.temperature;
    a.loss = loss; a.grad = grad; a.ld_grad = ld_grad;
    if (step) {
        a.step = *step;
        if (t.temperature > WIDE_TEMPERATURE) launch_rows<KGE_F32, true, true>(step->c, a, st);
        else launch_rows<KGE_F32, false, true>(step->c, a, st);
        return;
    }
    if (in.n > KGE_ROW_RESIDENT) {
        a.groups = pieces(in.n, GROUP);
        a.per = groups_per_workgroup(in.rows * a.groups);
        a.sums = static_cast<double*>(workspace);
        a.rows = reinterpret_cast<RowGrad*>(static_cast<char*>(workspace) + up256(in.rows * a.groups * 16));
    }
    if (in.dtype == KGE_F32) launch<KGE_F32>(a, st);
    else if (in.dtype == KGE_BF16) launch<KGE_BF16>(a, st);
    else launch<KGE_F16>(a, st);
}
