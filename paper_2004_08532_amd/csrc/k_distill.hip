// Divergence of rows of scores from a teacher's lists of best candidates, and its gradient (kge_distill_loss, kge_distill_step).
//
// With z = s / T, w_j = exp(z_j - max z), Z = sum w, q_j = w_j / Z and the teacher's p_e over the entries e of a row's list:
//     loss   = T^2 [ sum_e p_e log(p_e / q_{id_e})  +  p_r log(p_r / q_r) ]
//     grad_j = c T [ P q_j - sum_{e: id_e = j} p_e ]   listed candidates, and all where the lists are all there is
//     grad_j = c T [ P - p_r Z / Z_r ] q_j             candidates that are not listed, where there is a rest
// p_r = 1 - sum p is the mass that the teacher has outside of the list, q_r = Z_r / Z the student's, P = sum p + p_r.
//
// A row is read once and its gradient written once: the weights stay in registers between the sum and the gradient.  Long
// rows are cut: one launch sums, a second one reads the row again.  What a list adds is little beside its row; its exponentials
// and everything that is a difference of near values (logarithms of the loss, the rest) are formed in 64 bits.
#include "k_rows.h"

namespace {

struct DistillArgs {
    RowScores in;
    TeacherLists t;
    double inv_t;
    float grad_scale, loss_scale;  // loss_scale: T^2, and 1 / b in a step
    float* loss;
    void* grad;
    int64_t ld_grad;
    StepRows step;
    int segments;
    double* parts;  // [rows][segments][3]: best score, Z and Z_r relative to it
    double* lists;  // [rows][4]: see ListSums
};

struct ListSums {
    double mass;      // sum p
    double rest;      // p_r, 0 without one
    double cross;     // sum_e p_e (log p_e - s_e / T)
    double shift;     // p_e = exp(t_e / T - shift)
};

// Weight of a score relative to the largest of its row, which is finite (or NaN comes out).  The argument of the exponential is
// formed in 64 bits and its fraction taken in 32: the weight is off by the roundings of exp2 alone, whatever the distance.
__device__ __forceinline__ float weight32(float s, double best, double scale /* log2(e) / T */) {
    const double x = ((double)s - best) * scale, n = rint(x);
    const float e = __builtin_amdgcn_exp2f((float)(x - n));
    return s > -INFINITY || s != s ? ldexpf(e, (int)fmax(n, -400.0)) : 0.f;
}

template <int DT> struct RowAt {
    const typename Score<DT>::type* s;
    int64_t n;
    bool is_dist;
    float gamma;
    __device__ __forceinline__ float of(float raw) const { return is_dist ? gamma - raw : raw; }
    __device__ __forceinline__ float at(int64_t j) const { return of(widen<DT>(s[j])); }
};

// Sums over a row's list, by a workgroup.
template <int DT, int WAVES>
__device__ __forceinline__ ListSums sum_list(const DistillArgs& a, int64_t row, const RowAt<DT>& r, double* slot) {
    const int64_t* ids = a.t.ids + row * a.t.m;
    const float* ts = a.t.scores + row * a.t.m;
    auto used = [&](int e) { return ids[e] >= 0 && ids[e] < r.n && !(ts[e] == -INFINITY); };
    ListSums l;
    if (a.t.lse) {
        l.shift = (double)a.t.lse[row];
    } else {
        float best = -INFINITY;
        for (int e = threadIdx.x; e < a.t.m; e += WAVES * 64) if (used(e)) best = fmaxf(best, ts[e]);
        best = block_max<WAVES>(best, reinterpret_cast<float*>(slot));
        l.shift = best > -INFINITY ? (double)best * a.inv_t : 0.0;
        double z = 0.0;
        for (int e = threadIdx.x; e < a.t.m; e += WAVES * 64) if (used(e)) z += exp((double)ts[e] * a.inv_t - l.shift);
        z = block_sum64<WAVES>(z, slot);
        if (z > 0.0 || z != z) l.shift += log(z);
    }
    double mass = 0.0, cross = 0.0;
    for (int e = threadIdx.x; e < a.t.m; e += WAVES * 64) {
        if (!used(e)) continue;
        const double lp = (double)ts[e] * a.inv_t - l.shift, p = exp(lp);
        mass += p;
        cross += p > 0.0 || p != p ? p * (lp - (double)r.at(ids[e]) * a.inv_t) : 0.0;
    }
    l.mass = block_sum64<WAVES>(mass, slot);
    l.cross = block_sum64<WAVES>(cross, slot);
    l.rest = a.t.lse ? fmax(1.0 - l.mass, 0.0) : 0.0;
    return l;
}

struct RowSums { double best, z, rest; };  // best score; sum of all weights, and of those that are not listed

// What the gradients of a row have in common: w * (listed or other) - p * unit
struct RowGrad { double best; float listed, other, unit; };

__device__ __forceinline__ RowGrad row_grad(const DistillArgs& a, const RowSums& s, ListSums& l, double& loss) {
    if (!(s.rest > 0.0)) l.rest = 0.0;  // no candidate that the rest could go to
    const double mass = l.mass + l.rest;
    loss = 0.0;
    RowGrad g = {s.best, 0.f, 0.f, 0.f};
    if (s.z != 0.0 && mass != 0.0) {
        const double c = (double)a.grad_scale;
        loss = l.cross + l.mass * (s.best * a.inv_t + log(s.z));
        if (l.rest > 0.0) loss += l.rest * log(l.rest * s.z / s.rest);
        g.listed = (float)(c * mass / s.z);
        g.other = l.rest > 0.0 ? (float)(c * (mass / s.z - l.rest / s.rest)) : g.listed;
        g.unit = (float)c;
    }
    return g;
}

template <int DT>
__device__ __forceinline__ void store4(typename Score<DT>::type* row, int64_t j, int64_t n, const float v[4]) {
    if (j + 4 <= n) {
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
        for (int q = 0; q < 4; ++q) if (j + q < n) row[j + q] = narrow<DT>(v[q]);
    }
}

enum { WHOLE_ROW, SEGMENT_SUMS, SEGMENT_GRAD };

template <int DT, int WAVES, int TPW, int PASS, bool STEP>
__global__ __launch_bounds__(WAVES * 64) void k_distill(DistillArgs a) {
    constexpr int CAP = WAVES * TPW * 256, THREADS = WAVES * 64, N = TPW * 4;
    constexpr bool GRAD = PASS != SEGMENT_SUMS;
    __shared__ uint32_t listed[CAP / 32];  // a bit per candidate of this row (segment)
    __shared__ int32_t list_at[GRAD ? KGE_TOP_MAX : 1];
    __shared__ float list_grad[GRAD ? KGE_TOP_MAX : 1];
    __shared__ double slot[WAVES];
    __shared__ int twice;  // a candidate is listed more than once
    const int64_t block = flat_block();
    if (block >= a.in.rows * a.segments) return;
    const int64_t row = PASS == WHOLE_ROW ? block : block / a.segments, seg = block - row * a.segments, first = seg * CAP;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    RowAt<DT> r;
    r.s = static_cast<const typename Score<DT>::type*>(a.in.p) + row * a.in.ld;
    r.n = a.in.n;
    r.is_dist = STEP && a.step.is_dist; r.gamma = STEP ? a.step.gamma : 0.f;

    float v[N];
    float best = -INFINITY;
#pragma unroll
    for (int i = 0; i < TPW; ++i) {
        const int64_t tile = first + (int64_t)(i * WAVES + wave) * 256;
        Quad<DT> x;
        x.load(r.s, tile + lane * 4, r.n);
        x.template values<false>(tile, r.n, v + 4 * i);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if constexpr (STEP) { if (tile + lane * 4 + q < r.n) v[4 * i + q] = r.of(v[4 * i + q]); }
            best = fmaxf(best, v[4 * i + q]);
        }
    }
    for (int x = threadIdx.x; x < CAP / 32; x += THREADS) listed[x] = 0;
    if (threadIdx.x == 0) twice = 0;
    __syncthreads();
    // the list's candidates among these
    const int64_t* ids = a.t.ids + row * a.t.m;
    const float* ts = a.t.scores + row * a.t.m;
    for (int e = threadIdx.x; e < a.t.m; e += THREADS) {
        const int64_t id = ids[e], at = id - first;
        const bool in = id >= first && id < r.n && at < CAP && ts[e] != -INFINITY;
        if (in) {
            const uint32_t bit = 1u << (at & 31);
            if (atomicOr(&listed[at >> 5], bit) & bit) twice = 1;
        }
        if constexpr (GRAD) list_at[e] = in ? (int)at : -1;
    }
    ListSums l = {};
    if (PASS == WHOLE_ROW || (PASS == SEGMENT_SUMS && seg == 0)) l = sum_list<DT, WAVES>(a, row, r, slot);

    const double scale = a.inv_t * 1.4426950408889634;
    RowSums s = {};
    if constexpr (PASS == SEGMENT_GRAD) {
        const double* p = a.parts + 3 * row * a.segments;
        float best = -INFINITY;
        for (int g = threadIdx.x; g < a.segments; g += THREADS) best = fmaxf(best, (float)p[3 * g]);
        const double top = (double)block_max<WAVES>(best, reinterpret_cast<float*>(slot));
        for (int g = threadIdx.x; g < a.segments; g += THREADS) {
            if (p[3 * g + 1] == 0.0) continue;
            const double w = p[3 * g] == top ? 1.0 : exp((p[3 * g] - top) * a.inv_t);
            s.z += p[3 * g + 1] * w;
            s.rest += p[3 * g + 2] * w;
        }
        s.best = top;
        const double* q = a.lists + 4 * row;
        l.mass = q[0]; l.rest = q[1]; l.cross = q[2]; l.shift = q[3];
    } else {
        s.best = (double)block_max<WAVES>(best, reinterpret_cast<float*>(slot));
    }
#pragma unroll
    for (int i = 0; i < TPW; ++i) {
        const int at = (i * WAVES + wave) * 256 + lane * 4;
        const uint32_t bits = a.t.lse ? listed[at >> 5] >> (at & 31) : 0u;
        float z = 0.f, zr = 0.f;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            v[4 * i + q] = weight32(v[4 * i + q], s.best, scale);
            z += v[4 * i + q];
            zr += bits >> q & 1 ? 0.f : v[4 * i + q];
        }
        if constexpr (PASS != SEGMENT_GRAD) {
            s.z += (double)z;
            s.rest += (double)zr;
        }
    }
    s.z = block_sum64<WAVES>(s.z, slot);
    s.rest = a.t.lse ? block_sum64<WAVES>(s.rest, slot) : 0.0;

    if constexpr (PASS == SEGMENT_SUMS) {
        if (threadIdx.x == 0) {
            double* p = a.parts + 3 * block;
            p[0] = s.best; p[1] = s.z; p[2] = s.rest;
            if (seg == 0) {
                double* q = a.lists + 4 * row;
                q[0] = l.mass; q[1] = l.rest; q[2] = l.cross; q[3] = l.shift;
            }
        }
        return;
    }
    if constexpr (GRAD) {
        double loss;
        const RowGrad g = row_grad(a, s, l, loss);
        if (threadIdx.x == 0 && seg == 0 && a.loss) a.loss[row] = (float)(loss * (double)a.loss_scale);
        if constexpr (STEP) { if (threadIdx.x == 0) a.step.cpos[row] = 0.f; }
        if (!a.grad) return;
        auto* out = static_cast<typename Score<DT>::type*>(a.grad) + row * a.ld_grad + first;
        const auto* in = r.s + first;
        auto shape = [&](float x, float raw) {  // a gradient as the backward products of a step want it
            if constexpr (STEP) {
                if (r.is_dist) x = raw > 0.f ? x / raw : 0.f;
                if (a.step.bf16) x = round_bf16(x);
            }
            return x;
        };
        auto p_of = [&](int e) { return exp((double)ts[e] * a.inv_t - l.shift); };
        auto stands = [&](int e) {  // the first entry of a candidate stands for all of them
            bool ok = true;
            if (twice) for (int x = 0; x < e; ++x) ok = ok && list_at[x] != list_at[e];
            return ok;
        };
        // the list's candidates: formed before any score is overwritten, stored behind the others
        for (int e = threadIdx.x; e < a.t.m; e += THREADS) {
            const int at = list_at[e];
            if (at < 0 || !stands(e)) continue;
            double p = p_of(e);
            if (twice) for (int x = e + 1; x < a.t.m; ++x) if (list_at[x] == at) p += p_of(x);
            const float raw = widen<DT>(in[at]);
            list_grad[e] = shape(fmaf(weight32(r.of(raw), s.best, scale), g.listed, -(float)p * g.unit), raw);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < TPW; ++i) {
            const int64_t tile = (int64_t)(i * WAVES + wave) * 256, j = tile + lane * 4;
            float x[4], raw[4] = {};
            if constexpr (STEP) {
                Quad<DT> again;
                again.load(in, j, r.n);
                again.template values<false>(tile, r.n, raw);
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) x[q] = shape(v[4 * i + q] * g.other, raw[q]);
            if (j < r.n - first) store4<DT>(out, j, r.n - first, x);
        }
        __syncthreads();
        for (int e = threadIdx.x; e < a.t.m; e += THREADS)
            if (list_at[e] >= 0 && stands(e)) out[list_at[e]] = narrow<DT>(list_grad[e]);
    }
}

// c: the context of a training step, whose launches are timed; null otherwise
template <int DT, bool STEP>
void launch_rows(kge_ctx* c, const DistillArgs& a, hipStream_t st) {
    const int64_t n = a.in.n;
    const dim3 grid = flat_grid(a.in.rows);
    auto go = [&](auto kernel, int threads) {
        if (c) KGE_LAUNCH(c, kernel, grid, dim3(threads), 0, st, a);
        else hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, st, a);
    };
    if (n <= 256) go(k_distill<DT, 1, 1, WHOLE_ROW, STEP>, 64);
    else if (n <= 1024) go(k_distill<DT, 4, 1, WHOLE_ROW, STEP>, 256);
    else if (n <= 4096) go(k_distill<DT, 4, 4, WHOLE_ROW, STEP>, 256);
    else if (n <= 16384) go(k_distill<DT, 16, 4, WHOLE_ROW, STEP>, 1024);
    else go(k_distill<DT, 16, 8, WHOLE_ROW, STEP>, 1024);
}

template <int DT>
void launch(const DistillArgs& a, hipStream_t st) {
    if (a.segments == 1) { launch_rows<DT, false>(nullptr, a, st); return; }
    const dim3 grid = flat_grid(a.in.rows * a.segments);
    k_distill<DT, 16, 4, SEGMENT_SUMS, false><<<grid, 1024, 0, st>>>(a);
    k_distill<DT, 16, 4, SEGMENT_GRAD, false><<<grid, 1024, 0, st>>>(a);
}

}  // namespace

int64_t kge_distill_workspace(int64_t rows, int64_t n) {
    if (n <= KGE_ROW_RESIDENT) return 0;
    return up256(rows * pieces(n, KGE_ROW_SEGMENT) * 24) + up256(rows * 32);
}

void kge_launch_distill(const RowScores& in, const TeacherLists& t, float grad_scale, float loss_scale, float* loss, void* grad, int64_t ld_grad,
                        const StepRows* step, void* workspace, hipStream_t st) {
    DistillArgs a = {};
    a.in = in; a.t = t;
    a.inv_t = 1.0 / (double)t.temperature;
    a.grad_scale = grad_scale * t.temperature;
    a.loss_scale = loss_scale * t.temperature * t.temperature;
    a.loss = loss; a.grad = grad; a.ld_grad = ld_grad;
    a.segments = in.n <= KGE_ROW_RESIDENT ? 1 : (int)pieces(in.n, KGE_ROW_SEGMENT);
    if (step) {
        a.step = *step;
        launch_rows<KGE_F32, true>(step->c, a, st);
        return;
    }
    if (a.segments > 1) {
        a.parts = static_cast<double*>(workspace);
        a.lists = reinterpret_cast<double*>(static_cast<char*>(workspace) + up256(in.rows * a.segments * 24));
    }
    if (in.dtype == KGE_F32) launch<KGE_F32>(a, st);
    else if (in.dtype == KGE_BF16) launch<KGE_BF16>(a, st);
    else launch<KGE_F16>(a, st);
}
