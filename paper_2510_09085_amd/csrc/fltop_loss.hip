// Losses over the scores of hypotheses, with their gradients: pairs of hypotheses (log ratios of the
// better to the worse), and a clipped policy loss with a KL term.  Everything is fp64: the scores
// are, and there are few of them.
//
// A mean over what takes part needs its number before the gradient: one workgroup per utterance
// sums its own values, counts them and leaves the gradient unscaled; a second kernel adds the
// utterances' sums up (each of its workgroups all of them, in one order) and scales.
#include "fltop_learn.h"

namespace fltop {
namespace {

constexpr int kThreads = 256;
constexpr int kWave = 64;

// Sum over the workgroup in a fixed order; every thread gets it.
__device__ double block_sum(double x, double* scratch) {
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) x += __shfl_xor(x, o, kWave);
    __syncthreads();
    if ((threadIdx.x & (kWave - 1)) == 0) scratch[threadIdx.x / kWave] = x;
    __syncthreads();
    double s = 0.0;
    for (int w = 0; w < (int)blockDim.x / kWave; ++w) s += scratch[w];
    return s;
}

struct PairSums {
    double loss;
    double n;
};

// ln(1 + e^x)
__device__ inline double softplus(double x) { return fmax(x, 0.0) + log1p(exp(-fabs(x))); }

__global__ __launch_bounds__(kThreads) void preference_kernel(fltop_preference p, PairSums* sums) {
    extern __shared__ double shared[];
    __shared__ double scratch[kThreads / kWave];
    double* ratio = shared;           // [N] s - q
    const int32_t b = blockIdx.x;
    const double* s = p.scores + (int64_t)b * p.N;
    const double* q = p.ref_scores ? p.ref_scores + (int64_t)b * p.N : nullptr;
    for (int32_t n = threadIdx.x; n < p.N; n += kThreads) {
        const bool fine = isfinite(s[n]) && (!q || isfinite(q[n]));
        ratio[n] = fine ? (q ? s[n] - q[n] : s[n]) : NAN;
    }
    __syncthreads();
    int32_t count = p.pair_counts ? p.pair_counts[b] : p.M;
    count = count < 0 ? 0 : (count > p.M ? p.M : count);
    const int32_t* pairs = p.pairs + (int64_t)b * p.M * 2;
    double* margins = p.margins + (int64_t)b * p.M;
    double loss = 0.0, used = 0.0;
    for (int32_t m = threadIdx.x; m < p.M; m += kThreads) {
        double h = NAN;
        if (m < count) {
            const int32_t i = pairs[2 * m], j = pairs[2 * m + 1];
            if ((uint32_t)i < (uint32_t)p.N && (uint32_t)j < (uint32_t)p.N) h = ratio[i] - ratio[j];
        }
        margins[m] = h;
        if (h != h) continue;
        used += 1.0;
        const double x = p.beta * h;
        if (p.kind == FLTOP_PREFERENCE_SIGMOID)
            loss += (1.0 - p.label_smoothing) * softplus(-x) + p.label_smoothing * softplus(x);
        else if (p.kind == FLTOP_PREFERENCE_HINGE)
            loss += fmax(0.0, 1.0 - x);
        else
            loss += (h - 0.5 / p.beta) * (h - 0.5 / p.beta);
    }
    loss = block_sum(loss, scratch);
    used = block_sum(used, scratch);
    if (threadIdx.x == 0) sums[b] = {loss, used};
    // the margins are this workgroup's own writes: visible to it after the barriers in block_sum
    for (int32_t n = threadIdx.x; n < p.N; n += kThreads) {
        double d = 0.0;
        for (int32_t m = 0; m < count; ++m) {
            const int32_t i = pairs[2 * m], j = pairs[2 * m + 1];
            if ((i != n && j != n) || i == j) continue;
            const double h = margins[m];
            if (h != h) continue;
            const double x = p.beta * h;
            double g;
            if (p.kind == FLTOP_PREFERENCE_SIGMOID)
                g = p.beta * (1.0 / (1.0 + exp(-x)) - (1.0 - p.label_smoothing));
            else if (p.kind == FLTOP_PREFERENCE_HINGE)
                g = x < 1.0 ? -p.beta : 0.0;
            else
                g = 2.0 * (h - 0.5 / p.beta);
            d += i == n ? g : -g;
        }
        p.grad_scores[(int64_t)b * p.N + n] = d;
    }
}

__global__ __launch_bounds__(kThreads) void preference_mean_kernel(fltop_preference p, const PairSums* sums) {
    __shared__ double scratch[kThreads / kWave];
    double loss = 0.0, used = 0.0;
    for (int32_t b = threadIdx.x; b < p.B; b += kThreads) {
        loss += sums[b].loss;
        used += sums[b].n;
    }
    loss = block_sum(loss, scratch);
    used = block_sum(used, scratch);
    const double each = used > 0.0 ? 1.0 / used : 0.0;
    if (blockIdx.x == 0 && threadIdx.x == 0) *p.loss = loss * each;
    const int64_t total = (int64_t)p.B * p.N;
    for (int64_t i = blockIdx.x * (int64_t)kThreads + threadIdx.x; i < total; i += (int64_t)gridDim.x * kThreads)
        p.grad_scores[i] *= each * p.scale;
}

__global__ __launch_bounds__(kThreads) void policy_kernel(const double* scores, const double* old_scores,
                                                          const double* ref_scores, const double* advantages,
                                                          const int32_t* counts, int32_t N, fltop_policy p,
                                                          PolicySums* sums, double* grad_scores) {
    __shared__ double scratch[kThreads / kWave];
    const int32_t b = blockIdx.x;
    int32_t count = counts ? counts[b] : N;
    count = count > N ? N : count;
    PolicySums s = {0.0, 0.0, 0.0, 0.0};
    for (int32_t n = threadIdx.x; n < N; n += kThreads) {
        const int64_t at = (int64_t)b * N + n;
        double d = 0.0;
        if (n < count) {
            const double l = scores[at], o = old_scores[at], A = advantages[at];
            const double q = ref_scores ? ref_scores[at] : 0.0;
            if (isfinite(l) && isfinite(o) && isfinite(A) && isfinite(q))
                d = policy_entry(l, o, ref_scores != nullptr, q, A, p, &s);
        }
        grad_scores[at] = d;
    }
    s.loss = block_sum(s.loss, scratch);
    s.kl = block_sum(s.kl, scratch);
    s.clipped = block_sum(s.clipped, scratch);
    s.n = block_sum(s.n, scratch);
    if (threadIdx.x == 0) sums[b] = s;
}

// What a row's entries weigh, and the whole batch's results.
struct PolicyTotal {
    double loss, kl, clipped, n, rows;
};

__device__ PolicyTotal policy_total(const PolicySums* sums, int32_t B, int32_t reduction, double* scratch) {
    PolicyTotal t = {0.0, 0.0, 0.0, 0.0, 0.0};
    for (int32_t b = threadIdx.x; b < B; b += (int32_t)blockDim.x) {
        const PolicySums s = sums[b];
        if (s.n == 0.0) continue;
        const double w = reduction == FLTOP_REDUCE_SEQUENCE ? 1.0 / s.n : 1.0;
        t.loss += s.loss * w;
        t.kl += s.kl * w;
        t.clipped += s.clipped;
        t.n += s.n;
        t.rows += 1.0;
    }
    t.loss = block_sum(t.loss, scratch);
    t.kl = block_sum(t.kl, scratch);
    t.clipped = block_sum(t.clipped, scratch);
    t.n = block_sum(t.n, scratch);
    t.rows = block_sum(t.rows, scratch);
    const double by = t.n == 0.0                          ? 0.0
                      : reduction == FLTOP_REDUCE_TOKEN    ? 1.0 / t.n
                      : reduction == FLTOP_REDUCE_SEQUENCE ? 1.0 / t.rows
                                                           : 1.0;
    t.loss *= by;
    t.kl *= by;
    t.clipped *= t.n == 0.0 ? 0.0 : 1.0 / t.n;
    return t;
}

__device__ inline double policy_weight(double n, const PolicyTotal& t, int32_t reduction) {
    if (n == 0.0) return 0.0;
    if (reduction == FLTOP_REDUCE_TOKEN) return 1.0 / t.n;
    if (reduction == FLTOP_REDUCE_SEQUENCE) return 1.0 / (n * t.rows);
    return 1.0;
}

__global__ __launch_bounds__(kThreads) void policy_mean_kernel(const PolicySums* sums, int32_t B, int32_t N,
                                                               fltop_policy p, double* summary, double* grad_scores) {
    __shared__ double scratch[kThreads / kWave];
    const PolicyTotal t = policy_total(sums, B, p.reduction, scratch);
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        summary[0] = t.loss;
        summary[1] = t.kl;
        summary[2] = t.clipped;
    }
    const int64_t total = (int64_t)B * N;
    for (int64_t i = blockIdx.x * (int64_t)kThreads + threadIdx.x; i < total; i += (int64_t)gridDim.x * kThreads)
        grad_scores[i] *= policy_weight(sums[i / N].n, t, p.reduction) * p.scale;
}

unsigned blocks_for(int64_t n) {
    const int64_t blocks = (n + kThreads - 1) / kThreads;
    return (unsigned)(blocks < 1024 ? blocks : 1024);
}

}  // namespace

hipError_t launch_preference(const fltop_preference& p, void* workspace, hipStream_t stream) {
    PairSums* sums = static_cast<PairSums*>(workspace);
    hipLaunchKernelGGL(preference_kernel, dim3(p.B), dim3(kThreads), (size_t)p.N * sizeof(double), stream, p, sums);
    hipLaunchKernelGGL(preference_mean_kernel, dim3(blocks_for((int64_t)p.B * p.N)), dim3(kThreads), 0, stream, p, sums);
    return hipGetLastError();
}

hipError_t launch_policy(const double* scores, const double* old_scores, const double* ref_scores,
                         const double* advantages, const int32_t* counts, int32_t B, int32_t N,
                         const fltop_policy& policy, void* workspace, double* summary, double* grad_scores,
                         hipStream_t stream) {
    PolicySums* sums = static_cast<PolicySums*>(workspace);
    hipLaunchKernelGGL(policy_kernel, dim3(B), dim3(kThreads), 0, stream, scores, old_scores, ref_scores, advantages,
                       counts, N, policy, sums, grad_scores);
    hipLaunchKernelGGL(policy_mean_kernel, dim3(blocks_for((int64_t)B * N)), dim3(kThreads), 0, stream, sums, B, N,
                       policy, summary, grad_scores);
    return hipGetLastError();
}

}  // namespace fltop
