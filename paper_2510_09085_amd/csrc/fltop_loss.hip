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

// Sums over what takes part of a row.
struct PolicySums {
    double loss, kl, clipped, n;
};

// One entry: adds to the row's sums and returns the loss's derivative to the log-probability.
__device__ inline double policy_entry(double l, double l_old, bool has_ref, double l_ref, double A,
                                      const fltop_policy& p, PolicySums* s) {
    const double r = exp(l - l_old);
    const double plain = r * A;
    const double cut = fmin(fmax(r, 1.0 - p.clip_low), 1.0 + p.clip_high) * A;
    const double gap = has_ref ? l_ref - l : 0.0;
    const double e = expm1(gap);
    const double kl = e - gap;
    s->loss += fmax(-plain, -cut) + p.kl_weight * kl;
    s->kl += kl;
    s->clipped += plain > cut ? 1.0 : 0.0;
    s->n += 1.0;
    return (plain <= cut ? -plain : 0.0) - p.kl_weight * e;
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

// ---- the policy loss from logits -----------------------------------------------------------------

__global__ __launch_bounds__(kThreads) void part_kernel(fltop_rows x, const int32_t* tokens, PolicySums* sums) {
    __shared__ double scratch[kThreads / kWave];
    const int32_t b = blockIdx.x;
    const int32_t frames = min(x.lengths[b], x.T);
    double n = 0.0;
    for (int32_t t = threadIdx.x; t < frames; t += kThreads)
        n += (uint32_t)tokens[(int64_t)b * x.T + t] < (uint32_t)x.V ? 1.0 : 0.0;
    n = block_sum(n, scratch);
    if (threadIdx.x == 0) sums[b] = {0.0, 0.0, 0.0, n};
}

template <typename T>
__global__ __launch_bounds__(kThreads) void policy_rows_kernel(fltop_rows x, const int32_t* tokens,
                                                               const float* old_logps, const float* ref_logps,
                                                               const float* advantages, bool per_frame,
                                                               fltop_policy p, const PolicySums* counted,
                                                               double* entries, float* logps, T* grad) {
    __shared__ double scratch[kThreads / kWave];
    __shared__ float tops[kThreads / kWave];
    const PolicyTotal total = policy_total(counted, x.B, p.reduction, scratch);
    const int64_t rows = (int64_t)x.B * x.T;
    for (int64_t at = blockIdx.x; at < rows; at += gridDim.x) {
        const int32_t b = (int32_t)(at / x.T), t = (int32_t)(at % x.T);
        T* out = grad + at * x.V;
        const int32_t tok = t < x.lengths[b] ? tokens[at] : -1;
        if ((uint32_t)tok >= (uint32_t)x.V) {
            for (int32_t v = threadIdx.x; v < x.V; v += kThreads) out[v] = from_float<T>(0.0f);
            if (threadIdx.x == 0) {
                logps[at] = 0.0f;
                entries[3 * at] = entries[3 * at + 1] = entries[3 * at + 2] = 0.0;
            }
            continue;
        }
        const T* row = static_cast<const T*>(x.data) + b * x.batch_stride + t * x.frame_stride;
        float top = -INFINITY;
        for (int32_t v = threadIdx.x; v < x.V; v += kThreads) top = fmaxf(top, to_float(row[v]));
#pragma unroll
        for (int o = kWave / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, kWave));
        __syncthreads();
        if ((threadIdx.x & (kWave - 1)) == 0) tops[threadIdx.x / kWave] = top;
        __syncthreads();
        for (int w = 0; w < kThreads / kWave; ++w) top = fmaxf(top, tops[w]);
        // the others' mass apart from the token's own: 1 - p and ln p keep their digits where p is nearly 1
        float rest = 0.0f;
        for (int32_t v = threadIdx.x; v < x.V; v += kThreads) rest += v == tok ? 0.0f : expf(to_float(row[v]) - top);
        const double others = block_sum((double)rest, scratch);
        const double gap = (double)to_float(row[tok]) - (double)top;
        const double own = exp(gap);
        const double sum = others + own;
        const double l = own > others ? -log1p(others / own) : gap - log(sum);
        PolicySums s = {0.0, 0.0, 0.0, 0.0};
        const double A = advantages[per_frame ? at : b];
        const double d = policy_entry(l, old_logps[at], ref_logps != nullptr, ref_logps ? ref_logps[at] : 0.0, A, p, &s) *
                         (policy_weight(counted[b].n, total, p.reduction) * p.scale);
        const float by = (float)(-d / sum);
        for (int32_t v = threadIdx.x; v < x.V; v += kThreads)
            out[v] = from_float<T>(v == tok ? (float)(d * (others / sum)) : expf(to_float(row[v]) - top) * by);
        if (threadIdx.x == 0) {
            logps[at] = (float)l;
            entries[3 * at] = s.loss;
            entries[3 * at + 1] = s.kl;
            entries[3 * at + 2] = s.clipped;
        }
    }
}

// The frames' losses of each utterance, then of the batch.
__global__ __launch_bounds__(kThreads) void policy_rows_sum_kernel(int32_t T, const double* entries, PolicySums* sums) {
    __shared__ double scratch[kThreads / kWave];
    const int32_t b = blockIdx.x;
    double s[3] = {0.0, 0.0, 0.0};
    for (int32_t t = threadIdx.x; t < T; t += kThreads)
        for (int k = 0; k < 3; ++k) s[k] += entries[3 * ((int64_t)b * T + t) + k];
    for (int k = 0; k < 3; ++k) s[k] = block_sum(s[k], scratch);
    if (threadIdx.x == 0) sums[b] = {s[0], s[1], s[2], sums[b].n};
}

__global__ __launch_bounds__(kThreads) void policy_summary_kernel(const PolicySums* sums, int32_t B, int32_t reduction,
                                                                  float* summary) {
    __shared__ double scratch[kThreads / kWave];
    const PolicyTotal t = policy_total(sums, B, reduction, scratch);
    if (threadIdx.x == 0) {
        summary[0] = (float)t.loss;
        summary[1] = (float)t.kl;
        summary[2] = (float)t.clipped;
    }
}

template <typename T>
hipError_t policy_rows(const fltop_rows& x, const int32_t* tokens, const float* old_logps, const float* ref_logps,
                       const float* advantages, bool per_frame, const fltop_policy& policy, void* workspace,
                       float* summary, float* logps, void* grad, hipStream_t stream) {
    PolicySums* sums = static_cast<PolicySums*>(workspace);
    double* entries = reinterpret_cast<double*>(static_cast<char*>(workspace) + policy_sums_bytes(x.B));
    hipLaunchKernelGGL(part_kernel, dim3(x.B), dim3(kThreads), 0, stream, x, tokens, sums);
    const int64_t rows = (int64_t)x.B * x.T;
    hipLaunchKernelGGL(policy_rows_kernel<T>, dim3((unsigned)(rows < 4096 ? rows : 4096)), dim3(kThreads), 0, stream, x,
                       tokens, old_logps, ref_logps, advantages, per_frame, policy, sums, entries, logps,
                       static_cast<T*>(grad));
    hipLaunchKernelGGL(policy_rows_sum_kernel, dim3(x.B), dim3(kThreads), 0, stream, x.T, entries, sums);
    hipLaunchKernelGGL(policy_summary_kernel, dim3(1), dim3(kThreads), 0, stream, sums, x.B, policy.reduction, summary);
    return hipGetLastError();
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

hipError_t launch_policy_logits(const fltop_rows& x, const int32_t* tokens, const float* old_logps,
                                const float* ref_logps, const float* advantages, bool per_frame,
                                const fltop_policy& policy, void* workspace, float* summary, float* logps, void* grad,
                                hipStream_t stream) {
    if (x.type == FLTOP_TYPE_BF16)
        return policy_rows<__hip_bfloat16>(x, tokens, old_logps, ref_logps, advantages, per_frame, policy, workspace,
                                           summary, logps, grad, stream);
    if (x.type == FLTOP_TYPE_F16)
        return policy_rows<__half>(x, tokens, old_logps, ref_logps, advantages, per_frame, policy, workspace, summary,
                                   logps, grad, stream);
    return policy_rows<float>(x, tokens, old_logps, ref_logps, advantages, per_frame, policy, workspace, summary, logps,
                              grad, stream);
}

}  // namespace fltop
