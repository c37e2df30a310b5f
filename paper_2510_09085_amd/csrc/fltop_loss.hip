// Losses over the scores of hypotheses, with their gradients: pairs of hypotheses (log ratios of the
// better to the worse), and a clipped policy loss with a KL term.  Everything is fp64: the scores
// are, and there are few of them.
//
// A mean over what takes part needs its number before the gradient.  Small batches are one workgroup's, in one launch (64
// pairs: 4.6 us, nearly all of it latency; 256 x 32 scores of a policy: 10.5 us in two launches, 18 by one workgroup).
// Else one workgroup per utterance sums its own values, counts them and leaves the gradient unscaled; a second kernel adds
// the utterances' sums up (each of its workgroups all of them, in one order) and scales.
//
// A hypothesis may be in many pairs: its derivatives are added in LDS as whole multiples of 2^-50 of its utterance's largest
// one (of 2^-S, S less, for lists of 2^11 pairs and more), so that the order in which threads add does not matter.  The
// one workgroup of a small batch keeps its pairs' derivatives in registers while the largest are found, each utterance's
// for itself.  Longer lists: a pair's derivative grows with its margin for each kind of loss, so the largest one is that
// of the smallest or of the largest margin, a first pass over the pairs makes the margins, a second one the rest.
#include "fltop_learn.h"

namespace fltop {
namespace {

constexpr int kThreads = 256;
constexpr int kWave = 64;
constexpr int kOneThreads = 1024;    // of the one workgroup that takes a small batch
constexpr int32_t kOneScores = 2048, kOnePairs = 4096, kOneEntries = 2048;

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

__device__ inline double block_most(double x, double* scratch) {
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) x = fmax(x, __shfl_xor(x, o, kWave));
    __syncthreads();
    if ((threadIdx.x & (kWave - 1)) == 0) scratch[threadIdx.x / kWave] = x;
    __syncthreads();
    double s = scratch[0];
    for (int w = 1; w < (int)blockDim.x / kWave; ++w) s = fmax(s, scratch[w]);
    return s;
}

// A pair's margin, loss and derivative; whether it takes part.
__device__ inline bool pair_loss(const fltop_preference& p, double h, double* loss, double* slope) {
    if (!isfinite(h)) return false;
    const double x = p.beta * h;
    if (p.kind == FLTOP_PREFERENCE_SIGMOID) {
        const double e = exp(-fabs(x)), l = log1p(e);
        // ln(1 + e^-x) and ln(1 + e^x), sigma(x)
        *loss = (1.0 - p.label_smoothing) * (fmax(-x, 0.0) + l);
        if (p.label_smoothing > 0.0) *loss += p.label_smoothing * (fmax(x, 0.0) + l);   // (x may be infinite)
        // sigma(x) - (1 - label_smoothing), without cancellation where nothing is smoothed
        *slope = p.beta * (p.label_smoothing - (x >= 0.0 ? e : 1.0) / (1.0 + e));
    } else if (p.kind == FLTOP_PREFERENCE_HINGE) {
        *loss = fmax(0.0, 1.0 - x);
        *slope = x < 1.0 ? -p.beta : 0.0;
    } else {
        const double d = h - 0.5 / p.beta;
        *loss = d * d;
        *slope = fmin(fmax(2.0 * d, -1.7e308), 1.7e308);
    }
    return true;
}

__device__ inline double slope_of(const fltop_preference& p, double h) {
    double f, g;
    return pair_loss(p, h, &f, &g) ? fabs(g) : 0.0;
}

constexpr double kShift = 6755399441055744.0;   // 1.5 * 2^52: its last bit is worth one

// How derivatives are kept as whole numbers: g as g * to, and back.
struct Steps {
    double to, back;
    __device__ Steps(double most, int32_t M) {
        const int bits = min(50, 61 - (32 - __clz(M)));
        most = fmax(most, 1e-290);   // `to` stays finite
        to = ldexp(1.0, bits) / most;
        back = ldexp(most, -bits);
    }
    __device__ unsigned long long whole(double g) const {
        return (unsigned long long)(__double_as_longlong(g * to + kShift) - __double_as_longlong(kShift));
    }
    __device__ double value(unsigned long long sum) const { return (double)(long long)sum * back; }
};

// Log ratio of a hypothesis to its reference, NaN if it takes no part.
__device__ inline double log_ratio(const fltop_preference& p, int64_t at) {
    const double s = p.scores[at], q = p.ref_scores ? p.ref_scores[at] : 0.0;
    return isfinite(s) && isfinite(q) ? s - q : NAN;
}

__device__ inline int32_t pairs_of(const fltop_preference& p, int32_t b) {
    const int32_t count = p.pair_counts ? p.pair_counts[b] : p.M;
    return count < 0 ? 0 : (count > p.M ? p.M : count);
}

__device__ inline int2 pair_at(const int32_t* list, int64_t m) {
    int2 pair;
    __builtin_memcpy(&pair, list + 2 * m, sizeof(pair));
    return pair;
}

// A pair's margin from the log ratios of its utterance, NaN if it takes no part.
__device__ inline double margin_of(const fltop_preference& p, const double* ratio, int2 pair, bool there) {
    const bool fine = there && (uint32_t)pair.x < (uint32_t)p.N && (uint32_t)pair.y < (uint32_t)p.N;
    const double h = fine ? ratio[pair.x] - ratio[pair.y] : NAN;
    return isfinite(h) ? h : NAN;
}

// A small batch in one workgroup.  LDS holds the log ratios, their derivatives' sums, and each utterance's largest
// derivative (as bits: those of numbers from 0 up are ordered as they are).
__global__ __launch_bounds__(kOneThreads) void preference_one_kernel(fltop_preference p) {
    extern __shared__ double shared[];
    __shared__ double scratch[kOneThreads / kWave];
    constexpr int kEach = kOnePairs / kOneThreads;
    const int32_t count = p.B * p.N, pairs = p.B * p.M;
    double* const ratio = shared;
    unsigned long long* const slopes = reinterpret_cast<unsigned long long*>(shared + count);
    unsigned long long* const most = slopes + count;
    int2 pair[kEach];
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const int32_t m = k * kOneThreads + threadIdx.x;
        pair[k] = m < pairs ? pair_at(p.pairs, m) : int2{0, 0};
    }
    for (int32_t i = threadIdx.x; i < count; i += kOneThreads) {
        ratio[i] = log_ratio(p, i);
        slopes[i] = 0;
    }
    for (int32_t b = threadIdx.x; b < p.B; b += kOneThreads) most[b] = 0;
    __syncthreads();
    double loss = 0.0, used = 0.0, slope[kEach];
    int32_t of[kEach];   // the pair's utterance, -1 if it takes no part
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const int32_t m = k * kOneThreads + threadIdx.x, b = (uint32_t)m / (uint32_t)p.M;
        of[k] = -1;
        if (m >= pairs) continue;
        const double h = margin_of(p, ratio + b * p.N, pair[k], m - b * p.M < pairs_of(p, b));
        p.margins[m] = h;
        double f;
        if (!pair_loss(p, h, &f, &slope[k])) continue;
        loss += f;
        used += 1.0;
        of[k] = b;
        atomicMax(&most[b], (unsigned long long)__double_as_longlong(fabs(slope[k])));
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const int32_t b = of[k];
        if (b < 0) continue;
        const unsigned long long whole = Steps(__longlong_as_double((long long)most[b]), p.M).whole(slope[k]);
        atomicAdd(&slopes[b * p.N + pair[k].x], whole);
        atomicAdd(&slopes[b * p.N + pair[k].y], 0ull - whole);
    }
    loss = block_sum(loss, scratch);
    used = block_sum(used, scratch);
    const double by = used > 0.0 ? p.scale / used : 0.0;
    if (threadIdx.x == 0) *p.loss = used > 0.0 ? loss / used : 0.0;
    for (int32_t i = threadIdx.x; i < count; i += kOneThreads) {
        const Steps steps(__longlong_as_double((long long)most[(uint32_t)i / (uint32_t)p.N]), p.M);
        p.grad_scores[i] = steps.value(slopes[i]) * by;
    }
}

// A workgroup for each utterance.  LDS holds its log ratios and their derivatives' sums.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void preference_kernel(fltop_preference p, PairSums* sums) {
    extern __shared__ double shared[];
    __shared__ double scratch[THREADS / kWave];
    const int32_t b = blockIdx.x;
    double* const ratio = shared;
    unsigned long long* const slopes = reinterpret_cast<unsigned long long*>(shared + p.N);
    for (int32_t i = threadIdx.x; i < p.N; i += THREADS) {
        ratio[i] = log_ratio(p, (int64_t)b * p.N + i);
        slopes[i] = 0;
    }
    __syncthreads();
    const int32_t* const list = p.pairs + (int64_t)b * p.M * 2;
    double* const margins = p.margins + (int64_t)b * p.M;
    const int32_t there = pairs_of(p, b);
    double high = -INFINITY, low = INFINITY;
#pragma unroll 4
    for (int32_t m = threadIdx.x; m < p.M; m += THREADS) {
        const double h = margin_of(p, ratio, pair_at(list, m), m < there);
        margins[m] = h;
        high = fmax(high, h);   // (NaN is passed over)
        low = fmin(low, h);
    }
    high = block_most(high, scratch);
    low = -block_most(-low, scratch);
    const Steps steps(fmax(slope_of(p, high), slope_of(p, low)), p.M);
    double loss = 0.0, used = 0.0;
#pragma unroll 4
    for (int32_t m = threadIdx.x; m < p.M; m += THREADS) {
        const double h = margins[m];
        const int2 pair = pair_at(list, m);
        double f, g;
        if (!pair_loss(p, h, &f, &g)) continue;
        loss += f;
        used += 1.0;
        const unsigned long long whole = steps.whole(g);
        atomicAdd(&slopes[pair.x], whole);
        atomicAdd(&slopes[pair.y], 0ull - whole);
    }
    loss = block_sum(loss, scratch);
    used = block_sum(used, scratch);
    if (threadIdx.x == 0) sums[b] = {loss, used};
    for (int32_t i = threadIdx.x; i < p.N; i += THREADS) p.grad_scores[(int64_t)b * p.N + i] = steps.value(slopes[i]);
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
    const double by = used > 0.0 ? p.scale / used : 0.0;
    if (blockIdx.x == 0 && threadIdx.x == 0) *p.loss = used > 0.0 ? loss / used : 0.0;
    const int64_t total = (int64_t)p.B * p.N;
    for (int64_t i = blockIdx.x * (int64_t)kThreads + threadIdx.x; i < total; i += (int64_t)gridDim.x * kThreads)
        p.grad_scores[i] *= by;
}

// An entry's numbers, and whether it takes part.
struct Entry {
    double l, old, ref, A;
    bool part;
    __device__ Entry(const double* scores, const double* old_scores, const double* ref_scores, const double* advantages,
                     int64_t at, bool there) {
        l = old = ref = A = 0.0;
        if (there) {
            l = scores[at];
            old = old_scores[at];
            A = advantages[at];
            if (ref_scores) ref = ref_scores[at];
        }
        part = there && isfinite(l) && isfinite(old) && isfinite(A) && isfinite(ref);
    }
};

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
        const Entry e(scores, old_scores, ref_scores, advantages, at, n < count);
        grad_scores[at] = e.part ? policy_entry(e.l, e.old, ref_scores != nullptr, e.ref, e.A, p, &s) : 0.0;
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

// A small batch in one workgroup: rows' numbers in LDS, then the entries.
__global__ __launch_bounds__(kOneThreads) void policy_one_kernel(const double* scores, const double* old_scores,
                                                                 const double* ref_scores, const double* advantages,
                                                                 const int32_t* counts, int32_t B, int32_t N,
                                                                 fltop_policy p, double* summary, double* grad_scores) {
    __shared__ int32_t numbers[kOneEntries];
    __shared__ double scratch[kOneThreads / kWave];
    constexpr int kEach = kOneEntries / kOneThreads;
    const int32_t total = B * N;
    for (int32_t b = threadIdx.x; b < B; b += kOneThreads) numbers[b] = 0;
    __syncthreads();
    double d[kEach];
    int32_t row[kEach];
    PolicySums mine[kEach];
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const int32_t at = k * kOneThreads + threadIdx.x, b = (uint32_t)at / (uint32_t)N;
        row[k] = at < total ? b : -1;
        const bool there = at < total && at - b * N < (counts ? counts[b] : N);
        const Entry e(scores, old_scores, ref_scores, advantages, at, there);
        mine[k] = {0.0, 0.0, 0.0, 0.0};
        d[k] = e.part ? policy_entry(e.l, e.old, ref_scores != nullptr, e.ref, e.A, p, &mine[k]) : 0.0;
        if (e.part) atomicAdd(&numbers[b], 1);
    }
    __syncthreads();
    PolicyTotal t = {0.0, 0.0, 0.0, 0.0, 0.0};
    for (int32_t b = threadIdx.x; b < B; b += kOneThreads) {
        t.n += numbers[b];
        t.rows += numbers[b] > 0 ? 1.0 : 0.0;
    }
    t.n = block_sum(t.n, scratch);
    t.rows = block_sum(t.rows, scratch);
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const double weight = row[k] >= 0 ? policy_weight(numbers[row[k]], t, p.reduction) : 0.0;
        if (mine[k].n > 0.0) {
            t.loss += mine[k].loss * weight;
            t.kl += mine[k].kl * weight;
            t.clipped += mine[k].clipped;
        }
        if (row[k] >= 0) grad_scores[k * kOneThreads + threadIdx.x] = mine[k].n > 0.0 ? d[k] * (weight * p.scale) : 0.0;
    }
    t.loss = block_sum(t.loss, scratch);
    t.kl = block_sum(t.kl, scratch);
    t.clipped = block_sum(t.clipped, scratch);
    if (threadIdx.x == 0) {
        summary[0] = t.loss;
        summary[1] = t.kl;
        summary[2] = t.n > 0.0 ? t.clipped / t.n : 0.0;
    }
}

unsigned blocks_for(int64_t n) {
    const int64_t blocks = (n + kThreads - 1) / kThreads;
    return (unsigned)(blocks < 1024 ? blocks : 1024);
}

}  // namespace

hipError_t launch_preference(const fltop_preference& p, void* workspace, hipStream_t stream) {
    PairSums* sums = static_cast<PairSums*>(workspace);
    const int64_t scores = (int64_t)p.B * p.N, pairs = (int64_t)p.B * p.M;
    if (scores <= kOneScores && pairs <= kOnePairs) {
        hipLaunchKernelGGL(preference_one_kernel, dim3(1), dim3(kOneThreads), (size_t)scores * 16 + (size_t)p.B * 8, stream,
                           p);
        return hipGetLastError();
    }
    // 128 utterances of 4950 pairs: 29 us with 256 threads, 20 us with 1024, about half of which are the exponentials and
    // logarithms of the 128 compute units in use.  (A launch has fewer than 2^32 threads.)
    if (p.M > kThreads * 2 && (int64_t)p.B * kOneThreads < (int64_t)1 << 32)
        hipLaunchKernelGGL((preference_kernel<kOneThreads>), dim3(p.B), dim3(kOneThreads), (size_t)p.N * 16, stream, p,
                           sums);
    else
        hipLaunchKernelGGL((preference_kernel<kThreads>), dim3(p.B), dim3(kThreads), (size_t)p.N * 16, stream, p, sums);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(preference_mean_kernel, dim3(blocks_for(scores)), dim3(kThreads), 0, stream, p, sums);
    return hipGetLastError();
}

hipError_t launch_policy(const double* scores, const double* old_scores, const double* ref_scores,
                         const double* advantages, const int32_t* counts, int32_t B, int32_t N,
                         const fltop_policy& policy, void* workspace, double* summary, double* grad_scores,
                         hipStream_t stream) {
    PolicySums* sums = static_cast<PolicySums*>(workspace);
    if ((int64_t)B * N <= kOneEntries) {
        hipLaunchKernelGGL(policy_one_kernel, dim3(1), dim3(kOneThreads), 0, stream, scores, old_scores, ref_scores, advantages,
                           counts, B, N, policy, summary, grad_scores);
        return hipGetLastError();
    }
    hipLaunchKernelGGL(policy_kernel, dim3(B), dim3(kThreads), 0, stream, scores, old_scores, ref_scores, advantages,
                       counts, N, policy, sums, grad_scores);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(policy_mean_kernel, dim3(blocks_for((int64_t)B * N)), dim3(kThreads), 0, stream, sums, B, N,
                       policy, summary, grad_scores);
    return hipGetLastError();
}

}  // namespace fltop
