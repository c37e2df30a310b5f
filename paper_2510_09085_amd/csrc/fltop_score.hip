// Log-probabilities of hypotheses under the emissions, summed over all alignments, and their
// gradient to the emissions.
//
// The lattice of a hypothesis y_1..y_L has the states blank_0 y_1 blank_1 .. y_L blank_L.  With
// b_i the mass of the alignments of the frames so far that end in blank_i and l_i of those that
// end in token y_{i+1},
//     b_i' = (b_i + l_{i-1}) p(blank)
//     l_i' = (l_i + b_i + [y_{i+1} != y_i] l_{i-1}) p(y_{i+1})
// from b_0 = 1 before the first frame, and P = b_L + l_{L-1} after the last.  Backwards the same
// holds for the reversed hypothesis over the reversed frames, and what stands in the brackets is
// then the mass of the frames after the present one, so that
//     P(pi_t = state) = forward mass after frame t * backward bracket at frame t / P.
#include "fltop_learn.h"

namespace fltop {
namespace {

constexpr int kThreads = 256;

// One hypothesis as the kernels see it: its tokens in lattice order or reversed.
struct Hyp {
    const int32_t* tokens;
    int32_t L;       // -1: not there, -2: longer than U
    int32_t frames;
};

__device__ inline Hyp hypothesis(const fltop_rows& x, const fltop_hypotheses& h, int32_t b, int32_t n) {
    Hyp y;
    const int32_t count = h.counts ? h.counts[b] : h.N;
    y.tokens = h.tokens + b * h.token_batch_stride + n * h.token_stride;
    y.L = n < count ? h.lengths[b * h.length_batch_stride + n] : -1;
    if (y.L < 0) y.L = -1;
    if (y.L > h.U) y.L = -2;
    const int32_t f = x.lengths[b];
    y.frames = f < 0 ? 0 : (f > x.T ? x.T : f);
    return y;
}

// The lattice of one hypothesis: thread t of 256 holds the pairs (b_i, l_i) for i = t K .. t K + K - 1,
// and only the last token's mass of each thread goes to its neighbour, through LDS.
template <int K>
struct Lattice {
    Mass b[K], l[K];
    int32_t tok[K];   // token of l_i, or 0 behind the last
    bool skip[K];     // y_{i+1} != y_i

    // Returns whether this thread's tokens are ones that an alignment can emit.
    __device__ bool start(const Hyp& y, int32_t V, bool reversed) {
        bool fine = true;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int32_t i = (int32_t)threadIdx.x * K + k;
            tok[k] = i < y.L ? y.tokens[reversed ? y.L - 1 - i : i] : 0;
            const int32_t before = i > 0 && i < y.L ? y.tokens[reversed ? y.L - i : i - 1] : 0;
            skip[k] = i > 0 && tok[k] != before;
            if (i < y.L && (tok[k] < 1 || tok[k] >= V)) {
                fine = false;
                tok[k] = 0;
            }
            b[k] = i == 0 ? unit_mass() : no_mass();
            l[k] = no_mass();
        }
        return fine;
    }

    // The brackets of the next frame; `left` is l_{i-1} of this thread's first pair.
    __device__ void brackets(Mass left, int32_t L) {
#pragma unroll
        for (int k = K - 1; k >= 0; --k) {
            const Mass in = k > 0 ? l[k > 0 ? k - 1 : 0] : left;
            const Mass stay = plus(l[k], b[k]);
            l[k] = skip[k] ? plus(stay, in) : stay;
            b[k] = plus(b[k], in);
            const int32_t i = (int32_t)threadIdx.x * K + k;
            l[k] = i < L ? normalized(l[k].m, l[k].e) : no_mass();
            b[k] = i <= L ? normalized(b[k].m, b[k].e) : no_mass();
        }
    }

    template <typename T>
    __device__ void emit(const T* row) {
        const Mass blank = mass_of(to_float(row[0]));
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const Mass p = mass_of(to_float(row[tok[k]]));
            l[k] = normalized(l[k].m * p.m, l[k].e + p.e);
            b[k] = normalized(b[k].m * blank.m, b[k].e + blank.e);
        }
    }
};

template <typename T, int K>
__global__ __launch_bounds__(kThreads) void score_kernel(fltop_rows x, fltop_hypotheses h, double* out_scores,
                                                         ScoreSpace ws, bool keep) {
    __shared__ Mass edge[2][kThreads + 1];
    __shared__ Mass ends[2];
    const int64_t at = blockIdx.x;
    const int32_t b = (int32_t)(at / h.N), n = (int32_t)(at % h.N);
    const Hyp y = hypothesis(x, h, b, n);
    Lattice<K> z;
    const bool fine = y.L >= 0 && z.start(y, x.V, false);
    if (__syncthreads_or(!fine)) {
        if (threadIdx.x == 0) {
            out_scores[at] = y.L == -2 ? NAN : -INFINITY;
            if (keep) ws.total_m[at] = 0.0, ws.total_e[at] = kNoMass;
        }
        return;
    }
    if (threadIdx.x == 0) edge[0][0] = edge[1][0] = no_mass();
    if (threadIdx.x < 2) ends[threadIdx.x] = no_mass();
    edge[1][threadIdx.x + 1] = z.l[K - 1];
    __syncthreads();
    const T* row = static_cast<const T*>(x.data) + b * x.batch_stride;
    for (int32_t t = 0; t < y.frames; ++t, row += x.frame_stride) {
        z.brackets(edge[(t + 1) & 1][threadIdx.x], y.L);
        z.emit(row);
        edge[t & 1][threadIdx.x + 1] = z.l[K - 1];
        if (keep) {
            Mass32* to = ws.rows + (at * x.T + t) * ws.row;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int32_t i = (int32_t)threadIdx.x * K + k;
                if (i <= y.L) to[i] = {(float)z.b[k].m, z.b[k].e};
                if (i < y.L) to[h.U + 1 + i] = {(float)z.l[k].m, z.l[k].e};
            }
        }
        __syncthreads();
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int32_t i = (int32_t)threadIdx.x * K + k;
        if (i == y.L) ends[0] = z.b[k];
        if (i == y.L - 1) ends[1] = z.l[k];
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        Mass p = plus(ends[0], ends[1]);
        p = normalized(p.m, p.e);
        out_scores[at] = ln_of(p);
        if (keep) ws.total_m[at] = p.m, ws.total_e[at] = p.e;
    }
}

template <typename T, int K>
__global__ __launch_bounds__(kThreads) void shares_kernel(fltop_rows x, fltop_hypotheses h, ScoreSpace ws) {
    __shared__ Mass edge[2][kThreads + 1];
    const int64_t at = blockIdx.x;
    const int32_t b = (int32_t)(at / h.N), n = (int32_t)(at % h.N);
    const double total = ws.total_m[at];
    const int32_t total_e = ws.total_e[at];
    if (total_e <= kNoMass) return;
    const Hyp y = hypothesis(x, h, b, n);
    Lattice<K> z;
    if (y.L < 0) return;
    z.start(y, x.V, true);
    if (threadIdx.x == 0) edge[0][0] = edge[1][0] = no_mass();
    edge[0][threadIdx.x + 1] = z.l[K - 1];
    __syncthreads();
    const T* rows = static_cast<const T*>(x.data) + b * x.batch_stride;
    for (int32_t t = y.frames - 1, turn = 0; t >= 0; --t, turn ^= 1) {
        z.brackets(edge[turn][threadIdx.x], y.L);
        const Mass32* from = ws.rows + (at * x.T + t) * ws.row;
        float* to = ws.shares + (at * x.T + t) * ws.row;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int32_t i = (int32_t)threadIdx.x * K + k;
            if (i <= y.L) {
                const Mass32 f = from[y.L - i];
                to[y.L - i] = (float)ldexp(f.m * z.b[k].m / total, f.e + z.b[k].e - total_e);
            }
            if (i < y.L) {
                const int32_t s = h.U + 1 + y.L - 1 - i;
                const Mass32 f = from[s];
                to[s] = (float)ldexp(f.m * z.l[k].m / total, f.e + z.l[k].e - total_e);
            }
        }
        z.emit(rows + t * x.frame_stride);
        edge[turn ^ 1][threadIdx.x + 1] = z.l[K - 1];
        __syncthreads();
    }
}

// One workgroup for each frame: occupancies into the frame's row of V sums, kept as whole numbers
// so that the order in which threads add does not matter.
template <typename T>
__global__ __launch_bounds__(kThreads) void score_grad_kernel(fltop_rows x, fltop_hypotheses h,
                                                              const double* grad_scores, ScoreSpace ws, T* grad) {
    extern __shared__ unsigned long long sums[];
    const int64_t frame = blockIdx.x;
    const int32_t b = (int32_t)(frame / x.T), t = (int32_t)(frame % x.T);
    T* out = grad + frame * x.V;
    const int32_t frames = x.lengths[b];
    if (t >= frames) {
        for (int32_t v = threadIdx.x; v < x.V; v += kThreads) out[v] = from_float<T>(0.0f);
        return;
    }
    double most = 0.0;
    bool odd = false;
    for (int32_t n = 0; n < h.N; ++n) {
        const int64_t at = (int64_t)b * h.N + n;
        if (ws.total_e[at] <= kNoMass) continue;
        const double w = fabs(grad_scores[at]);
        odd |= !(w <= 1.7976931348623157e308);
        most = fmax(most, w);
    }
    if (odd || most == 0.0) {
        for (int32_t v = threadIdx.x; v < x.V; v += kThreads) out[v] = from_float<T>(odd ? NAN : 0.0f);
        return;
    }
    for (int32_t v = threadIdx.x; v < x.V; v += kThreads) sums[v] = 0;
    __syncthreads();
    constexpr double kOne = 1125899906842624.0;       // 2^50
    constexpr double kShift = 6755399441055744.0;     // 1.5 * 2^52: its last bit is worth one
    for (int32_t n = 0; n < h.N; ++n) {
        const int64_t at = (int64_t)b * h.N + n;
        if (ws.total_e[at] <= kNoMass) continue;
        const double w = grad_scores[at] / most * kOne;
        const Hyp y = hypothesis(x, h, b, n);
        const float* from = ws.shares + (at * x.T + t) * ws.row;
        for (int32_t i = threadIdx.x; i < 2 * y.L + 1; i += kThreads) {
            const bool blank = i <= y.L;
            const float share = from[blank ? i : h.U + i - y.L];
            const int32_t v = blank ? 0 : y.tokens[i - y.L - 1];
            const long long q = __double_as_longlong(share * w + kShift) - __double_as_longlong(kShift);
            if ((uint32_t)v < (uint32_t)x.V) atomicAdd(&sums[v], (unsigned long long)q);
        }
    }
    __syncthreads();
    for (int32_t v = threadIdx.x; v < x.V; v += kThreads)
        out[v] = from_float<T>((float)((double)(long long)sums[v] * (most / kOne)));
}

template <typename T, int K>
hipError_t score_as(const fltop_rows& x, const fltop_hypotheses& h, double* out_scores, const ScoreSpace* keep,
                    hipStream_t stream) {
    const ScoreSpace none = {};
    hipLaunchKernelGGL((score_kernel<T, K>), dim3((unsigned)(x.B * h.N)), dim3(kThreads), 0, stream, x, h, out_scores,
                       keep ? *keep : none, keep != nullptr);
    return hipGetLastError();
}

template <typename T, int K>
hipError_t shares_as(const fltop_rows& x, const fltop_hypotheses& h, const ScoreSpace& ws, hipStream_t stream) {
    hipLaunchKernelGGL((shares_kernel<T, K>), dim3((unsigned)(x.B * h.N)), dim3(kThreads), 0, stream, x, h, ws);
    return hipGetLastError();
}

template <typename T>
hipError_t score_of(const fltop_rows& x, const fltop_hypotheses& h, double* out_scores, const ScoreSpace* keep,
                    hipStream_t stream) {
    if (h.U < kThreads) return score_as<T, 1>(x, h, out_scores, keep, stream);
    if (h.U < 4 * kThreads) return score_as<T, 4>(x, h, out_scores, keep, stream);
    return score_as<T, 16>(x, h, out_scores, keep, stream);
}

template <typename T>
hipError_t grad_of(const fltop_rows& x, const fltop_hypotheses& h, const double* grad_scores, const ScoreSpace& ws,
                   void* grad, hipStream_t stream) {
    hipError_t e = h.U < kThreads       ? shares_as<T, 1>(x, h, ws, stream)
                   : h.U < 4 * kThreads ? shares_as<T, 4>(x, h, ws, stream)
                                        : shares_as<T, 16>(x, h, ws, stream);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(score_grad_kernel<T>, dim3((unsigned)(x.B * x.T)), dim3(kThreads),
                       (size_t)x.V * sizeof(unsigned long long), stream, x, h, grad_scores, ws, static_cast<T*>(grad));
    return hipGetLastError();
}

}  // namespace

hipError_t launch_score(const fltop_rows& x, const fltop_hypotheses& h, double* out_scores, const ScoreSpace* keep,
                        hipStream_t stream) {
    if (x.type == FLTOP_TYPE_BF16) return score_of<__hip_bfloat16>(x, h, out_scores, keep, stream);
    if (x.type == FLTOP_TYPE_F16) return score_of<__half>(x, h, out_scores, keep, stream);
    return score_of<float>(x, h, out_scores, keep, stream);
}

hipError_t launch_score_grad(const fltop_rows& x, const fltop_hypotheses& h, const double* grad_scores,
                             const ScoreSpace& ws, void* grad, hipStream_t stream) {
    if (x.type == FLTOP_TYPE_BF16) return grad_of<__hip_bfloat16>(x, h, grad_scores, ws, grad, stream);
    if (x.type == FLTOP_TYPE_F16) return grad_of<__half>(x, h, grad_scores, ws, grad, stream);
    return grad_of<float>(x, h, grad_scores, ws, grad, stream);
}

}  // namespace fltop
