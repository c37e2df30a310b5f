// The clipped policy loss from logits: for each frame the log-softmax at its token, the loss and its derivative to that
// log-probability, and from it the gradient of the whole row,
//     d/dx_v = c ([v = token] - softmax(x)_v),   c = df/dl * weight.
// Rows are read once and stay in registers between their statistics and their gradient: what bounds these kernels is
// reading the logits and writing the gradient.
//
// Three launches.  Means need the number of frames that take part before any gradient: one kernel counts them for each
// utterance.  Then the rows; each workgroup adds the counts up, in one order.  The frames' losses are summed lane by lane
// in a fixed assignment of rows, one sum is left by each workgroup, and the last kernel adds those.
//
// Statistics, exponentials and logarithms of a row are fp32: 256 x 1500 rows of 32 values are off by 1.3e-7 of the results'
// size from 64 bits, where elementary operations in fp32 throughout are by 2.1e-7.
#include <type_traits>

#include "fltop_learn.h"

namespace fltop {
namespace {

constexpr int kWave = 64;
constexpr int kThreads = 256;
constexpr int kLongThreads = 1024;

template <typename T> constexpr int kVec = 16 / sizeof(T);

typedef float Float2 __attribute__((ext_vector_type(2)));
typedef __bf16 Bf2 __attribute__((ext_vector_type(2)));
typedef _Float16 Half2 __attribute__((ext_vector_type(2)));

// 16 bytes of a row, as they lie in memory: two values of 16 bits in one register.
template <typename T>
struct Vec {
    static constexpr int N = kVec<T>;
    uint32_t w[4];

    __device__ float operator[](int e) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[e]);
        const uint32_t x = w[e / 2];
        if constexpr (std::is_same<T, __hip_bfloat16>::value) return __uint_as_float(e & 1 ? x & 0xFFFF0000u : x << 16);
        return __half2float(__ushort_as_half((unsigned short)(e & 1 ? x >> 16 : x)));
    }
    static __device__ uint32_t bits(T x) {
        if constexpr (sizeof(T) == 4) return __float_as_uint(x);
        unsigned short u;
        __builtin_memcpy(&u, &x, 2);
        return u;
    }
    __device__ void set(int e, uint32_t bits) {
        if constexpr (sizeof(T) == 4)
            w[e] = bits;
        else
            w[e / 2] = e & 1 ? (w[e / 2] & 0xFFFFu) | bits << 16 : (w[e / 2] & 0xFFFF0000u) | bits;
    }
    static __device__ uint32_t no_mass() { return bits(from_float<T>(-INFINITY)); }
    __device__ void clear() {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = sizeof(T) == 4 ? no_mass() : no_mass() << 16 | no_mass();
    }
    // Rounds fp32 values, two by two where the type has an instruction for that.
    __device__ void round(const float (&f)[N]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(T) == 4) {
                w[i] = __float_as_uint(f[i]);
            } else if constexpr (std::is_same<T, __hip_bfloat16>::value) {
                const Bf2 p = __builtin_convertvector((Float2){f[2 * i], f[2 * i + 1]}, Bf2);
                __builtin_memcpy(&w[i], &p, 4);
            } else {
                const Half2 p = __builtin_convertvector((Float2){f[2 * i], f[2 * i + 1]}, Half2);
                __builtin_memcpy(&w[i], &p, 4);
            }
        }
    }
    // Makes the compiler take the values for new ones: what it made of them before (floats, exponentials, one or two
    // registers a value) is worked out again rather than kept in registers next to them.
    __device__ void renew() {
#pragma unroll
        for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(w[i]));
    }
};

// A row's vectors are loaded and stored wherever they lie (gfx950 does so at any address); the part behind the last whole
// one is moved value by value, and places behind it hold -inf.
template <typename T>
__device__ inline Vec<T> load_part(const T* row, int32_t at, int32_t V) {
    Vec<T> v;
    if (at + kVec<T> <= V) {
        __builtin_memcpy(v.w, row + at, 16);
        return v;
    }
    v.clear();
#pragma unroll
    for (int e = 0; e < kVec<T> - 1; ++e)
        if (at + e < V) v.set(e, Vec<T>::bits(row[at + e]));
    return v;
}
template <typename T>
__device__ inline void store_part(T* row, int32_t at, int32_t V, const Vec<T>& v) {
    if (at + kVec<T> <= V) {
        __builtin_memcpy(row + at, v.w, 16);
        return;
    }
#pragma unroll
    for (int e = 0; e < kVec<T> - 1; ++e)
        if (at + e < V) {
            const uint32_t x = sizeof(T) == 4 ? v.w[e] : v.w[e / 2] >> (e & 1 ? 16 : 0);
            __builtin_memcpy(row + at + e, &x, sizeof(T));
        }
}

// Takes the token out of a lane's vector that starts at c (its place then has no mass); whether it was there.
template <typename T>
__device__ inline bool take_token(Vec<T>& v, int32_t c, int32_t token, float* x_token) {
    if ((uint32_t)(token - c) >= (uint32_t)kVec<T>) return false;
#pragma unroll
    for (int e = 0; e < kVec<T>; ++e) {
        if (c + e != token) continue;
        *x_token = v[e];
        v.set(e, Vec<T>::no_mass());
    }
    return true;
}

// exp(x) for x <= 0, within two steps of fp32 and what x * log2(e) is off.
__device__ inline float exp_down(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896341f); }

template <int N>
__device__ inline float max_of(float x) {
#pragma unroll
    for (int o = N / 2; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor(x, o, kWave));
    return x;
}
template <int N>
__device__ inline float sum_of(float x) {
#pragma unroll
    for (int o = N / 2; o > 0; o >>= 1) x += __shfl_xor(x, o, kWave);
    return x;
}
__device__ inline double sum_of_wave(double x) {
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) x += __shfl_xor(x, o, kWave);
    return x;
}

__device__ inline void wave_fence() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

__global__ __launch_bounds__(kThreads) void part_kernel(fltop_rows x, const int32_t* tokens, int32_t* counts) {
    __shared__ int32_t of_wave[kThreads / kWave];
    const int32_t b = blockIdx.x;
    const int32_t frames = min(x.lengths[b], x.T);
    int32_t n = 0;
#pragma unroll 4
    for (int32_t t = threadIdx.x; t < frames; t += kThreads)
        n += (uint32_t)tokens[(int64_t)b * x.T + t] < (uint32_t)x.V ? 1 : 0;
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) n += __shfl_xor(n, o, kWave);
    if (threadIdx.x % kWave == 0) of_wave[threadIdx.x / kWave] = n;
    __syncthreads();
    if (threadIdx.x == 0) counts[b] = of_wave[0] + of_wave[1] + of_wave[2] + of_wave[3];
}

// Everything but the logits of a call.
struct Frames {
    const int32_t* tokens;
    const float *old_logps, *ref_logps, *advantages;
    int32_t per_frame;
    const int32_t* counts;   // [B]
    double* partial;         // [kMostRowGroups][3], and one more
    float* logps;
};

// What a frame's entry weighs: frames that take part, and utterances that have any.
struct Weights {
    double all, rows;
    int32_t reduction;
    // `scratch`: two numbers for each wavefront
    __device__ Weights(const int32_t* counts, int32_t B, int32_t how, int64_t* scratch) : reduction(how) {
        int64_t n = 0, some = 0;
        for (int32_t b = threadIdx.x; b < B; b += blockDim.x) {
            n += counts[b];
            some += counts[b] > 0;
        }
#pragma unroll
        for (int o = kWave / 2; o > 0; o >>= 1) {
            n += __shfl_xor(n, o, kWave);
            some += __shfl_xor(some, o, kWave);
        }
        const int wave = threadIdx.x / kWave, waves = blockDim.x / kWave;
        if (threadIdx.x % kWave == 0) {
            scratch[wave] = n;
            scratch[waves + wave] = some;
        }
        __syncthreads();
        n = some = 0;
        for (int w = 0; w < waves; ++w) {
            n += scratch[w];
            some += scratch[waves + w];
        }
        all = (double)n;
        rows = (double)some;
        __syncthreads();
    }
    __device__ double of(int32_t count) const {
        return reduction == FLTOP_REDUCE_TOKEN ? 1.0 / all : reduction == FLTOP_REDUCE_SEQUENCE ? 1.0 / (count * rows) : 1.0;
    }
};

struct Sums {
    double loss = 0.0, kl = 0.0, clipped = 0.0;
};

// What the row needs of a frame: gradients are e * by for the others' exponentials e, and `own` at the token.
struct RowGradient {
    float by, own;
};

// exp(x) - x - 1 and exp(x) - 1, with their digits where x is small: x^2 (1/2 + x/6 + .. + x^6/40320) leaves out
// x^9/9!, below 2^-24 of it.  Infinities are what the formulas give.
struct Beyond {
    float kl;
    double slope;
};
__device__ inline Beyond exp_beyond_line(float x) {
    if (fabsf(x) > 0.5f) {
        const float e = expm1f(x);
        return {e < INFINITY ? e - x : e, e};
    }
    float p = 1.0f / 40320.0f;
    p = fmaf(p, x, 1.0f / 5040.0f);
    p = fmaf(p, x, 1.0f / 720.0f);
    p = fmaf(p, x, 1.0f / 120.0f);
    p = fmaf(p, x, 1.0f / 24.0f);
    p = fmaf(p, x, 1.0f / 6.0f);
    p = fmaf(p, x, 0.5f);
    const float kl = p * x * x;
    return {kl, (double)kl + x};
}

// A frame of a token, from its row's statistics: rest = sum of exp(x_v - top) over v other than the token (so that 1 - p
// and ln p keep their digits where p is nearly 1).  Exponentials and logarithms are fp32, as the statistics are; the
// log-probability they make and its differences are taken in fp64, sums of frames too.
__device__ inline RowGradient frame_gradient(const Frames& f, int64_t at, int32_t b, float top, float rest, float x_token,
                                             const fltop_policy& p, const Weights& weights, Sums* sums) {
    const float gap = x_token - top, own = expf(gap), sum = rest + own;
    const double l = own > rest ? -(double)log1pf(rest / own) : (double)gap - (double)logf(sum);
    const double weight = weights.of(f.counts[b]);
    const float A = f.advantages[f.per_frame ? at : b];
    const float r = expf((float)(l - f.old_logps[at]));
    const float cut_r = fminf(fmaxf(r, (float)(1.0 - p.clip_low)), (float)(1.0 + p.clip_high));
    const float plain = r * A, cut = cut_r * A;
    const float beyond = f.ref_logps ? (float)(f.ref_logps[at] - l) : 0.0f;
    const Beyond kl = exp_beyond_line(beyond);
    // (a weight of 0 leaves the KL out: it may be infinite)
    const bool weighs = p.kl_weight != 0.0;
    const double d = (plain <= cut ? -(double)plain : 0.0) - (weighs ? p.kl_weight * kl.slope : 0.0);
    sums->loss += (fmaxf(-plain, -cut) + (weighs ? p.kl_weight * kl.kl : 0.0)) * weight;
    sums->kl += kl.kl * weight;
    sums->clipped += plain > cut ? 1.0 : 0.0;
    f.logps[at] = (float)l;
    const float c = (float)(d * (weight * p.scale));
    return {-c / sum, c * (rest / sum)};
}

// Leaves a workgroup's sums, and the first one the number of all frames that take part.
template <int THREADS>
__device__ inline void leave_sums(const Sums& mine, const Weights& weights, double* partial) {
    if (blockIdx.x == 0 && threadIdx.x == 0) partial[3 * kMostRowGroups] = weights.all;
    __shared__ double of_wave[THREADS / kWave][3];
    const double s[3] = {sum_of_wave(mine.loss), sum_of_wave(mine.kl), sum_of_wave(mine.clipped)};
    if (threadIdx.x % kWave == 0)
        for (int k = 0; k < 3; ++k) of_wave[threadIdx.x / kWave][k] = s[k];
    __syncthreads();
    if (threadIdx.x < 3) {
        double sum = 0.0;
        for (int w = 0; w < THREADS / kWave; ++w) sum += of_wave[w][threadIdx.x];
        partial[3 * (int64_t)blockIdx.x + threadIdx.x] = sum;
    }
}

// Short rows: LANES lanes take a row, ITER vectors each, and a wavefront PASSES times kWave / LANES rows before it goes on
// to their losses, for which each row has a lane of its own: that arithmetic, a few hundred instructions, is done once for
// all of them.
template <typename T, int LANES, int ITER, int PASSES>
__global__ __launch_bounds__(kThreads, 4) void short_rows_kernel(fltop_rows x, Frames f, fltop_policy p, T* grad) {
    constexpr int kAtOnce = kWave / LANES, kRows = kAtOnce * PASSES, N = kVec<T>;
    static_assert(kRows <= kWave, "a lane for each row");
    struct Row {
        int64_t start;   // of its logits
        int32_t token;   // -1: takes no part
        float top, rest, x_token;
        RowGradient g;
    };
    __shared__ Row rows_of[kThreads / kWave][kRows];
    __shared__ int64_t scratch[2 * kThreads / kWave];
    const Weights weights(f.counts, x.B, p.reduction, scratch);
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int group = lane / LANES, within = lane % LANES;
    Row* const rows = rows_of[wave];
    const int64_t total = (int64_t)x.B * x.T, step = (int64_t)gridDim.x * (kThreads / kWave) * kRows;
    const T* const data = static_cast<const T*>(x.data);
    Sums sums;
    for (int64_t first = ((int64_t)blockIdx.x * (kThreads / kWave) + wave) * kRows; first < total; first += step) {
        const int64_t at = first + lane;
        int32_t b = 0, token = -1;
        if (lane < kRows) {
            if (at < total) {
                b = (int32_t)((uint32_t)at / (uint32_t)x.T);
                const int32_t t = (int32_t)at - b * x.T;
                if (t < x.lengths[b]) token = f.tokens[at];
                if ((uint32_t)token >= (uint32_t)x.V) token = -1;
                rows[lane].start = b * x.batch_stride + t * x.frame_stride;
            }
            rows[lane].token = token;
        }
        wave_fence();
        Vec<T> v[PASSES][ITER];
#pragma unroll
        for (int s = 0; s < PASSES; ++s) {
            const Row& row = rows[s * kAtOnce + group];
#pragma unroll
            for (int i = 0; i < ITER; ++i) {
                const int32_t c = (i * LANES + within) * N;
                if (row.token >= 0 && c < x.V) {
                    v[s][i] = load_part(data + row.start, c, x.V);
                } else {
                    v[s][i].clear();
                }
            }
        }
#pragma unroll
        for (int s = 0; s < PASSES; ++s) {
            Row& row = rows[s * kAtOnce + group];
            const int32_t tok = row.token;
            float top = -INFINITY;
#pragma unroll
            for (int i = 0; i < ITER; ++i) {
                float x_token;
                if (take_token(v[s][i], (i * LANES + within) * N, tok, &x_token)) row.x_token = top = x_token;
            }
#pragma unroll
            for (int i = 0; i < ITER; ++i)
#pragma unroll
                for (int e = 0; e < N; ++e) top = fmaxf(top, v[s][i][e]);
            top = max_of<LANES>(top);
            float rest = 0.0f;
#pragma unroll
            for (int i = 0; i < ITER; ++i)
#pragma unroll
                for (int e = 0; e < N; ++e) rest += exp_down(v[s][i][e] - top);
            rest = sum_of<LANES>(rest);
            if (within == 0) {
                row.top = top;
                row.rest = rest;
            }
        }
        wave_fence();
#pragma unroll
        for (int s = 0; s < PASSES; ++s)
#pragma unroll
            for (int i = 0; i < ITER; ++i) v[s][i].renew();
        if (token >= 0)
            rows[lane].g = frame_gradient(f, at, b, rows[lane].top, rows[lane].rest, rows[lane].x_token, p, weights, &sums);
        else if (lane < kRows && at < total)
            f.logps[at] = 0.0f;
        wave_fence();
#pragma unroll
        for (int s = 0; s < PASSES; ++s) {
            const int r = s * kAtOnce + group;
            const Row& row = rows[r];
            if (first + r >= total) continue;
            T* const out = grad + (first + r) * x.V;
            const int32_t tok = row.token;
            const float top = row.top, by = row.g.by;
#pragma unroll
            for (int i = 0; i < ITER; ++i) {
                const int32_t c = (i * LANES + within) * N;
                if (c >= x.V) continue;
                float g[N];
#pragma unroll
                for (int e = 0; e < N; ++e) g[e] = tok >= 0 ? exp_down(v[s][i][e] - top) * by : 0.0f;
                Vec<T> o;
                o.round(g);
                store_part(out, c, x.V, o);
                // (a wavefront's stores to one place come in their order)
                if ((uint32_t)(tok - c) < (uint32_t)N) out[tok] = from_float<T>(row.g.own);
            }
        }
        wave_fence();
    }
    leave_sums<kThreads>(sums, weights, f.partial);
}

// Long rows: a workgroup for each.  With HELD the row's vectors stay in registers; rows beyond what THREADS hold are read
// again for their gradient.
template <typename T, int THREADS, int ITER, bool HELD>
__global__ __launch_bounds__(THREADS, 4) void long_rows_kernel(fltop_rows x, Frames f, fltop_policy p, T* grad) {
    constexpr int N = kVec<T>, kWaves = THREADS / kWave;
    __shared__ int64_t scratch[2 * kWaves];
    __shared__ float tops[kWaves], rests[kWaves];
    __shared__ RowGradient shared_g;
    const Weights weights(f.counts, x.B, p.reduction, scratch);
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int64_t total = (int64_t)x.B * x.T;
    Sums sums;
    for (int64_t at = blockIdx.x; at < total; at += gridDim.x) {
        const int32_t b = (int32_t)((uint32_t)at / (uint32_t)x.T), t = (int32_t)at - b * x.T;
        const int32_t token = t < x.lengths[b] ? f.tokens[at] : -1;
        T* const out = grad + at * x.V;
        if ((uint32_t)token >= (uint32_t)x.V) {
            const Vec<T> zero = {{0, 0, 0, 0}};
            for (int32_t c = threadIdx.x * N; c < x.V; c += THREADS * N) store_part(out, c, x.V, zero);
            if (threadIdx.x == 0) f.logps[at] = 0.0f;
            continue;
        }
        const T* const row = static_cast<const T*>(x.data) + b * x.batch_stride + t * x.frame_stride;
        const float x_token = to_float(row[token]);
        float taken;
        Vec<T> v[HELD ? ITER : 1];
        // this lane's own maximum and sum; lanes are put together afterwards
        float top = x_token, rest = 0.0f;
        if constexpr (HELD) {
#pragma unroll
            for (int i = 0; i < ITER; ++i) {
                const int32_t c = (i * THREADS + (int)threadIdx.x) * N;
                if (c < x.V) {
                    v[i] = load_part(row, c, x.V);
                    take_token(v[i], c, token, &taken);
                } else {
                    v[i].clear();
                }
            }
#pragma unroll
            for (int i = 0; i < ITER; ++i)
#pragma unroll
                for (int e = 0; e < N; ++e) top = fmaxf(top, v[i][e]);
            top = max_of<kWave>(top);
            if (lane == 0) tops[wave] = top;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < kWaves; ++w) top = fmaxf(top, tops[w]);
#pragma unroll
            for (int i = 0; i < ITER; ++i) v[i].renew();
#pragma unroll
            for (int i = 0; i < ITER; ++i)
#pragma unroll
                for (int e = 0; e < N; ++e) rest += exp_down(v[i][e] - top);
        } else {
            for (int32_t c = threadIdx.x * N; c < x.V; c += THREADS * N) {
                Vec<T> one = load_part(row, c, x.V);
                take_token(one, c, token, &taken);
                float m = top;
#pragma unroll
                for (int e = 0; e < N; ++e) m = fmaxf(m, one[e]);
                if (m > top) {   // the sum so far is rescaled
                    rest *= exp_down(top - m);
                    top = m;
                }
                if (top > -INFINITY) {
#pragma unroll
                    for (int e = 0; e < N; ++e) rest += exp_down(one[e] - top);
                }
            }
            const float mine = top;
            top = max_of<kWave>(top);
            if (lane == 0) tops[wave] = top;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < kWaves; ++w) top = fmaxf(top, tops[w]);
            if (mine < top) rest *= exp_down(mine - top);
        }
        rest = sum_of<kWave>(rest);
        if constexpr (HELD) {
#pragma unroll
            for (int i = 0; i < ITER; ++i) v[i].renew();
        }
        if (lane == 0) rests[wave] = rest;
        __syncthreads();
        if (wave == 0) {
            float all = lane < kWaves ? rests[lane] : 0.0f;
            all = sum_of<kWave>(all);
            if (lane == 0) shared_g = frame_gradient(f, at, b, top, all, x_token, p, weights, &sums);
        }
        __syncthreads();
        const RowGradient g = shared_g;
        auto give = [&](const Vec<T>& one, int32_t c) {
            float o[N];
#pragma unroll
            for (int e = 0; e < N; ++e) o[e] = exp_down(one[e] - top) * g.by;
            Vec<T> rounded;
            rounded.round(o);
            store_part(out, c, x.V, rounded);
            if ((uint32_t)(token - c) < (uint32_t)N) out[token] = from_float<T>(g.own);
        };
        if constexpr (HELD) {
#pragma unroll
            for (int i = 0; i < ITER; ++i) {
                const int32_t c = (i * THREADS + (int)threadIdx.x) * N;
                if (c < x.V) give(v[i], c);
            }
        } else {
            for (int32_t c = threadIdx.x * N; c < x.V; c += THREADS * N) give(load_part(row, c, x.V), c);
        }
    }
    leave_sums<THREADS>(sums, weights, f.partial);
}

__global__ __launch_bounds__(kLongThreads) void policy_summary_kernel(const double* partial, int32_t groups, float* summary) {
    __shared__ double of_wave[kLongThreads / kWave][3];
    const double all = partial[3 * kMostRowGroups];
    Sums s;
#pragma unroll
    for (int32_t k = 0; k < kMostRowGroups / kLongThreads; ++k) {
        const int32_t g = k * kLongThreads + threadIdx.x;
        if (g >= groups) continue;
        s.loss += partial[3 * g];
        s.kl += partial[3 * g + 1];
        s.clipped += partial[3 * g + 2];
    }
    const double mine[3] = {sum_of_wave(s.loss), sum_of_wave(s.kl), sum_of_wave(s.clipped)};
    if (threadIdx.x % kWave == 0)
        for (int k = 0; k < 3; ++k) of_wave[threadIdx.x / kWave][k] = mine[k];
    __syncthreads();
    if (threadIdx.x < 3) {
        double sum = 0.0;
        for (int w = 0; w < kLongThreads / kWave; ++w) sum += of_wave[w][threadIdx.x];
        if (threadIdx.x == 2) sum = all > 0.0 ? sum / all : 0.0;
        summary[threadIdx.x] = (float)sum;
    }
}

template <typename T, int LANES, int ITER, int PASSES>
int32_t short_rows(const fltop_rows& x, const Frames& f, const fltop_policy& p, void* grad, hipStream_t stream) {
    const int64_t rows = (int64_t)x.B * x.T, each = (int64_t)(kThreads / kWave) * (kWave / LANES) * PASSES;
    int64_t groups = (rows + each - 1) / each;
    if (groups > kMostRowGroups) groups = kMostRowGroups;
    hipLaunchKernelGGL((short_rows_kernel<T, LANES, ITER, PASSES>), dim3((unsigned)groups), dim3(kThreads), 0, stream, x, f, p,
                       static_cast<T*>(grad));
    return (int32_t)groups;
}

template <typename T, int THREADS, int ITER, bool HELD>
int32_t long_rows(const fltop_rows& x, const Frames& f, const fltop_policy& p, void* grad, hipStream_t stream) {
    const int64_t rows = (int64_t)x.B * x.T;
    const int32_t groups = (int32_t)(rows < kMostRowGroups ? rows : kMostRowGroups);
    hipLaunchKernelGGL((long_rows_kernel<T, THREADS, ITER, HELD>), dim3(groups), dim3(THREADS), 0, stream, x, f, p,
                       static_cast<T*>(grad));
    return groups;
}

// As few lanes as hold a row in one vector each, up to a wavefront; then as few vectors as a wavefront, a workgroup of
// 256 and one of 512 hold it in; longer rows are read again.  2^25 fp32 values in rows of 32: 137 us, 385 with a wavefront for
// each row; of 1024: 66, 107 with a workgroup; of 2048: 62 and 69; of 8192: 58, 118 if they were read again; of 32000: 65
// and 94.  Several vectors a lane in short rows save shuffles and lose more by loads that lie apart (rows of 32: 167).
template <typename T>
int32_t rows_of(const fltop_rows& x, const Frames& f, const fltop_policy& p, void* grad, hipStream_t stream) {
    const int32_t vectors = (x.V + kVec<T> - 1) / kVec<T>;
    if (vectors <= 4) return short_rows<T, 4, 1, 4>(x, f, p, grad, stream);
    if (vectors <= 8) return short_rows<T, 8, 1, 8>(x, f, p, grad, stream);
    if (vectors <= 16) return short_rows<T, 16, 1, 8>(x, f, p, grad, stream);
    if (vectors <= 32) return short_rows<T, 32, 1, 8>(x, f, p, grad, stream);
    if (vectors <= 64) return short_rows<T, 64, 1, 8>(x, f, p, grad, stream);
    if (vectors <= 128) return short_rows<T, 64, 2, 4>(x, f, p, grad, stream);
    if (vectors <= 256) return short_rows<T, 64, 4, 2>(x, f, p, grad, stream);
    if (vectors <= 512) return short_rows<T, 64, 8, 1>(x, f, p, grad, stream);
    if (vectors <= 1024) return long_rows<T, 256, 4, true>(x, f, p, grad, stream);
    if (vectors <= 2048) return long_rows<T, 256, 8, true>(x, f, p, grad, stream);
    if (vectors <= 4096) return long_rows<T, 512, 8, true>(x, f, p, grad, stream);
    if (vectors <= 8192) return long_rows<T, 512, 16, true>(x, f, p, grad, stream);
    return long_rows<T, 1024, 1, false>(x, f, p, grad, stream);
}

}  // namespace

hipError_t launch_policy_logits(const fltop_rows& x, const int32_t* tokens, const float* old_logps,
                                const float* ref_logps, const float* advantages, bool per_frame,
                                const fltop_policy& policy, void* workspace, float* summary, float* logps, void* grad,
                                hipStream_t stream) {
    int32_t* const counts = static_cast<int32_t*>(workspace);
    double* const partial = reinterpret_cast<double*>(static_cast<char*>(workspace) + row_counts_bytes(x.B));
    hipLaunchKernelGGL(part_kernel, dim3(x.B), dim3(kThreads), 0, stream, x, tokens, counts);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const Frames f = {tokens, old_logps, ref_logps, advantages, per_frame, counts, partial, logps};
    const int32_t groups = x.type == FLTOP_TYPE_BF16  ? rows_of<__hip_bfloat16>(x, f, policy, grad, stream)
                           : x.type == FLTOP_TYPE_F16 ? rows_of<__half>(x, f, policy, grad, stream)
                                                      : rows_of<float>(x, f, policy, grad, stream);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(policy_summary_kernel, dim3(1), dim3(kLongThreads), 0, stream, partial, groups, summary);
    return hipGetLastError();
}

}  // namespace fltop
