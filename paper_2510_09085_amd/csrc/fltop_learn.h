// Shared by the operators that learn from hypotheses: element types, numbers with an exponent of
// their own, and the launchers of the kernels.
#ifndef FLTOP_LEARN_H_
#define FLTOP_LEARN_H_

#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>

#include "fltop_internal.h"

namespace fltop {

__device__ inline float to_float(float x) { return x; }
__device__ inline float to_float(__hip_bfloat16 x) { return __bfloat162float(x); }
__device__ inline float to_float(__half x) { return __half2float(x); }

template <typename T> __device__ inline T from_float(float x);
template <> __device__ inline float from_float<float>(float x) { return x; }
template <> __device__ inline __hip_bfloat16 from_float<__hip_bfloat16>(float x) { return __float2bfloat16(x); }
template <> __device__ inline __half from_float<__half>(float x) { return __float2half(x); }

// A probability mass m * 2^e with m in [1/2, 1), or (0, kNoMass).  The masses of a lattice of a
// thousand frames lie anywhere between 1 and e^-100000, and one that looks negligible beside the
// others of its frame may be the only one the hypothesis can end with: each has its own exponent.
struct Mass {
    double m;
    int32_t e;
};
constexpr int32_t kNoMass = -(1 << 30);

__device__ inline Mass no_mass() { return {0.0, kNoMass}; }

// x * 2^e as a Mass.
__device__ inline Mass normalized(double x, int32_t e) {
    const int32_t n = e + __builtin_amdgcn_frexp_exp(x);
    if (x == 0.0 || n <= kNoMass) return no_mass();
    return {__builtin_amdgcn_frexp_mant(x), min(n, -kNoMass)};
}

// exp(lp): lp = k ln2 + r with |r| <= ln2 / 2, the mantissa from the series of e^r (the remainder
// after r^12 / 12! is below 2^-52).  An lp below -7e8 has no mass, so that exponents (below 2^30 in
// size here) can be added in 32 bits.
constexpr float kLeastLogprob = -7e8f;
__device__ inline Mass mass_of(float lp) {
    if (lp < kLeastLogprob) return no_mass();
    const double x = lp > -kLeastLogprob ? (double)-kLeastLogprob : (double)lp;
    const double k = rint(x * 1.4426950408889634);
    double r = fma(-k, 0.6931471805599453, x);
    r = fma(-k, 2.3190468138462996e-17, r);
    double p = 1.0 / 479001600.0;
    p = fma(p, r, 1.0 / 39916800.0);
    p = fma(p, r, 1.0 / 3628800.0);
    p = fma(p, r, 1.0 / 362880.0);
    p = fma(p, r, 1.0 / 40320.0);
    p = fma(p, r, 1.0 / 5040.0);
    p = fma(p, r, 1.0 / 720.0);
    p = fma(p, r, 1.0 / 120.0);
    p = fma(p, r, 1.0 / 24.0);
    p = fma(p, r, 1.0 / 6.0);
    p = fma(p, r, 0.5);
    p = fma(p, r, 1.0);
    p = fma(p, r, 1.0);
    return {p, (int32_t)k};  // p in [0.7, 1.42): used as a factor, which need not be normalized
}

__device__ inline double ln_of(Mass x) {
    return x.e <= kNoMass ? -INFINITY : fma((double)x.e, 0.6931471805599453, log(x.m));
}

// Sums in which the terms keep their own exponents until they are aligned to the largest.
__device__ inline Mass plus(Mass a, Mass b) {
    const int32_t e = max(a.e, b.e);
    return {ldexp(a.m, a.e - e) + ldexp(b.m, b.e - e), e};  // not normalized
}

constexpr int kMostWaves = 16;   // wavefronts that one direction of a lattice takes

// A mass at the border of a block of frames, as it is kept for the gradient: m 2^32 cut to a whole number, and e.  Cut to
// 32 bits a mass is off by 2^-31 of itself at most, an occupancy by 2^-30 of itself: a gradient in fp32 is rounded by 2^-24.
struct Kept {
    uint32_t m;
    int32_t e;
};
// Those of a pair of states, a blank and the token behind it.
struct alignas(16) Mark {
    Kept b, l;
};
__device__ inline Kept kept(double x, int32_t e) {   // x 2^e; x is normal or 0
    const uint32_t hi = (uint32_t)((uint64_t)__double_as_longlong(x) >> 32);
    const uint32_t m = 0x80000000u | (uint32_t)((uint64_t)__double_as_longlong(x) >> 21);
    return {m, hi != 0 ? e + (int32_t)(hi >> 20) - 1022 : kNoMass};
}
__device__ inline Mass mass_of(Kept x) {
    const uint64_t bits = (uint64_t)(x.m & 0x7fffffffu) << 21 | 0x3fe0000000000000ull;
    return x.e <= kNoMass ? no_mass() : Mass{__longlong_as_double((long long)bits), x.e};
}

// What fltop_ctc_score leaves for fltop_ctc_score_grad.
struct ScoreSpace {
    double* total_m;   // [B*N] P(hypothesis) as a Mass; kNoMass for one that takes no part
    int32_t* total_e;  // [B*N]
    Mark* marks;       // [B*N][2][blocks][row] both directions at the borders of blocks
    int64_t row;       // pairs that a direction's lanes hold
    int64_t marks_of;  // marks of one direction of one hypothesis
    size_t bytes;
};

// Pairs of states that a lane holds where a direction has a workgroup of its own: two while that has sixteen wavefronts at
// most, with the one that tabulates.  (With eight pairs the registers spill: 16 transcripts of 1700 tokens over 3600 frames
// of an untrained model took 12.5 ms, both directions at once, and take 5.4 ms now, 5.7 with the borders for a gradient.)
inline int lattice_pairs(int32_t U) { return U < 1920 ? 2 : 4; }
inline int waves_for(int32_t U, int pairs) { return (U + 64 * pairs) / (64 * pairs); }   // for U + 1 pairs
// Frames that are gone through together: exponents are kept once for each such block.
inline int block_frames(int pairs) { return pairs < 4 ? 8 : 4; }
__host__ __device__ inline int64_t blocks_of(int32_t T, int32_t R) { return ((int64_t)T + R - 1) / R; }

inline ScoreSpace carve_score(void* base, int32_t B, int32_t T, int32_t N, int32_t U) {
    ScoreSpace s;
    const size_t hyps = (size_t)B * (size_t)N;
    const int pairs = lattice_pairs(U);
    s.row = (int64_t)pairs * waves_for(U, pairs) * 64;
    s.marks_of = blocks_of(T, block_frames(pairs)) * s.row;
    const size_t off_e = align_up(hyps * sizeof(double), 256);
    const size_t off_marks = off_e + align_up(hyps * sizeof(int32_t), 256);
    s.bytes = align_up(off_marks + hyps * 2 * (size_t)s.marks_of * sizeof(Mark), 256);
    char* p = static_cast<char*>(base);
    s.total_m = p ? reinterpret_cast<double*>(p) : nullptr;
    s.total_e = p ? reinterpret_cast<int32_t*>(p + off_e) : nullptr;
    s.marks = p ? reinterpret_cast<Mark*>(p + off_marks) : nullptr;
    return s;
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
    const double kl = e < INFINITY ? e - gap : e;
    // (a weight of 0 leaves the KL out: it may be infinite)
    const bool weighs = p.kl_weight != 0.0;
    s->loss += fmax(-plain, -cut) + (weighs ? p.kl_weight * kl : 0.0);
    s->kl += kl;
    s->clipped += plain > cut ? 1.0 : 0.0;
    s->n += 1.0;
    return (plain <= cut ? -plain : 0.0) - (weighs ? p.kl_weight * e : 0.0);
}


// Workspace of the policy losses: over given log-probabilities the sums of each row; over logits the frames of each
// utterance that take part, then three sums from each workgroup and the number of all those frames.
inline size_t policy_sums_bytes(int32_t B) { return align_up((size_t)B * sizeof(PolicySums), 256); }
constexpr int32_t kMostRowGroups = 2048;
inline size_t row_counts_bytes(int32_t B) { return align_up((size_t)B * sizeof(int32_t), 256); }
inline size_t row_workspace_bytes(int32_t B) {
    return row_counts_bytes(B) + align_up((3 * kMostRowGroups + 1) * sizeof(double), 256);
}

hipError_t launch_score(const fltop_rows& x, const fltop_hypotheses& h, double* out_scores,
                        const ScoreSpace* keep, hipStream_t stream);
hipError_t launch_score_grad(const fltop_rows& x, const fltop_hypotheses& h,
                             const double* grad_scores, const ScoreSpace& ws, void* grad,
                             hipStream_t stream);
hipError_t launch_preference(const fltop_preference& p, void* workspace, hipStream_t stream);
hipError_t launch_policy(const double* scores, const double* old_scores, const double* ref_scores,
                         const double* advantages, const int32_t* counts, int32_t B, int32_t N,
                         const fltop_policy& policy, void* workspace, double* summary,
                         double* grad_scores, hipStream_t stream);
hipError_t launch_policy_logits(const fltop_rows& x, const int32_t* tokens, const float* old_logps,
                                const float* ref_logps, const float* advantages, bool per_frame,
                                const fltop_policy& policy, void* workspace, float* summary,
                                float* logps, void* grad, hipStream_t stream);

}  // namespace fltop
#endif  // FLTOP_LEARN_H_
