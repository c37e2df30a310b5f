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

// One hypothesis as the kernels see it: its tokens in lattice order or reversed.
struct Hyp {
    const int32_t* tokens;
    int32_t L;       // -1: not there, -2: longer than U
    int32_t frames;
};

__device__ inline Hyp hypothesis(const fltop_rows& x, const fltop_hypotheses& h, int32_t b, int32_t n) {
    Hyp y;
    const int32_t count = h.counts ? h.counts[b] : h.N;
    // (the same for a whole workgroup: kept in scalar registers)
    y.tokens = h.tokens + b * h.token_batch_stride + n * h.token_stride;
    y.L = __builtin_amdgcn_readfirstlane(n < count ? h.lengths[b * h.length_batch_stride + n] : -1);
    if (y.L < 0) y.L = -1;
    if (y.L > h.U) y.L = -2;
    const int32_t f = __builtin_amdgcn_readfirstlane(x.lengths[b]);
    y.frames = f < 0 ? 0 : (f > x.T ? x.T : f);
    return y;
}

// ---- how a hypothesis is laid out over the lanes -------------------------------------------------
//
// W wavefronts take a direction of a hypothesis, lane by lane K pairs (b_i, l_i) each.  For the score alone one workgroup
// takes both directions to the middle of the utterance: half as many serial frames as one direction would have.  With a
// gradient wanted each direction has a workgroup, goes all the way and leaves its masses at the borders of the blocks
// (below); a second kernel then goes through the blocks of all utterances at once, once more from either border, and needs
// no masses of single frames in memory.
//
// The serial frames bound it: 64 transcripts of 500 frames take 77 us, 63 blocks at about 1.2 us each, of which the five
// products and sums of a frame's two pairs are a third; the rest are the latencies of the barrier, of LDS, of the lanes'
// exponents and of the shifts (counted: vector instructions issue in a third of a wavefront's life, any in 58%).  2048
// hypotheses of 500 frames keep all compute units busy and take 245 us, in half of which the SIMDs issue a vector
// instruction.
//
// Frames come in blocks of R.  Within a block only l_{i-1} passes from lane to lane (one DPP shift),
// and the wavefront above takes the same block one turn later with the last lane's masses from LDS,
// so that there is one barrier for a block and none for a frame.
//
// Every mass has its own exponent (class Mass), but aligning three of them for each sum costs more
// than the sum.  So a block is entered with one exponent E for each lane, no smaller than that of any
// mass that can reach the lane within the block (those of the kReach lanes below), and if
//   - no mass of these lanes is below 2^(E - kSpread), and
//   - no emission needed in the block is below 2^-58 (e^-40) or from 2^14 up,
// then nothing leaves the range of fp64: masses stay above 2^(E - kSpread - 58 R) and below 2^(E + 128)
// until its end.  Of the lanes below a lane whose states all have mass only that lane's own count: what
// reaches it and leaves fp64 is below 2^-1022 of E, where each sum has a term of its own of 2^-957 at
// least, so that nothing of 64 bits is lost.  A frame is then three multiply-adds and two products for each
// pair.  Blocks that do not hold this (masks of -inf, masses of e^-3000 that may be needed yet) are gone
// through with aligned exponents.  Rows of a trained model stay within: 10 tokens at e^-25 are 360 bits.
//
// The exponential of an emission takes three times the frame's own work.  For vocabularies of up to
// kTabulated tokens a wavefront more for each direction takes all of a block's, a turn ahead, into a
// table in LDS; for larger ones each lane takes its tokens'.

constexpr int kWave = 64;
constexpr int kTabulated = 64;

// Lane i gets lane i - 1's value, lane 0 gets `first`.
__device__ inline int32_t from_below(int32_t x, int32_t first) {
    return __builtin_amdgcn_update_dpp(first, x, 0x138, 0xf, 0xf, false);  // wave_shr:1
}
__device__ inline double from_words(int32_t hi, int32_t lo) {
    return __longlong_as_double((long long)(((uint64_t)(uint32_t)hi << 32) | (uint32_t)lo));
}
__device__ inline double from_below(double x, double first) {
    const long long a = __double_as_longlong(x), f = __double_as_longlong(first);
    return from_words(from_below((int32_t)(a >> 32), (int32_t)(f >> 32)), from_below((int32_t)a, (int32_t)f));
}
__device__ inline double from_lane(double x, int lane) {
    const long long a = __double_as_longlong(x);
    return from_words(__builtin_amdgcn_readlane((int32_t)(a >> 32), lane),
                      __builtin_amdgcn_readlane((int32_t)a, lane));
}

// 2^e for e in [-1022, 1023], and 0 for -1023.
__device__ inline double power_of_two(int32_t e) { return from_words((e + 1023) << 20, 0); }
// 2^e as a factor of masses of which those that leave the range are 0.
__device__ inline double rescaling(int32_t e) { return power_of_two(max(min(e, 1000), -1023)); }
// x, or 0 with a mask of 0 (no branch).
__device__ inline double masked(double x, int32_t mask) {
    const long long a = __double_as_longlong(x);
    return from_words((int32_t)(a >> 32) & mask, (int32_t)a & mask);
}
__device__ inline uint32_t high_word(double x) { return (uint32_t)(__double_as_longlong(x) >> 32); }

// Emissions that a block may have to be gone through with one exponent for each lane.
constexpr float kLeastNear = -40.0f, kMostNear = 9.7f;
constexpr uint32_t kLeastWord = (1023u - 58) << 20, kMostWord = (1023u + 14) << 20;

// exp(lp) for lp within +-600, as mass_of, with k taken from the last bits of a number in which they are worth
// one and added to the result's exponent.
__device__ inline double exp_near(float lp) {
    const double x = lp;
    constexpr double kShift = 6755399441055744.0;   // 1.5 * 2^52
    const double t = fma(x, 1.4426950408889634, kShift);
    const double k = t - kShift;
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
    const long long bits = __double_as_longlong(p);
    return from_words((int32_t)(bits >> 32) + ((int32_t)__double_as_longlong(t) << 20), (int32_t)bits);
}

// exp(lp) of any emission, off where it leaves the range in which blocks are gone through with one exponent (and still
// outside of that range).
__device__ inline double exp_any(float lp) { return exp_near(fminf(fmaxf(lp, -600.0f), 600.0f)); }

// An element as it lies in memory; converted where it is used, so that loads stay in flight.
template <int TYPE>
__device__ inline uint32_t raw_at(const char* row, int32_t v) {
    if constexpr (TYPE == FLTOP_TYPE_F32)
        return reinterpret_cast<const uint32_t*>(row)[v];
    else
        return reinterpret_cast<const uint16_t*>(row)[v];
}
template <int TYPE>
__device__ inline float raw_as(uint32_t x) {
    if constexpr (TYPE == FLTOP_TYPE_F32) return __uint_as_float(x);
    if constexpr (TYPE == FLTOP_TYPE_BF16) return __uint_as_float(x << 16);
    return __half2float(__ushort_as_half((unsigned short)x));
}
__device__ inline float raw_value(uint32_t x, int32_t type) {
    const float half = __half2float(__ushort_as_half((unsigned short)x));
    return type == FLTOP_TYPE_F32 ? __uint_as_float(x) : type == FLTOP_TYPE_BF16 ? __uint_as_float(x << 16) : half;
}

__device__ inline float value_at(const char* row, int32_t v, int32_t type) {
    return raw_value(type == FLTOP_TYPE_F32 ? raw_at<FLTOP_TYPE_F32>(row, v) : raw_at<FLTOP_TYPE_F16>(row, v), type);
}

// An utterance's emissions.
struct Source {
    const char* rows;
    int64_t frame_bytes;
    int32_t type, V;
};

// A block's frames in the order in which a direction takes them.  Behind the end of an utterance that ends within the
// block lie frames in which the blank has probability 1 and all else 0: they leave every alignment's probability as
// it is, and stand where the backward direction begins.
template <int R>
struct Span {
    int32_t t0, end;
    bool reversed;
    __device__ int32_t frame(int f) const { return reversed ? t0 + R - 1 - f : t0 + f; }
    __device__ bool real(int f) const { return frame(f) < end; }
    __device__ const char* row(const Source& from, int f) const {   // of one behind the end, the last one
        return from.rows + (int64_t)min(frame(f), end - 1) * from.frame_bytes;
    }
};

// What the wavefront above needs of a block: the last lane's token mass before each frame.  (Below the first
// wavefront lies one without mass.)
template <int R>
struct alignas(8) Edge {
    double x[R];
    int32_t e[R];       // of x, if the block was gone through with aligned exponents; else E is
    int32_t E, least;   // the last lane's exponent, and the smallest that may reach it
    int32_t aligned;
};

// A workgroup's LDS: edges of each of its directions (`side`) and wavefronts (one below the first) for this turn and the one
// before; a place for what is written so that the lanes that have nothing to say need no branch; tables of exponentials of
// W + 1 blocks, and whether one of them is out of range.  In the middle, masses of U + 1 states in place of the last two.
template <int R, bool TABLE, int SIDES>
struct Lds {
    Edge<R>* edges;      // [SIDES][W + 1][2]
    int32_t* wide;       // [SIDES][W + 1]
    double* nowhere;     // [SIDES W][kWave + R]
    double* tables;      // [SIDES][W + 1][R][kTabulated]
    double* half_m;      // [U + 1]
    int32_t* half_e;
    int W;

    __device__ Lds(char* at, int waves, int32_t U) : W(waves) {
        edges = reinterpret_cast<Edge<R>*>(at);
        wide = reinterpret_cast<int32_t*>(edges + 2 * SIDES * (W + 1));
        nowhere = half_m = reinterpret_cast<double*>(wide + 2 * (W + 1));
        tables = nowhere + SIDES * W * (kWave + R);
        half_e = reinterpret_cast<int32_t*>(half_m + U + 1);
    }
    static size_t bytes(int W, int32_t U) {
        const size_t tables = TABLE ? SIDES * (W + 1) * R * kTabulated : 0;
        const size_t way = (SIDES * W * (kWave + R) + tables) * sizeof(double), half = SIDES == 2 ? (size_t)(U + 1) * 12 : 0;
        return 2 * SIDES * (W + 1) * sizeof(Edge<R>) + 2 * (W + 1) * sizeof(int32_t) + (way > half ? way : half);
    }
    __device__ Edge<R>& edge(int side, int wave_below, int turn) const {
        return edges[(side * (W + 1) + wave_below) * 2 + (turn & 1)];
    }
    __device__ int slot(int side, int32_t block) const { return side * (W + 1) + block % (W + 1); }
    __device__ double* table(int slot) const { return tables + slot * (R * kTabulated); }
};

// What a direction does in a launch.
struct Way {
    int32_t lo, hi;      // its frames
    bool reversed;
    int side;            // its part of the LDS
    Mark* marks;         // masses at the borders of blocks, [blocks][row] (or NULL), pair by pair as the direction sees them
    int32_t row;
};

// The part of the lattice that one lane holds.
template <int K, int R, bool TABLE>
struct Lane {
    static constexpr int kReach = (R + K - 1) / K;   // lanes that a block's masses can come from
    static constexpr int kSpread = 957 - 58 * R;

    double xb[K], xl[K];     // masses x * 2^E, or x * 2^eb and x * 2^el if not `common`
    int32_t E, eb[K], el[K];
    bool common;             // (alike in all lanes)
    int32_t tok[K];          // 0 behind the last token
    double skip[K];          // 1 where y_{i+1} != y_i, else 0
    double live[K];          // 1 for pairs with a token, else 0
    int32_t i0;              // first pair
    // Without a table: emissions of the next block as they lie in memory, those of the present one, the blank's of frame f
    // in lane f (mod R).
    uint32_t raw[TABLE ? 1 : R][K], raw_blank;
    float given[TABLE ? 1 : R][K], given_blank;

    __device__ bool start(const Hyp& y, int32_t V, bool reversed, int32_t first_pair) {
        bool fine = true;
        i0 = first_pair;
        E = 0;
        common = true;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int32_t i = i0 + k;
            tok[k] = i < y.L ? y.tokens[reversed ? y.L - 1 - i : i] : 0;
            const int32_t before = i > 0 && i < y.L ? y.tokens[reversed ? y.L - i : i - 1] : 0;
            skip[k] = i > 0 && i < y.L && tok[k] != before ? 1.0 : 0.0;
            live[k] = i < y.L ? 1.0 : 0.0;
            if (i < y.L && (tok[k] < 1 || tok[k] >= V)) {
                fine = false;
                tok[k] = 0;
            }
            xb[k] = i == 0 ? 1.0 : 0.0;
            xl[k] = 0.0;
            eb[k] = el[k] = 0;
        }
        return fine;
    }
    __device__ Mass blank_mass(int k) const { return normalized(xb[k], common ? E : eb[k]); }
    __device__ Mass token_mass(int k) const { return normalized(xl[k], common ? E : el[k]); }

    // Asks for a block's emissions.
    template <int TYPE>
    __device__ void ask_as(const Source& from, const Span<R>& span) {
#pragma unroll
        for (int f = 0; f < R; ++f) {
            const char* row = span.row(from, f);
#pragma unroll
            for (int k = 0; k < K; ++k) raw[TABLE ? 0 : f][k] = raw_at<TYPE>(row, tok[k]);
        }
        raw_blank = raw_at<TYPE>(span.row(from, threadIdx.x & (R - 1)), 0);
    }
    __device__ void ask(const Source& from, const Span<R>& span) {
        if (from.type == FLTOP_TYPE_F32)
            ask_as<FLTOP_TYPE_F32>(from, span);
        else
            ask_as<FLTOP_TYPE_F16>(from, span);   // 16 bits of either kind
    }
    template <int TYPE>
    __device__ void got_as() {
#pragma unroll
        for (int f = 0; f < R; ++f)
#pragma unroll
            for (int k = 0; k < K; ++k) given[TABLE ? 0 : f][k] = raw_as<TYPE>(raw[TABLE ? 0 : f][k]);
        given_blank = raw_as<TYPE>(raw_blank);
    }
    __device__ void got(int32_t type) {
        if (type == FLTOP_TYPE_F32)
            got_as<FLTOP_TYPE_F32>();
        else if (type == FLTOP_TYPE_BF16)
            got_as<FLTOP_TYPE_BF16>();
        else
            got_as<FLTOP_TYPE_F16>();
    }

    // Whether this lane's emissions of the block are in range.
    __device__ bool in_range(const double* table, const Span<R>& span) const {
        if constexpr (TABLE) {
            uint32_t most = 0, least = kMostWord;
#pragma unroll 1
            for (int f = 0; f < R; ++f)
#pragma unroll
                for (int k = -1; k < K; ++k) {
                    if (!span.real(f)) break;
                    const uint32_t w = high_word(table[f * kTabulated + (k < 0 ? 0 : tok[k < 0 ? 0 : k])]);
                    most = max(most, w);
                    least = min(least, w);
                }
            return least >= kLeastWord && most < kMostWord;
        } else {
            float most = given_blank, least = given_blank;
#pragma unroll
            for (int f = 0; f < R; ++f)
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    most = fmaxf(most, given[f][k]);
                    least = fminf(least, given[f][k]);
                }
            return least >= kLeastNear && most <= kMostNear;
        }
    }

    // The lane's exponent for a block, the smallest that may reach it, and the lane below's; returns whether the spread
    // is within bounds.
    __device__ bool enter(const Edge<R>& in, int32_t* to, int32_t* least, int32_t* below) const {
        int32_t top = kNoMass, low = -kNoMass;
        bool full = true;
#pragma unroll
        for (int k = 0; k < K; ++k) full &= xb[k] != 0.0 && (xl[k] != 0.0 || live[k] == 0.0);
        if (common) {
            uint32_t most = 0, few = UINT32_MAX;   // high words; less one, so that 0 is none
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const uint32_t a = high_word(xb[k]), c = high_word(xl[k]);
                most = max(most, max(a, c));
                few = min(few, min(a - 1, c - 1));
            }
            if (most != 0) {
                top = E + (int32_t)(most >> 20) - 1022;
                low = E + (int32_t)(few >> 20) - 1022;
            }
        } else {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int32_t a = xb[k] == 0.0 ? kNoMass : eb[k] + __builtin_amdgcn_frexp_exp(xb[k]);
                const int32_t c = xl[k] == 0.0 ? kNoMass : el[k] + __builtin_amdgcn_frexp_exp(xl[k]);
                top = max(top, max(a, c));
                low = min(low, min(a == kNoMass ? -kNoMass : a, c == kNoMass ? -kNoMass : c));
            }
        }
        int32_t m = top, n = low;
        const int32_t others = full ? -kNoMass : -2147483647 - 1;   // those of the lanes below count from here up
#pragma unroll
        for (int d = 0; d < kReach; ++d) {
            m = max(from_below(m, in.E), top);
            n = min(max(from_below(n, in.least), others), low);
        }
        *to = m;
        *least = n;
        *below = from_below(m, in.E);
        return m == kNoMass || m - n <= kSpread;
    }

    // Masses with the lane's new exponent.
    __device__ void rescale(int32_t to) {
        if (common) {
            const double by = rescaling(E - to);
#pragma unroll
            for (int k = 0; k < K; ++k) {
                xb[k] *= by;
                xl[k] *= by;
            }
        } else {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                xb[k] = ldexp(xb[k], eb[k] - to);
                xl[k] = ldexp(xl[k], el[k] - to);
            }
        }
        E = to;
        common = true;
    }
};

// Sums of v[0..R) over the wavefront, in a fixed order; lane f (mod R) returns that of v[f].  Each of the
// first steps halves the number of values that a lane carries.
template <int R>
__device__ inline double sums_by_lane(double (&v)[R]) {
    const int lane = threadIdx.x & (kWave - 1);
    int n = R;
#pragma unroll
    for (int o = 1; o < R; o <<= 1) {
        const bool upper = lane & o;
        n >>= 1;
#pragma unroll
        for (int j = 0; j < R / 2; ++j) {
            if (j >= n) break;
            // lanes without bit o keep the even places, lanes with it the odd ones
            const double keep = upper ? v[2 * j + 1] : v[2 * j];
            const double give = upper ? v[2 * j] : v[2 * j + 1];
            v[j] = keep + __shfl_xor(give, o, kWave);
        }
    }
#pragma unroll
    for (int o = R; o < kWave; o <<= 1) v[0] += __shfl_xor(v[0], o, kWave);
    return v[0];
}

// One block of frames for one wavefront.  `in`: from the wavefront below, `out`: for the one above.  AHEAD: a table's
// exponentials are read before all else, into registers.
template <int K, int R, bool TABLE, bool AHEAD>
__device__ inline void take_block(Lane<K, R, TABLE>& z, const Way& way, int32_t q, const double* table, bool wide,
                                  const Edge<R>& in, Edge<R>& out, double* nowhere, const Source& from) {
    const int lane = threadIdx.x & (kWave - 1);
    const Span<R> span = {q * R, way.hi, way.reversed};
    constexpr bool kRead = TABLE && AHEAD;
    double blanks[kRead ? R : 1], tokens[kRead ? R : 1][K];
    if constexpr (kRead) {
#pragma unroll
        for (int f = 0; f < R; ++f) {
            blanks[f] = table[f * kTabulated];
#pragma unroll
            for (int k = 0; k < K; ++k) tokens[f][k] = table[f * kTabulated + z.tok[k]];
        }
    }
    if (way.marks) {
        // (every lane has its place, with or without mass)
        Mark* const to = way.marks + (int64_t)q * way.row + z.i0;
#pragma unroll
        for (int k = 0; k < K; ++k)
            to[k] = {kept(z.xb[k], z.common ? z.E : z.eb[k]), kept(z.xl[k], z.common ? z.E : z.el[k])};
    }
    int32_t E, least, below;
    bool fine = z.enter(in, &E, &least, &below) && !in.aligned;
    if (!TABLE || wide) fine &= z.in_range(table, span);
    const bool near = __all(fine);
    if (lane == kWave - 1) {
        out.E = E;
        out.least = least;
        out.aligned = !near;
    }
    if (near) {
        // the lane below's scale in this one's
        const double fx = rescaling(below - E);
        const double fskip = fx * z.skip[0];
        double* const edge = lane == kWave - 1 ? out.x : nowhere + lane;
        z.rescale(E);
        double first[R];
#pragma unroll
        for (int f = 0; f < R; ++f) first[f] = in.x[f];
        double blank_by_lane = 0.0;
        if constexpr (!TABLE) blank_by_lane = span.real(lane & (R - 1)) ? exp_near(z.given_blank) : 1.0;
#pragma unroll
        for (int f = 0; f < R; ++f) {
            double pb;
            if constexpr (TABLE)
                pb = kRead ? blanks[kRead ? f : 0] : table[f * kTabulated];
            else
                pb = from_lane(blank_by_lane, f);
            edge[f] = z.xl[K - 1];
            const double moved = from_below(z.xl[K - 1], first[f]);
#pragma unroll
            for (int k = K - 1; k >= 0; --k) {
                const double prev = k > 0 ? z.xl[k > 0 ? k - 1 : 0] : moved;
                const double stay = fma(z.xb[k], z.live[k], z.xl[k]);
                const double l = fma(prev, k > 0 ? z.skip[k] : fskip, stay);
                const double b = k > 0 ? z.xb[k] + prev : fma(prev, fx, z.xb[k]);
                double p;
                if constexpr (TABLE)
                    p = kRead ? tokens[kRead ? f : 0][k] : table[f * kTabulated + z.tok[k]];
                else
                    p = masked(exp_near(z.given[TABLE ? 0 : f][k]), span.real(f) ? -1 : 0);
                z.xb[k] = b * pb;
                z.xl[k] = l * p;
            }
        }
    } else {
        Mass b[K], l[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            b[k] = z.blank_mass(k);
            l[k] = z.token_mass(k);
        }
        z.common = false;
#pragma unroll 1
        for (int f = 0; f < R; ++f) {
            // (frames behind the end too: the wavefront below may have gone through them as above, and has then given
            // up the masses of its tokens)
            const bool real = span.real(f);
            const char* emissions = span.row(from, f);
            const Mass blank = real ? mass_of(value_at(emissions, 0, from.type)) : Mass{1.0, 0};
            const Mass first = normalized(in.x[f], in.aligned ? in.e[f] : in.E);
            if (lane == kWave - 1) {
                out.x[f] = l[K - 1].m;
                out.e[f] = l[K - 1].e;
            }
            const Mass moved = {from_below(l[K - 1].m, first.m), from_below(l[K - 1].e, first.e)};
#pragma unroll
            for (int k = K - 1; k >= 0; --k) {
                const Mass prev = k > 0 ? l[k > 0 ? k - 1 : 0] : moved;
                Mass stay = plus(l[k], b[k]);
                if (z.skip[k] != 0.0) stay = plus(stay, prev);
                const Mass on = plus(b[k], prev);
                const Mass p = mass_of(value_at(emissions, z.tok[k], from.type));
                b[k] = normalized(on.m * blank.m, on.e + blank.e);
                l[k] = real && z.live[k] != 0.0 ? normalized(stay.m * p.m, stay.e + p.e) : no_mass();
            }
        }
#pragma unroll
        for (int k = 0; k < K; ++k) {
            z.xb[k] = b[k].m;
            z.eb[k] = b[k].e;
            z.xl[k] = l[k].m;
            z.el[k] = l[k].e;
        }
    }
}

// The blocks of a direction in the order in which it takes them, and the turns of the workgroup: wavefront w is w
// blocks behind its direction's first.
template <int R>
struct Blocks {
    int32_t first, count, turns;
    bool reversed;
    __device__ Blocks(const Way& way, const Way& other, int32_t used) : first(way.lo / R), reversed(way.reversed) {
        count = way.hi > way.lo ? (way.hi + R - 1) / R - first : 0;
        const int32_t others = other.hi > other.lo ? (other.hi + R - 1) / R - other.lo / R : 0;
        turns = max(count, others) + used - 1;
    }
    // (the last one again behind the end)
    __device__ int32_t operator[](int32_t n) const {
        n = min(n, count - 1);
        return reversed ? first + count - 1 - n : first + n;
    }
};

// The wavefront that tabulates: block n + 1 in turn n, asked for two turns before.
template <int R>
struct Tabulator {
    uint32_t raw[R];
    template <int TYPE>
    __device__ void ask_as(const Source& from, const Way& way, int32_t q) {
        const int32_t v = min((int32_t)(threadIdx.x & (kWave - 1)), from.V - 1);
        const Span<R> span = {q * R, way.hi, way.reversed};
#pragma unroll
        for (int f = 0; f < R; ++f) raw[f] = raw_at<TYPE>(span.row(from, f), v);
    }
    __device__ void ask(const Source& from, const Way& way, int32_t q) {
        if (from.type == FLTOP_TYPE_F32)
            ask_as<FLTOP_TYPE_F32>(from, way, q);
        else
            ask_as<FLTOP_TYPE_F16>(from, way, q);
    }
    template <int TYPE>
    __device__ void put_as(double* table, int32_t* wide, const Span<R>& span) {
        const int lane = threadIdx.x & (kWave - 1);
        float most = raw_as<TYPE>(raw[0]), least = most;
#pragma unroll
        for (int f = 0; f < R; ++f) {
            const float lp = raw_as<TYPE>(raw[f]);
            most = fmaxf(most, lp);
            least = fminf(least, lp);
            table[f * kTabulated + lane] = exp_any(lp);
            if (!span.real(f)) table[f * kTabulated + lane] = lane == 0 ? 1.0 : 0.0;
        }
        const bool all = __all(least >= kLeastNear && most <= kMostNear);
        if (lane == 0) *wide = !all;
    }
    __device__ void put(const Source& from, double* table, int32_t* wide, const Span<R>& span) {
        if (from.type == FLTOP_TYPE_F32)
            put_as<FLTOP_TYPE_F32>(table, wide, span);
        else if (from.type == FLTOP_TYPE_BF16)
            put_as<FLTOP_TYPE_BF16>(table, wide, span);
        else
            put_as<FLTOP_TYPE_F16>(table, wide, span);
    }
};

template <int R, int SIDES>
__device__ inline void tabulate_all(const Way& way, const Way& other, const Source& from, int32_t used,
                                    const Lds<R, true, SIDES>& lds) {
    const Blocks<R> blocks(way, other, used);
    Tabulator<R> even, odd;
    auto put = [&](Tabulator<R>& one, int32_t n) {
        const int slot = lds.slot(way.side, n);
        one.put(from, lds.table(slot), lds.wide + slot, Span<R>{blocks[n] * R, way.hi, way.reversed});
    };
    if (blocks.count > 0) {
        even.ask(from, way, blocks[0]);
        odd.ask(from, way, blocks[1]);
        put(even, 0);
        even.ask(from, way, blocks[2]);
    }
    __syncthreads();
    for (int32_t turn = 0; turn < blocks.turns; turn += 2) {
        if (turn + 1 < blocks.count) {
            put(odd, turn + 1);
            odd.ask(from, way, blocks[turn + 3]);
        }
        __syncthreads();
        if (turn + 1 >= blocks.turns) break;
        if (turn + 2 < blocks.count) {
            put(even, turn + 2);
            even.ask(from, way, blocks[turn + 4]);
        }
        __syncthreads();
    }
}

// A wavefront's blocks.
template <int K, int R, bool TABLE, bool AHEAD, int SIDES>
__device__ inline void take_all(Lane<K, R, TABLE>& z, const Way& way, const Way& other, const Source& from, int wave,
                                int32_t used, const Lds<R, TABLE, SIDES>& lds) {
    double* const nowhere = lds.nowhere + (way.side * lds.W + wave) * (kWave + R);
    if (wave == 0 && threadIdx.x % kWave < 2 * R) {   // nothing comes from below the first
        const int32_t f = threadIdx.x & (R - 1);
        Edge<R>& none = lds.edge(way.side, 0, threadIdx.x % kWave / R);
        none.x[f] = 0.0;
        none.e[f] = kNoMass;
        none.E = kNoMass;
        none.least = -kNoMass;
        none.aligned = 0;
    }
    const Blocks<R> blocks(way, other, used);
    auto ask = [&](int32_t n) {
        if constexpr (!TABLE) z.ask(from, Span<R>{blocks[n] * R, way.hi, way.reversed});
    };
    const bool works = wave < used && blocks.count > 0;
    if (works) ask(0);
    __syncthreads();
    // (three loops: with the idle turns in the loop of the blocks, a wait for a load would count on no store behind it)
    const int32_t before = works ? wave : blocks.turns, after = works ? wave + blocks.count : blocks.turns;
    for (int32_t turn = 0; turn < before; ++turn) __syncthreads();
    for (int32_t turn = before; turn < after; ++turn) {
        const int32_t n = turn - wave;
        bool wide = true;
        const double* table = nullptr;
        if constexpr (TABLE) {
            const int slot = lds.slot(way.side, n);
            wide = __builtin_amdgcn_readfirstlane(lds.wide[slot]);
            table = lds.table(slot);
        } else {
            z.got(from.type);
            ask(n + 1);
        }
        take_block<K, R, TABLE, AHEAD>(z, way, blocks[n], table, wide, lds.edge(way.side, wave, turn - 1),
                                lds.edge(way.side, wave + 1, turn), nowhere, from);
        __syncthreads();
    }
    for (int32_t turn = after; turn < blocks.turns; ++turn) __syncthreads();
}

// The emissions of utterance b.
__device__ inline Source source_of(const fltop_rows& x, int32_t b) {
    const int32_t bytes = x.type == FLTOP_TYPE_F32 ? 4 : 2;
    return {static_cast<const char*>(x.data) + b * x.batch_stride * bytes, x.frame_stride * bytes, x.type, x.V};
}

// Where the two directions of a first half meet: frames [0, middle) are the forward one's.
template <int R>
__host__ __device__ inline int32_t middle_of(int32_t frames) {
    const int32_t h = (frames / 2 + R - 1) / R * R;
    return h < frames ? h : frames;
}

// A wavefront's part in its workgroup: of each of its directions W wavefronts, then one that tabulates for them.
template <int K, bool TABLE, int SIDES>
struct Role {
    int W, wave, side, lane;
    bool tabulates;
    __device__ Role() {
        const int n = (int)blockDim.x / kWave / SIDES;   // of a direction
        const int all = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
        W = TABLE ? n - 1 : n;
        side = SIDES == 2 && all >= n ? 1 : 0;
        wave = all - side * n;
        tabulates = TABLE && wave == W;
        lane = threadIdx.x & (kWave - 1);
    }
    __device__ int32_t first_pair() const { return (wave * kWave + lane) * K; }
};

// Scores, both directions of a hypothesis in a workgroup.  With ONE, a direction: scores by the forward one, all the way;
// where a gradient is wanted (`ws`), the backward one has a workgroup too, and both leave the masses at the borders of
// blocks.
template <int K, int R, int WAVES, int THREADS, bool TABLE, bool ONE>
__global__ __launch_bounds__(THREADS) __attribute__((amdgpu_waves_per_eu(WAVES))) void score_kernel(
    fltop_rows x, fltop_hypotheses h, double* out_scores, ScoreSpace ws) {
    constexpr int kSides = ONE ? 1 : 2;
    extern __shared__ char dynamic[];
    __shared__ Mass sums[kMostWaves];
    __shared__ Mass last[kMostWaves];
    const bool keep = ONE && ws.marks != nullptr;
    const int64_t at = keep ? blockIdx.x / 2 : blockIdx.x;
    const int32_t b = (int32_t)(at / h.N), n = (int32_t)(at % h.N);
    const Hyp y = hypothesis(x, h, b, n);
    const Role<K, TABLE, kSides> role;
    const Lds<R, TABLE, kSides> lds(dynamic, role.W, h.U);
    const bool reversed = keep ? blockIdx.x % 2 : role.side;
    Lane<K, R, TABLE> z;
    // (the lanes of a wavefront that tabulates lie behind the last pair)
    const bool fine = y.L >= 0 && z.start(y, x.V, reversed, role.tabulates ? y.L + 1 : role.first_pair());
    if (__syncthreads_or(!fine)) {
        if (threadIdx.x == 0 && !(ONE && reversed)) {
            out_scores[at] = y.L == -2 ? NAN : -INFINITY;
            if (keep) ws.total_m[at] = 0.0, ws.total_e[at] = kNoMass;
        }
        return;
    }
    const int32_t used = y.L / (kWave * K) + 1;
    const int32_t middle = middle_of<R>(y.frames);
    const Way way = {!ONE && reversed ? middle : 0, ONE || reversed ? y.frames : middle, reversed, role.side,
                     keep ? ws.marks + (at * 2 + reversed) * ws.marks_of : nullptr, (int32_t)ws.row};
    const Way other =
        ONE ? way : Way{reversed ? 0 : middle, reversed ? middle : y.frames, !reversed, 1 - role.side, nullptr, 0};
    if (role.tabulates) {
        if constexpr (TABLE) tabulate_all<R, kSides>(way, other, source_of(x, b), used, lds);
    } else {
        take_all<K, R, TABLE, K == 2 && WAVES == 3, kSides>(z, way, other, source_of(x, b), role.wave, used, lds);
    }
    if constexpr (ONE) {
        // P = b_L + l_{L-1} after the last frame
        if (reversed) return;
        if (!role.tabulates) {
            Mass end = no_mass();
#pragma unroll
            for (int k = 0; k < K; ++k) {
                if (z.i0 + k == y.L) end = plus(end, z.blank_mass(k));
                if (z.i0 + k == y.L - 1) end = plus(end, z.token_mass(k));
                end = normalized(end.m, end.e);
            }
            if (z.i0 <= y.L && y.L < z.i0 + K) sums[0] = end;
            if (z.i0 <= y.L - 1 && y.L - 1 < z.i0 + K && !(z.i0 <= y.L && y.L < z.i0 + K)) sums[1] = end;
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            // (both states may be one lane's)
            Mass p = y.L % K != 0 || y.L == 0 ? sums[0] : plus(sums[0], sums[1]);
            p = normalized(p.m, p.e);
            out_scores[at] = ln_of(p);
            if (keep) {
                ws.total_m[at] = p.m;
                ws.total_e[at] = p.e;
            }
        }
        return;
    }

    // P = sum over states of the forward mass after frame middle - 1 and the backward bracket at that frame
    const bool back = reversed && !role.tabulates, fore = !reversed && !role.tabulates;
    if (back && role.lane == kWave - 1) last[role.wave] = z.token_mass(K - 1);
    __syncthreads();
    Mass on[K], stay[K], sum = no_mass();
    if (back) {
        const Mass first = role.wave > 0 ? last[role.wave - 1] : no_mass();
        const Mass top = z.token_mass(K - 1);
        const Mass moved = {from_below(top.m, first.m), from_below(top.e, first.e)};
#pragma unroll
        for (int k = K - 1; k >= 0; --k) {
            const Mass prev = k > 0 ? z.token_mass(k > 0 ? k - 1 : 0) : moved, blank = z.blank_mass(k);
            stay[k] = plus(z.token_mass(k), blank);
            if (z.skip[k] != 0.0) stay[k] = plus(stay[k], prev);
            on[k] = plus(blank, prev);
        }
    }
#pragma unroll
    for (int part = 0; part < 2; ++part) {   // blanks, then tokens
        if (fore) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int32_t i = z.i0 + k;
                const Mass m = part ? z.token_mass(k) : z.blank_mass(k);
                if (i < y.L + 1 - part) {
                    lds.half_m[i] = m.m;
                    lds.half_e[i] = m.e;
                }
            }
        }
        __syncthreads();
        if (back) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int32_t i = z.i0 + k;
                if (i >= y.L + 1 - part) continue;
                const Mass m = part ? stay[k] : on[k];
                const int32_t s = y.L - part - i;
                sum = plus(sum, normalized(lds.half_m[s] * m.m, max(lds.half_e[s] + m.e, kNoMass)));
            }
        }
        __syncthreads();
    }
    if (back) {
        int32_t e = sum.e;
#pragma unroll
        for (int o = kWave / 2; o > 0; o >>= 1) e = max(e, __shfl_xor(e, o, kWave));
        double m = ldexp(sum.m, sum.e - e);
#pragma unroll
        for (int o = kWave / 2; o > 0; o >>= 1) m += __shfl_xor(m, o, kWave);
        if (role.lane == 0) sums[role.wave] = normalized(m, e);
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        Mass p = no_mass();
        for (int w = 0; w < role.W; ++w) {
            p = plus(p, sums[w]);
            p = normalized(p.m, p.e);
        }
        out_scores[at] = ln_of(p);
    }
}

// ---- the gradient -----------------------------------------------------------------------------------
//
// A workgroup takes one block of R frames of an utterance, and its wavefronts that block's hypotheses, each in chunks
// of kWave K pairs: forwards from the masses at the block's lower border, with the masses after each frame in registers;
// then backwards from those at the upper border, both in the same lanes.  Within a block a mass goes R pairs far, so
// chunks that overlap by 2 R pairs need nothing from each other.  Occupancies are added to rows of V sums in LDS, as
// whole numbers: in any order the same.  One exponent for each lane does wherever P's is within reach of it (kMostShift).
//
// About a thousand vector instructions a chunk and block, and loads of the borders that depend on the hypothesis's length,
// which is loaded before: 64 transcripts of 500 frames take 26 us, 256 of up to 1500 frames 252 us, in two thirds of
// which the SIMDs issue a vector instruction; the borders' 0.36 GB alone are 73 us.  Four wavefronts a SIMD, the most that
// registers allow, are worth more than a few spills.

constexpr int kGradPairs = 2, kGradThreads = 256;   // (at most)

__device__ inline int32_t from_above(int32_t x, int32_t last) {
    return __builtin_amdgcn_update_dpp(last, x, 0x130, 0xf, 0xf, false);  // wave_shl:1
}
__device__ inline double from_above(double x) {
    const long long a = __double_as_longlong(x);
    return from_words(from_above((int32_t)(a >> 32), 0), from_above((int32_t)a, 0));
}

// 2^c by which the product of two masses of exponents that add up to c becomes an occupancy, less that of P.  Masses are
// below 2^128 in these exponents, so that an occupancy of weight (2^-50 up) has c > -306, and with c up to kMostShift
// both its masses are above 2^-678: what leaves the range of fp64 has none, nor has what passes an emission below e^-600,
// for which exp_any gives that.
constexpr int32_t kMostShift = 500;
__device__ inline int32_t share_shift(int32_t Ef, int32_t Eb, int32_t total) {
    if (Ef <= kNoMass || Eb <= kNoMass) return -2000;
    const long long c = (long long)Ef + Eb - total;
    return (int32_t)(c < -2000 ? -2000 : c > kMostShift ? kMostShift + 1 : c);
}

// A lane's pairs of one chunk.
template <int K, int R>
struct Chunk {
    int32_t tok[K], i0, L;
    double skip[K], skip_up[K], live[K];   // skip_up: of the pair above
    Mass fb[K], fl[K], bb[K], bl[K];       // masses at the lower border (forwards) and the upper one (backwards)

    __device__ Chunk(const Hyp& y, const ScoreSpace& ws, int64_t at, int32_t V, int32_t q, int32_t first_pair)
        : i0(first_pair + (int32_t)(threadIdx.x & (kWave - 1)) * K), L(y.L) {
        const Mark* const fore = ws.marks + at * 2 * ws.marks_of + q * ws.row;
        const Mark* const back = fore + ws.marks_of;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int32_t i = i0 + k;
            // pairs below the first and behind the last have no mass
            const bool blank = i >= 0 && i <= L, token = i >= 0 && i < L;
            const int32_t one = token ? y.tokens[i] : 0, before = token && i > 0 ? y.tokens[i - 1] : 0;
            const int32_t next = i >= -1 && i + 1 < L ? y.tokens[i + 1] : 0;
            tok[k] = (uint32_t)one < (uint32_t)V ? one : 0;   // (the hypotheses that were scored have no other)
            skip[k] = token && i > 0 && one != before ? 1.0 : 0.0;
            skip_up[k] = i >= 0 && i + 1 < L && next != one ? 1.0 : 0.0;
            live[k] = token ? 1.0 : 0.0;
            // backwards, pair j is blank L - j and token L - 1 - j
            const Mark f = fore[min(max(i, 0), L)], u = back[min(max(L - i, 0), L)], v = back[min(max(L - 1 - i, 0), L)];
            fb[k] = blank ? mass_of(f.b) : no_mass();
            fl[k] = token ? mass_of(f.l) : no_mass();
            bb[k] = blank ? mass_of(u.b) : no_mass();
            bl[k] = token ? mass_of(v.l) : no_mass();
        }
    }

    // One exponent for the lane's masses and those that may reach it, and that of the lane which they come from.  From a mass
    // at one border to the one at the other that an alignment goes on with it is R + 1 pairs, a step for each frame and one
    // to the frame behind: every lane on that way counts both, so that none of them takes an exponent by what is of no
    // use to the alignment and finds its masses too small to hold, while no sum of exponents tells of it.
    template <bool UP>
    __device__ static void window(const Mass (&b)[K], const Mass (&l)[K], int32_t* E, int32_t* beside) {
        int32_t top = kNoMass;
#pragma unroll
        for (int k = 0; k < K; ++k) top = max(top, max(b[k].e, l[k].e));
        int32_t m = top;
#pragma unroll
        for (int d = 0; d < (R + K) / K; ++d) m = max(UP ? from_below(m, kNoMass) : from_above(m, kNoMass), top);
        *E = m;
        *beside = UP ? from_below(m, kNoMass) : from_above(m, kNoMass);
    }

    // One frame forwards / the bracket of one frame backwards, with aligned exponents.
    __device__ void forward(Mass (&b)[K], Mass (&l)[K], const char* row, int32_t type) const {
        const Mass blank = mass_of(value_at(row, 0, type));
        const Mass moved = {from_below(l[K - 1].m, 0.0), from_below(l[K - 1].e, kNoMass)};
#pragma unroll
        for (int k = K - 1; k >= 0; --k) {
            const Mass prev = k > 0 ? l[k > 0 ? k - 1 : 0] : moved;
            Mass stay = plus(l[k], b[k]);
            if (skip[k] != 0.0) stay = plus(stay, prev);
            const Mass on = plus(b[k], prev), p = mass_of(value_at(row, tok[k], type));
            b[k] = normalized(on.m * blank.m, on.e + blank.e);
            l[k] = live[k] != 0.0 ? normalized(stay.m * p.m, stay.e + p.e) : no_mass();
        }
    }
    __device__ void bracket(Mass (&b)[K], Mass (&l)[K]) const {
        const Mass up_b = {from_above(b[0].m), from_above(b[0].e, kNoMass)};
        const Mass up_l = {from_above(l[0].m), from_above(l[0].e, kNoMass)};
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const Mass nb = k + 1 < K ? b[k + 1 < K ? k + 1 : 0] : up_b, nl = k + 1 < K ? l[k + 1 < K ? k + 1 : 0] : up_l;
            const Mass blank = plus(b[k], l[k]);
            Mass token = plus(l[k], nb);
            if (skip_up[k] != 0.0) token = plus(token, nl);
            b[k] = normalized(blank.m, blank.e);
            l[k] = live[k] != 0.0 ? normalized(token.m, token.e) : no_mass();
        }
    }
};

constexpr double kOne = 1125899906842624.0;       // 2^50
constexpr double kShift = 6755399441055744.0;     // 1.5 * 2^52: its last bit is worth one

__device__ inline void add_share(unsigned long long* sum, double share) {
    const long long a = __double_as_longlong(share + kShift) - __double_as_longlong(kShift);
    atomicAdd(sum, (unsigned long long)a);
}

// The pairs own_first .. own_last with aligned exponents, a pair a lane so that few registers are needed, and forwards
// once more for each frame.
template <int R>
__device__ inline void aligned_chunk(const Hyp& y, const ScoreSpace& ws, int64_t at, const Source& from, int32_t t0, int32_t q,
                                     int32_t nf, int32_t own_first, int32_t own_last, int32_t total_e, double w, int32_t v0,
                                     int32_t v1, unsigned long long* sums, int32_t width) {
    const int lane = threadIdx.x & (kWave - 1);
    constexpr int32_t kStep = kWave - 2 * R;
#pragma unroll 1
    for (int32_t c = own_first; c <= own_last; c += kStep) {
        const Chunk<1, R> z(y, ws, at, from.V, q, c - R);
        const bool own = z.i0 >= c && z.i0 < c + kStep && z.i0 <= own_last;
        Mass ub[1] = {z.bb[0]}, ul[1] = {z.bl[0]};
#pragma unroll 1
        for (int f = nf - 1; f >= 0; --f) {
            Mass kb[1] = {z.fb[0]}, kl[1] = {z.fl[0]};
#pragma unroll 1
            for (int g = 0; g <= f; ++g) z.forward(kb, kl, from.rows + (int64_t)(t0 + g) * from.frame_bytes, from.type);
            z.bracket(ub, ul);
            const char* row = from.rows + (int64_t)(t0 + f) * from.frame_bytes;
            double blank = own ? ldexp(kb[0].m * ub[0].m, kb[0].e + ub[0].e - total_e) : 0.0;
            const int32_t v = z.tok[0] - v0;
            if (own && z.live[0] != 0.0 && (uint32_t)v < (uint32_t)(v1 - v0))
                add_share(&sums[f * width + v], ldexp(kl[0].m * ul[0].m, kl[0].e + ul[0].e - total_e) * w);
            const Mass pb = mass_of(value_at(row, 0, from.type)), p = mass_of(value_at(row, z.tok[0], from.type));
            ub[0] = normalized(ub[0].m * pb.m, ub[0].e + pb.e);
            ul[0] = normalized(ul[0].m * p.m, ul[0].e + p.e);
            for (int o = kWave / 2; o > 0; o >>= 1) blank += __shfl_xor(blank, o, kWave);
            if (v0 == 0 && lane == 0) add_share(&sums[f * width], blank * w);
        }
    }
}

template <typename T, int R, bool TABLE>
__global__ __launch_bounds__(kGradThreads, TABLE ? 4 : 2) void score_grad_kernel(fltop_rows x, fltop_hypotheses h,
                                                                  const double* grad_scores, ScoreSpace ws, int32_t blocks,
                                                                  int32_t parts, T* grad) {
    constexpr int K = kGradPairs;
    const int kWaves = (int)blockDim.x / kWave;
    constexpr int kPairs = kWave * K, kStep = kPairs - 2 * R;   // of a chunk, and from one to the next
    extern __shared__ char dynamic[];
    __shared__ double of_wave[kGradThreads / kWave];
    __shared__ int32_t flags[kGradThreads / kWave];   // weights that are no numbers, emissions out of range
    // the vocabulary is taken in `parts` ranges where a block's sums would not fit
    const int32_t width = (x.V + parts - 1) / parts;
    unsigned long long* const sums = reinterpret_cast<unsigned long long*>(dynamic);   // [R][width]
    double* const table = reinterpret_cast<double*>(sums + R * width);                 // [R][kTabulated]
    const int lane = threadIdx.x & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    const int64_t group = blockIdx.x / parts;
    const int32_t v0 = (int32_t)(blockIdx.x % parts) * width, v1 = min(v0 + width, x.V);
    const int32_t b = (int32_t)(group / blocks), q = (int32_t)(group % blocks), t0 = q * R;
    const int32_t rows = min(R, x.T - t0);
    T* const out = grad + ((int64_t)b * x.T + t0) * x.V;
    const Source from = source_of(x, b);
    const int32_t frames = __builtin_amdgcn_readfirstlane(max(min(x.lengths[b], x.T), 0)), nf = min(R, frames - t0);
    if (nf <= 0) {   // (nothing behind the end of an utterance is read)
        for (int32_t f = 0; f < rows; ++f)
            for (int32_t v = v0 + threadIdx.x; v < v1; v += blockDim.x) out[(int64_t)f * x.V + v] = from_float<T>(0.0f);
        return;
    }
    // (all of what the following loads fetch is asked for before any of it is waited for)
    uint32_t block_raw[TABLE ? R : 1];
    if constexpr (TABLE) {
#pragma unroll
        for (int j = 0; j < R; ++j) {
            if (j * kWaves >= R) break;
            const int32_t f = min(j * kWaves + wave, nf - 1), v = min(lane, x.V - 1);
            const char* row = from.rows + (int64_t)(t0 + f) * from.frame_bytes;
            block_raw[j] = x.type == FLTOP_TYPE_F32 ? raw_at<FLTOP_TYPE_F32>(row, v) : raw_at<FLTOP_TYPE_F16>(row, v);
        }
    }
    double most = 0.0;
    bool odd = false, near = true;
    for (int32_t n = threadIdx.x; n < h.N; n += blockDim.x) {
        const int64_t at = (int64_t)b * h.N + n;
        const double w = fabs(grad_scores[at]);
        if (ws.total_e[at] <= kNoMass) continue;
        odd |= !(w <= 1.7976931348623157e308);
        most = fmax(most, w);
    }
    for (int32_t i = threadIdx.x; i < R * width; i += blockDim.x) sums[i] = 0;
    if constexpr (TABLE) {
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int32_t f = j * kWaves + wave;
            if (f >= R) break;
            const float lp = raw_value(block_raw[j], x.type);
            near &= lp <= kMostNear || f >= nf;
            table[f * kTabulated + lane] = f < nf ? exp_any(lp) : lane == 0 ? 1.0 : 0.0;
        }
    }
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) most = fmax(most, __shfl_xor(most, o, kWave));
    const int32_t flag = (__any(odd) ? 1 : 0) | (__all(near) ? 0 : 2);
    if (lane == 0) {
        of_wave[wave] = most;
        flags[wave] = flag;
    }
    __syncthreads();
    int32_t any = 0;
    for (int w = 0; w < kWaves; ++w) {
        most = fmax(most, of_wave[w]);
        any |= flags[w];
    }
    odd = any & 1;
    const bool wide = any & 2;
    if (odd || most == 0.0) {
        for (int32_t f = 0; f < rows; ++f)
            for (int32_t v = v0 + threadIdx.x; v < v1; v += blockDim.x)
                out[(int64_t)f * x.V + v] = from_float<T>(odd && f < nf ? NAN : 0.0f);
        return;
    }
    int32_t task = 0;   // chunks of hypotheses, one wavefront after the other
    for (int32_t n = 0; n < h.N; ++n) {
        const int64_t at = (int64_t)b * h.N + n;
        const int32_t total_e = __builtin_amdgcn_readfirstlane(ws.total_e[at]);
        if (total_e <= kNoMass) continue;
        const Hyp y = hypothesis(x, h, b, n);
        const double w = grad_scores[at] / most * (kOne / ws.total_m[at]);
        if (y.L < 0) continue;
        // one chunk if the pairs fit, else chunks of which R pairs at either end are only passed through
        const bool one = y.L + 1 <= kPairs;
        const int32_t chunks = one ? 1 : (y.L + kStep) / kStep;
        for (int32_t c = 0; c < chunks; ++c, ++task) {
            if (task % kWaves != wave) continue;
            const int32_t first = one ? 0 : c * kStep - R;
            const Chunk<K, R> z(y, ws, at, x.V, q, first);
            // the chunk's own pairs, and whether they are this lane's
            const int32_t own_first = one ? 0 : c * kStep, own_last = one ? y.L : min(y.L, (c + 1) * kStep - 1);
            bool own[K];
#pragma unroll
            for (int k = 0; k < K; ++k) own[k] = z.i0 + k >= own_first && z.i0 + k <= own_last;
            int32_t Ef, Eb, below, above;
            Chunk<K, R>::template window<true>(z.fb, z.fl, &Ef, &below);
            Chunk<K, R>::template window<false>(z.bb, z.bl, &Eb, &above);
            const int32_t shift = share_shift(Ef, Eb, total_e);
            bool fine = shift <= kMostShift;
            // emissions
            uint32_t raw[TABLE ? 1 : R][K], raw_blank = 0;
            if constexpr (!TABLE) {
#pragma unroll
                for (int f = 0; f < R; ++f) {
                    const char* row = from.rows + (int64_t)(t0 + min(f, nf - 1)) * from.frame_bytes;
#pragma unroll
                    for (int k = 0; k < K; ++k)
                        raw[f][k] = x.type == FLTOP_TYPE_F32 ? raw_at<FLTOP_TYPE_F32>(row, z.tok[k])
                                                             : raw_at<FLTOP_TYPE_F16>(row, z.tok[k]);
                }
                const char* row = from.rows + (int64_t)(t0 + min((int32_t)(lane & (R - 1)), nf - 1)) * from.frame_bytes;
                raw_blank = x.type == FLTOP_TYPE_F32 ? raw_at<FLTOP_TYPE_F32>(row, 0) : raw_at<FLTOP_TYPE_F16>(row, 0);
                fine &= raw_value(raw_blank, x.type) <= kMostNear;
#pragma unroll
                for (int f = 0; f < R; ++f)
#pragma unroll
                    for (int k = 0; k < K; ++k) fine &= raw_value(raw[f][k], x.type) <= kMostNear;
            } else {
                fine &= !wide;
            }
            if (__all(fine)) {
                double blanks[R];
                double p[TABLE ? 1 : R][K], pb[TABLE ? 1 : R];   // (a table is read again)
                double blank_by_lane = 0.0;
                if constexpr (!TABLE) blank_by_lane = exp_any(raw_value(raw_blank, x.type));
                if constexpr (!TABLE) {
#pragma unroll
                    for (int f = 0; f < R; ++f) {
                        pb[f] = f < nf ? from_lane(blank_by_lane, f) : 1.0;
#pragma unroll
                        for (int k = 0; k < K; ++k) p[f][k] = f < nf ? exp_any(raw_value(raw[f][k], x.type)) : 0.0;
                    }
                }
                auto blank_p = [&](int f) { return TABLE ? table[f * kTabulated] : pb[TABLE ? 0 : f]; };
                auto token_p = [&](int f, int k) { return TABLE ? table[f * kTabulated + z.tok[k]] : p[TABLE ? 0 : f][k]; };
                const double fx = rescaling(below - Ef), fskip = fx * z.skip[0];
                const double gx = rescaling(above - Eb), gskip = gx * z.skip_up[K - 1];
                double xb[K], xl[K], ub[K], ul[K], kb[R][K], kl[R][K];
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    xb[k] = ldexp(z.fb[k].m, z.fb[k].e - Ef);
                    xl[k] = ldexp(z.fl[k].m, z.fl[k].e - Ef);
                    ub[k] = ldexp(z.bb[k].m, z.bb[k].e - Eb);
                    ul[k] = ldexp(z.bl[k].m, z.bl[k].e - Eb);
                }
                auto forward = [&](int f) {
                    const double moved = from_below(xl[K - 1], 0.0);
#pragma unroll
                    for (int k = K - 1; k >= 0; --k) {
                        const double prev = k > 0 ? xl[k > 0 ? k - 1 : 0] : moved;
                        const double stay = fma(xb[k], z.live[k], xl[k]);
                        const double l = fma(prev, k > 0 ? z.skip[k] : fskip, stay);
                        const double on = k > 0 ? xb[k] + prev : fma(prev, fx, xb[k]);
                        kb[f][k] = xb[k] = on * blank_p(f);
                        kl[f][k] = xl[k] = l * token_p(f, k);
                    }
                };
                const double factor = shift < -1000 ? 0.0 : power_of_two(min(shift, kMostShift));
                auto backward = [&](int f) {
                    const double up_b = from_above(ub[0]), up_l = from_above(ul[0]);
                    blanks[f] = 0.0;
#pragma unroll
                    for (int k = 0; k < K; ++k) {
                        const double nb = k + 1 < K ? ub[k + 1 < K ? k + 1 : 0] : up_b * gx;
                        const double nl = k + 1 < K ? ul[k + 1 < K ? k + 1 : 0] : up_l;
                        const double blank = ub[k] + ul[k];
                        const double token =
                            fma(nl, k + 1 < K ? z.skip_up[k] : gskip, fma(nb, z.live[k], ul[k]));
                        const double sb = kb[f][k] * factor * blank, sl = kl[f][k] * factor * token;
                        blanks[f] += own[k] ? sb : 0.0;
                        const int32_t v = z.tok[k] - v0;
                        if (own[k] && z.live[k] != 0.0 && (uint32_t)v < (uint32_t)(v1 - v0))
                            add_share(&sums[f * width + v], sl * w);
                        ub[k] = blank * blank_p(f);
                        ul[k] = token * token_p(f, k);
                    }
                };
#pragma unroll
                for (int f = 0; f < R; ++f) forward(f);
#pragma unroll
                for (int f = R - 1; f >= 0; --f) backward(f);
                const double sum = sums_by_lane<R>(blanks);
                if (v0 == 0 && lane < nf) add_share(&sums[lane * width], sum * w);
            } else {
                aligned_chunk<R>(y, ws, at, from, t0, q, nf, own_first, own_last, total_e, w, v0, v1, sums, width);
            }
        }
    }
    __syncthreads();
    for (int32_t f = 0; f < rows; ++f)
        for (int32_t v = v0 + threadIdx.x; v < v1; v += blockDim.x)
            out[(int64_t)f * x.V + v] =
                from_float<T>(f < nf ? (float)((double)(long long)sums[f * width + v - v0] * (most / kOne)) : 0.0f);
}

// Pairs of a lane, wavefronts of a direction (at most), frames of a block, wavefronts a SIMD has registers for.
template <int K, int MOST, int R, int WAVES, bool TABLE, bool ONE>
hipError_t score_with(const fltop_rows& x, const fltop_hypotheses& h, double* out_scores, const ScoreSpace* keep,
                      hipStream_t stream) {
    constexpr int kSides = ONE ? 1 : 2, kThreads = kWave * kSides * (MOST + (TABLE ? 1 : 0));
    const int W = waves_for(h.U, K);
    const unsigned hyps = (unsigned)(x.B * h.N), threads = kWave * kSides * (TABLE ? W + 1 : W);
    const size_t bytes = Lds<R, TABLE, kSides>::bytes(W, h.U);
    hipLaunchKernelGGL((score_kernel<K, R, WAVES, kThreads, TABLE, ONE>), dim3(keep ? 2 * hyps : hyps), dim3(threads), bytes,
                       stream, x, h, out_scores, keep ? *keep : ScoreSpace{});
    return hipGetLastError();
}

template <bool TABLE>
hipError_t score_as(const fltop_rows& x, const fltop_hypotheses& h, double* out_scores, const ScoreSpace* keep,
                    hipStream_t stream) {
    // Registers for three wavefronts a SIMD, so that a table's exponentials can be read ahead, where a direction has four at
    // most and the hypotheses do not fill the chip twice (64 transcripts of 229 tokens: 79 us, 86 with the other build); else
    // for four (2048 hypotheses of 229: 269 us, 345 with the first).  This and all that follows goes by the room for tokens,
    // which the host knows, not by the hypotheses' lengths, which it does not.
    const bool few = h.U < 512 && (int64_t)x.B * h.N < 512;
    if (!keep && h.U < 896) {
        if (few) return score_with<2, 4, 8, 3, TABLE, false>(x, h, out_scores, keep, stream);
        return score_with<2, 7, 8, 4, TABLE, false>(x, h, out_scores, keep, stream);
    }
    // Two directions in a workgroup have no place for more than 1024 pairs of two a lane, so four (16 transcripts of 1000
    // tokens over 2400 frames: 0.9 ms, 2.5 ms with one direction all the way); longer ones go one way.
    if (!keep && h.U < 1024) return score_with<4, 4, 4, 3, TABLE, false>(x, h, out_scores, keep, stream);
    if (lattice_pairs(h.U) == 4) return score_with<4, 16, 4, 4, false, true>(x, h, out_scores, keep, stream);
    if (few) return score_with<2, 4, 8, 3, TABLE, true>(x, h, out_scores, keep, stream);
    return score_with<2, 15, 8, 4, TABLE, true>(x, h, out_scores, keep, stream);
}

template <typename T, int R, bool TABLE>
hipError_t grad_as(const fltop_rows& x, const fltop_hypotheses& h, const double* grad_scores, const ScoreSpace& ws,
                   void* grad, hipStream_t stream) {
    // ranges of the vocabulary whose sums take at most 64 KB
    const int32_t parts = (x.V * R * 8 + 65535) / 65536, width = (x.V + parts - 1) / parts;
    const int32_t blocks = (int32_t)blocks_of(x.T, R);
    const size_t bytes = (size_t)R * width * 8 + (TABLE ? R * kTabulated * 8 : 0);
    // With a table one wavefront for six chunks: shorter hypotheses than the longest leave none idle, and the others' loads
    // go on while one waits.  With one, two and four wavefronts, in us: 64 x 500 frames of 3 chunks 27, 30, 43; 256 x 1500 of
    // 7 chunks 613, 650, 825; 64 x 1000 of 10 130, 135, 148; 32 x 500 of 12 47, 39, 45; 16 x 500 of 24 71, 48, 41; 8 x 500 of
    // 96 250, 156, 95 (where 8 chunks are eight short hypotheses, 46, 38, 42, the rule takes one).  Without a table as many
    // as there may be chunks, which share the block's long rows of sums (32 x 8: 212 us with one, 127 with two, 80 with four).
    const int64_t chunks = (int64_t)h.N * ((h.U + 1) / (kWave * kGradPairs - 2 * R) + 1);
    const int64_t waves = TABLE ? chunks / 6 : chunks, most = kGradThreads / kWave;
    const unsigned threads = kWave * (unsigned)(waves < 1 ? 1 : waves < most ? waves : most);
    hipLaunchKernelGGL((score_grad_kernel<T, R, TABLE>), dim3((unsigned)(x.B * (int64_t)blocks * parts)), dim3(threads), bytes,
                       stream, x, h, grad_scores, ws, blocks, parts, static_cast<T*>(grad));
    return hipGetLastError();
}

template <typename T>
hipError_t grad_of(const fltop_rows& x, const fltop_hypotheses& h, const double* grad_scores, const ScoreSpace& ws,
                   void* grad, hipStream_t stream) {
    const bool table = x.V <= kTabulated;
    if (block_frames(lattice_pairs(h.U)) == 8)
        return table ? grad_as<T, 8, true>(x, h, grad_scores, ws, grad, stream)
                     : grad_as<T, 8, false>(x, h, grad_scores, ws, grad, stream);
    return table ? grad_as<T, 4, true>(x, h, grad_scores, ws, grad, stream)
                 : grad_as<T, 4, false>(x, h, grad_scores, ws, grad, stream);
}

}  // namespace

hipError_t launch_score(const fltop_rows& x, const fltop_hypotheses& h, double* out_scores, const ScoreSpace* keep,
                        hipStream_t stream) {
    return x.V <= kTabulated ? score_as<true>(x, h, out_scores, keep, stream)
                             : score_as<false>(x, h, out_scores, keep, stream);
}

hipError_t launch_score_grad(const fltop_rows& x, const fltop_hypotheses& h, const double* grad_scores,
                             const ScoreSpace& ws, void* grad, hipStream_t stream) {
    if (x.type == FLTOP_TYPE_BF16) return grad_of<__hip_bfloat16>(x, h, grad_scores, ws, grad, stream);
    if (x.type == FLTOP_TYPE_F16) return grad_of<__half>(x, h, grad_scores, ws, grad, stream);
    return grad_of<float>(x, h, grad_scores, ws, grad, stream);
}

}  // namespace fltop
