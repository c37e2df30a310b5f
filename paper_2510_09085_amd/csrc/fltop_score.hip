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
// A workgroup takes one hypothesis, forwards and backwards at once: W wavefronts for each direction,
// lane by lane K pairs (b_i, l_i) each.  Both directions go to the middle of the utterance (the
// score is there), and with a gradient wanted a second kernel goes on from the middle to the two
// ends, each direction past the masses that the other has left: half as many serial frames as one
// direction after the other.
//
// Frames come in blocks of R.  Within a block only l_{i-1} passes from lane to lane (one DPP shift),
// and the wavefront above takes the same block one turn later with the last lane's masses from LDS,
// so that there is one barrier for a block and none for a frame.
//
// Every mass has its own exponent (class Mass), but aligning three of them for each sum costs more
// than the sum.  So a block is entered with one exponent E for each lane, no smaller than that of any
// mass that can reach the lane within the block (those of the kReach lanes below), and if
//   - no mass of these lanes is below 2^(E - kSpread),
//   - no emission needed in the block is outside [kLeast, kMost] (a little wider if tabulated), and
//   - the block has all its R frames
// then nothing leaves the range of fp64: masses stay above 2^(E - 440 - 577) and below 2^(E + 128)
// until its end.  A frame is then three multiply-adds and two products for each pair.  Blocks that do
// not hold this (masks of -inf, masses of e^-3000 that may be needed yet) are gone through with
// aligned exponents.  Rows of a trained model stay within: 8 tokens at e^-25 are 288 bits.
//
// The exponential of an emission takes three times the frame's own work.  For vocabularies of up to
// kTabulated tokens those of a block are taken once for all lanes, into a table in LDS, a turn ahead
// and by all wavefronts of the direction together; for larger ones each lane takes its tokens'.

constexpr int kWave = 64;
constexpr int kSpread = 440;
constexpr int kTabulated = 64;
constexpr int32_t kAligned = INT32_MIN;   // in place of a lane's exponent: masses are kept as Mass32

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

// 2^e for e in [-1022, 1023].
__device__ inline double power_of_two(int32_t e) { return from_words((e + 1023) << 20, 0); }

// exp(lp) for lp in [kLeast, kMost], as mass_of, with k taken from the last bits of a number in which they are worth
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

// exp(lp) of any emission: 0 or infinity where it leaves the range in which blocks are gone through with one exponent.
__device__ inline double exp_any(float lp) {
    const double near = exp_near(fminf(fmaxf(lp, -600.0f), 600.0f));
    return lp < -600.0f ? 0.0 : lp <= 600.0f ? near : INFINITY;
}

// An element as it lies in memory; converted where it is used, so that loads stay in flight.
template <int TYPE>
__device__ inline uint32_t raw_at(const char* row, int32_t v) {
    if constexpr (TYPE == FLTOP_TYPE_F32)
        return reinterpret_cast<const uint32_t*>(row)[v];
    else
        return reinterpret_cast<const uint16_t*>(row)[v];
}
template <int TYPE>
__device__ inline float raw_value(uint32_t x) {
    if constexpr (TYPE == FLTOP_TYPE_F32) return __uint_as_float(x);
    if constexpr (TYPE == FLTOP_TYPE_BF16) return __uint_as_float(x << 16);
    return __half2float(__ushort_as_half((unsigned short)x));
}

__device__ inline float value_at(const char* row, int32_t v, int32_t type) {
    if (type == FLTOP_TYPE_F32) return raw_value<FLTOP_TYPE_F32>(raw_at<FLTOP_TYPE_F32>(row, v));
    const uint32_t x = raw_at<FLTOP_TYPE_F16>(row, v);
    return type == FLTOP_TYPE_BF16 ? raw_value<FLTOP_TYPE_BF16>(x) : raw_value<FLTOP_TYPE_F16>(x);
}

template <bool FIRST, typename A, typename B> struct Choose { using type = A; };
template <typename A, typename B> struct Choose<false, A, B> { using type = B; };

// An utterance's emissions.
struct Source {
    const char* rows;
    int64_t frame_bytes;
    int32_t type, V;
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

// A workgroup's LDS: edges of each direction and wavefront (one below the first) for this turn and the one before;
// a place for what is written so that the lanes that have nothing to say need no branch; tables of exponentials of
// W + 1 blocks.  In the middle, masses of U + 1 states in place of the last two.
template <int R>
struct Lds {
    Edge<R>* edges;      // [2][W + 1][2]
    double* nowhere;     // [2 W][kWave + R]
    double* tables;      // [2][W + 1][R][stride]
    double* half_m;      // [U + 1]
    int32_t* half_e;
    int stride, W;

    __host__ __device__ static int stride_for(int32_t V) { return V > kTabulated ? 0 : V > 32 ? 64 : 32; }
    __device__ Lds(char* at, int waves, int32_t V, int32_t U) : stride(stride_for(V)), W(waves) {
        edges = reinterpret_cast<Edge<R>*>(at);
        nowhere = half_m = reinterpret_cast<double*>(edges + 4 * (W + 1));
        tables = nowhere + 2 * W * (kWave + R);
        half_e = reinterpret_cast<int32_t*>(half_m + U + 1);
    }
    static size_t bytes(int W, int32_t V, int32_t U, bool middle) {
        const size_t way = (size_t)(2 * W * (kWave + R) + 2 * (W + 1) * R * stride_for(V)) * sizeof(double);
        const size_t half = middle ? (size_t)(U + 1) * 12 : 0;
        return 4 * (W + 1) * sizeof(Edge<R>) + (way > half ? way : half);
    }
    __device__ Edge<R>& edge(bool reversed, int wave_below, int turn) const {
        return edges[((reversed ? W + 1 : 0) + wave_below) * 2 + (turn & 1)];
    }
    __device__ double* table(bool reversed, int32_t block) const {
        return tables + ((reversed ? W + 1 : 0) + block % (W + 1)) * R * stride;
    }
};

// What a launch does with the masses.
constexpr int kScore = 0, kKeep = 1, kMeet = 2;

// What a direction does in a launch.
struct Way {
    int32_t lo, hi;      // its frames
    bool reversed;
    double* rows;        // masses: written (kKeep), or the other direction's (kMeet); [T][row]
    int32_t* exps;       // their exponents, [T / R][row]
    float* shares;       // [T][share_row]
    int32_t total_e;
    int32_t row, share_row;
    int32_t U;
};

// The part of the lattice that one lane holds.
template <int K, int R, bool TABLE>
struct Lane {
    static constexpr int kReach = (R + K - 1) / K;   // lanes that a block's masses can come from
    static constexpr float kLeast = -400.0f / R, kMost = 80.0f / R;
    static constexpr uint32_t kLeastWord = (1023u - 576 / R) << 20, kMostWord = (1023u + 112 / R) << 20;

    double xb[K], xl[K];     // masses x * 2^e
    int32_t eb[K], el[K];
    int32_t tok[K];          // 0 behind the last token
    double skip[K];          // 1 where y_{i+1} != y_i, else 0
    double live[K];          // 1 for pairs with a token, else 0
    int32_t i0;              // first pair
    // Emissions of the next block as they lie in memory, and those of the present one; the blank's of frame f in lane
    // f (mod R).  With a table: what this lane adds to the next one, and its tokens' exponentials of the present block.
    uint32_t raw[R][TABLE ? 1 : K], raw_blank;
    using Given = typename Choose<TABLE, double, float>::type;
    Given given[R][K], given_blank[TABLE ? R : 1];

    __device__ bool start(const Hyp& y, int32_t V, bool reversed, int32_t first_pair) {
        bool fine = true;
        i0 = first_pair;
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
            eb[k] = i == 0 ? 0 : kNoMass;
            xl[k] = 0.0;
            el[k] = kNoMass;
        }
        return fine;
    }

    // Asks for the emissions of frames t0 .. t0 + nf - 1, in the order in which they are taken.
    template <int TYPE>
    __device__ void ask_as(const Source& from, int32_t t0, int32_t nf, bool reversed) {
#pragma unroll
        for (int f = 0; f < R; ++f) {
            const int32_t g = min(f, nf - 1);
            const char* row = from.rows + (int64_t)(t0 + (reversed ? nf - 1 - g : g)) * from.frame_bytes;
#pragma unroll
            for (int k = 0; k < K; ++k) raw[f][TABLE ? 0 : k] = raw_at<TYPE>(row, tok[k]);
        }
        const int32_t g = min((int32_t)(threadIdx.x & (R - 1)), nf - 1);
        raw_blank = raw_at<TYPE>(from.rows + (int64_t)(t0 + (reversed ? nf - 1 - g : g)) * from.frame_bytes, 0);
    }
    __device__ void ask(const Source& from, int32_t t0, int32_t nf, bool reversed) {
        if (from.type == FLTOP_TYPE_F32)
            ask_as<FLTOP_TYPE_F32>(from, t0, nf, reversed);
        else
            ask_as<FLTOP_TYPE_F16>(from, t0, nf, reversed);   // 16 bits of either kind
    }
    template <int TYPE>
    __device__ void got_as() {
#pragma unroll
        for (int f = 0; f < R; ++f)
#pragma unroll
            for (int k = 0; k < K; ++k) given[f][k] = raw_value<TYPE>(raw[f][TABLE ? 0 : k]);
        given_blank[0] = raw_value<TYPE>(raw_blank);
    }
    __device__ void got(int32_t type) {
        if (type == FLTOP_TYPE_F32)
            got_as<FLTOP_TYPE_F32>();
        else if (type == FLTOP_TYPE_BF16)
            got_as<FLTOP_TYPE_BF16>();
        else
            got_as<FLTOP_TYPE_F16>();
    }

    // With a table: its rows are taken n = kWave / stride at a time, by one wavefront after the other.
    template <int TYPE>
    __device__ void ask_table_as(const Source& from, int stride, int wave, int W, int32_t t0, int32_t nf, bool reversed) {
        const int lane = threadIdx.x & (kWave - 1);
        const int n = kWave / stride;
        const int32_t v = min((int32_t)(lane & (stride - 1)), from.V - 1);
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int f0 = (j * W + wave) * n;
            if (f0 >= R) break;
            const int32_t g = min(f0 + (lane >= stride ? 1 : 0), nf - 1);
            raw[j][0] = raw_at<TYPE>(from.rows + (int64_t)(t0 + (reversed ? nf - 1 - g : g)) * from.frame_bytes, v);
        }
    }
    __device__ void ask_table(const Source& from, int stride, int wave, int W, int32_t t0, int32_t nf, bool reversed) {
        if (from.type == FLTOP_TYPE_F32)
            ask_table_as<FLTOP_TYPE_F32>(from, stride, wave, W, t0, nf, reversed);
        else
            ask_table_as<FLTOP_TYPE_F16>(from, stride, wave, W, t0, nf, reversed);
    }
    __device__ void put_table(const Source& from, double* table, int stride, int wave, int W) {
        const int lane = threadIdx.x & (kWave - 1);
        const int n = kWave / stride;
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int f0 = (j * W + wave) * n;
            if (f0 >= R) break;
            const uint32_t x = raw[j][0];
            table[f0 * stride + lane] = exp_any(from.type == FLTOP_TYPE_F32    ? raw_value<FLTOP_TYPE_F32>(x)
                                                : from.type == FLTOP_TYPE_BF16 ? raw_value<FLTOP_TYPE_BF16>(x)
                                                                               : raw_value<FLTOP_TYPE_F16>(x));
        }
    }
    __device__ void look_up(const double* table, int stride) {
#pragma unroll
        for (int f = 0; f < R; ++f) {
            given_blank[TABLE ? f : 0] = table[f * stride];
#pragma unroll
            for (int k = 0; k < K; ++k) given[f][k] = table[f * stride + tok[k]];
        }
    }

    // The lane's exponent for a block, and the lane below's; returns whether the block can be gone through with them as
    // far as this lane goes.
    __device__ bool enter(const Edge<R>& in, int32_t* E, int32_t* least, int32_t* below) {
        int32_t top = kNoMass, low = -kNoMass;
        bool fine = true;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int32_t a = xb[k] == 0.0 ? kNoMass : eb[k] + __builtin_amdgcn_frexp_exp(xb[k]);
            const int32_t c = xl[k] == 0.0 ? kNoMass : el[k] + __builtin_amdgcn_frexp_exp(xl[k]);
            top = max(top, max(a, c));
            low = min(low, min(a == kNoMass ? -kNoMass : a, c == kNoMass ? -kNoMass : c));
        }
        if constexpr (TABLE) {
            uint32_t most = 0, least_p = kMostWord;
#pragma unroll
            for (int f = 0; f < R; ++f)
#pragma unroll
                for (int k = -1; k < K; ++k) {
                    const double one = k < 0 ? given_blank[f] : given[f][k < 0 ? 0 : k];
                    const uint32_t w = (uint32_t)(__double_as_longlong(one) >> 32);
                    most = max(most, w);
                    least_p = min(least_p, w);
                }
            fine = least_p >= kLeastWord && most < kMostWord;
        } else {
            float most = given_blank[0], least_lp = given_blank[0];
#pragma unroll
            for (int f = 0; f < R; ++f)
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    most = fmaxf(most, given[f][k]);
                    least_lp = fminf(least_lp, given[f][k]);
                }
            fine = least_lp >= kLeast && most <= kMost;
        }
        int32_t m = top, n = low;
#pragma unroll
        for (int d = 0; d < kReach; ++d) {
            m = max(from_below(m, in.E), top);
            n = min(from_below(n, in.least), low);
        }
        *E = m;
        *least = n;
        *below = from_below(m, in.E);
        return fine && (m == kNoMass || m - n <= kSpread) && !in.aligned;
    }
};

// Sums of v[0..R) over the wavefront, in a fixed order; lane f (mod R) returns that of v[f].  Each of the
// first steps halves the number of values that a lane carries.
template <int R>
__device__ inline float sums_by_lane(float (&v)[R]) {
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
            const float keep = upper ? v[2 * j + 1] : v[2 * j];
            const float give = upper ? v[2 * j] : v[2 * j + 1];
            v[j] = keep + __shfl_xor(give, o, kWave);
        }
    }
#pragma unroll
    for (int o = R; o < kWave; o <<= 1) v[0] += __shfl_xor(v[0], o, kWave);
    return v[0];
}

// Where a lane's states are in a row (bytes of the masses; exponents and shares have half of it): a direction's own
// view of the hypothesis.  Lanes behind the last pair have a place of no meaning at the row's end, so that loads and
// stores need no branch: a branch around a store would have every later wait for a load wait for the store too.
template <int K>
struct Places {
    uint32_t b[K], l[K], share[K];
    __device__ Places(const Way& way, int32_t i0, int32_t L) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int32_t i = i0 + k;
            const int32_t bi = way.reversed ? L - i : i, li = way.reversed ? L - 1 - i : i;
            b[k] = 8u * (uint32_t)(i <= L ? bi : way.row - 1);
            l[k] = 8u * (uint32_t)(i < L ? way.U + 1 + li : way.row - 1);
            share[k] = 4u * (uint32_t)(i < L ? li : way.U + kShareBlanks);
        }
    }
};
template <typename T>
__device__ inline T& at_byte(T* base, uint32_t offset) {
    return *reinterpret_cast<T*>(reinterpret_cast<char*>(base) + offset);
}

// The other direction's masses of a block.
template <int K, int R>
struct Met {
    double b[R][K], l[R][K];
    int32_t eb[K], el[K];
    __device__ void ask(const Way& way, const Places<K>& at, int32_t t0, int32_t nf) {
        int32_t* exps = way.exps + (int64_t)(t0 / R) * way.row;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            eb[k] = at_byte(exps, at.b[k] / 2);
            el[k] = at_byte(exps, at.l[k] / 2);
        }
#pragma unroll
        for (int f = 0; f < R; ++f) {
            const int32_t g = min(f, nf - 1);
            double* row = way.rows + (int64_t)(t0 + (way.reversed ? nf - 1 - g : g)) * way.row;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                b[f][k] = at_byte(row, at.b[k]);
                l[f][k] = at_byte(row, at.l[k]);
            }
        }
    }
};

// A kept mass with its exponent e, whichever way it was kept.
__device__ inline Mass kept_mass(double x, int32_t e) {
    if (e != kAligned) return normalized(x, e);
    const long long bits = __double_as_longlong(x);
    return {__uint_as_float((uint32_t)bits), (int32_t)(bits >> 32)};
}
__device__ inline double keep_mass(Mass x) { return from_words(x.e, (int32_t)__float_as_uint((float)x.m)); }

// The product of two masses becomes a share by 2^c, with c their exponents less that of P.  Masses are below 2^128, so
// that a share of weight has c > -300; up to kMostShift one mass times 2^c stays in range whatever the other is.
constexpr int32_t kMostShift = 880;
__device__ inline int32_t share_shift(int32_t E, int32_t kept, int32_t total) {
    if (kept == kAligned) return kMostShift + 1;
    if (kept <= kNoMass || E <= kNoMass) return -2000;
    const long long c = (long long)E + kept - total;
    return (int32_t)(c < -2000 ? -2000 : c > kMostShift ? kMostShift + 1 : c);
}
__device__ inline double share_factor(int32_t c) { return c < -1000 ? 0.0 : power_of_two(c); }

// One block of frames for one wavefront.  `in`: from the wavefront below, `out`: for the one above.
template <int K, int R, int TASK, bool TABLE>
__device__ inline void take_block(Lane<K, R, TABLE>& z, const Way& way, const Met<K, R>& met, const Places<K>& at, int32_t L,
                                  int32_t q, int wave, const Edge<R>& in, Edge<R>& out, double* nowhere,
                                  const Source& from) {
    const int lane = threadIdx.x & (kWave - 1);
    const int32_t t0 = q * R;
    const int32_t nf = min(R, way.hi - t0);
    float blanks[R];
    int32_t E, least, below;
    bool fine = z.enter(in, &E, &least, &below) && nf == R;
    double fb[K], fl[K];
    if constexpr (TASK == kMeet) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int32_t cb = share_shift(E, met.eb[k], way.total_e), cl = share_shift(E, met.el[k], way.total_e);
            fine &= z.i0 + k > L || cb <= kMostShift;
            fine &= z.i0 + k >= L || cl <= kMostShift;
            fb[k] = share_factor(min(cb, kMostShift));
            fl[k] = share_factor(min(cl, kMostShift));
        }
    }
    const bool near = __all(fine);
    if (lane == kWave - 1) {
        out.E = E;
        out.least = least;
        out.aligned = !near;
    }
    if constexpr (TASK == kKeep) {
        int32_t* to = way.exps + (int64_t)q * way.row;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            at_byte(to, at.b[k] / 2) = near ? E : kAligned;
            at_byte(to, at.l[k] / 2) = near ? E : kAligned;
        }
    }
    if (near) {
        // the lane below's scale in this one's
        const double fx = ldexp(1.0, min(below - E, 1000));
        const double fskip = fx * z.skip[0];
        double* const edge = lane == kWave - 1 ? out.x : nowhere + lane;
        double first[R];
#pragma unroll
        for (int f = 0; f < R; ++f) first[f] = in.x[f];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            z.xb[k] = ldexp(z.xb[k], z.eb[k] - E);
            z.xl[k] = ldexp(z.xl[k], z.el[k] - E);
            z.eb[k] = z.el[k] = E;
        }
        double blank_by_lane = 0.0;
        if constexpr (!TABLE) blank_by_lane = exp_near(z.given_blank[0]);
#pragma unroll
        for (int f = 0; f < R; ++f) {
            const int32_t t = t0 + (way.reversed ? R - 1 - f : f);
            double pb;
            if constexpr (TABLE)
                pb = z.given_blank[f];
            else
                pb = from_lane(blank_by_lane, f);
            edge[f] = z.xl[K - 1];
            const double moved = from_below(z.xl[K - 1], first[f]);
            double blank = 0.0;
#pragma unroll
            for (int k = K - 1; k >= 0; --k) {
                const double prev = k > 0 ? z.xl[k > 0 ? k - 1 : 0] : moved;
                const double stay = fma(z.xb[k], z.live[k], z.xl[k]);
                const double l = fma(prev, k > 0 ? z.skip[k] : fskip, stay);
                const double b = k > 0 ? z.xb[k] + prev : fma(prev, fx, z.xb[k]);
                if constexpr (TASK == kMeet) {
                    // (behind the last pair there is no mass: b = 0)
                    blank += met.b[f][k] * fb[k] * b;
                    at_byte(way.shares + (int64_t)t * way.share_row, at.share[k]) = (float)(met.l[f][k] * fl[k] * l);
                }
                z.xb[k] = b * pb;
                if constexpr (TABLE)
                    z.xl[k] = l * z.given[f][k];
                else
                    z.xl[k] = l * exp_near(z.given[f][k]);
                if constexpr (TASK == kKeep) {
                    double* to = way.rows + (int64_t)t * way.row;
                    at_byte(to, at.b[k]) = z.xb[k];
                    at_byte(to, at.l[k]) = z.xl[k];
                }
            }
            blanks[f] = (float)blank;
        }
    } else {
        Mass b[K], l[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            b[k] = normalized(z.xb[k], z.eb[k]);
            l[k] = normalized(z.xl[k], z.el[k]);
        }
#pragma unroll
        for (int f = 0; f < R; ++f) blanks[f] = 0.0f;
#pragma unroll 1
        for (int f = 0; f < nf; ++f) {
            const int32_t t = t0 + (way.reversed ? nf - 1 - f : f);
            const char* emissions = from.rows + (int64_t)t * from.frame_bytes;
            const Mass blank = mass_of(value_at(emissions, 0, from.type));
            const Mass first = normalized(in.x[f], in.aligned ? in.e[f] : in.E);
            if (lane == kWave - 1) {
                out.x[f] = l[K - 1].m;
                out.e[f] = l[K - 1].e;
            }
            const Mass moved = {from_below(l[K - 1].m, first.m), from_below(l[K - 1].e, first.e)};
            float share = 0.0f;
#pragma unroll
            for (int k = K - 1; k >= 0; --k) {
                const int32_t i = z.i0 + k;
                const Mass prev = k > 0 ? l[k > 0 ? k - 1 : 0] : moved;
                Mass stay = plus(l[k], b[k]);
                if (z.skip[k] != 0.0) stay = plus(stay, prev);
                stay = normalized(stay.m, stay.e);
                Mass on = plus(b[k], prev);
                on = normalized(on.m, on.e);
                if constexpr (TASK == kMeet) {
                    double* row = way.rows + (int64_t)t * way.row;
                    if (i <= L) {
                        const Mass m = kept_mass(at_byte(row, at.b[k]), met.eb[k]);
                        share += (float)ldexp(m.m * on.m, m.e + on.e - way.total_e);
                    }
                    if (i < L) {
                        const Mass m = kept_mass(at_byte(row, at.l[k]), met.el[k]);
                        at_byte(way.shares + (int64_t)t * way.share_row, at.share[k]) =
                            (float)ldexp(m.m * stay.m, m.e + stay.e - way.total_e);
                    }
                }
                const Mass p = mass_of(value_at(emissions, z.tok[k], from.type));
                b[k] = normalized(on.m * blank.m, on.e + blank.e);
                l[k] = i < L ? normalized(stay.m * p.m, stay.e + p.e) : no_mass();
                if constexpr (TASK == kKeep) {
                    double* to = way.rows + (int64_t)t * way.row;
                    at_byte(to, at.b[k]) = keep_mass(b[k]);
                    at_byte(to, at.l[k]) = keep_mass(l[k]);
                }
            }
#pragma unroll
            for (int g = 0; g < R; ++g) blanks[g] = g == f ? share : blanks[g];
        }
#pragma unroll
        for (int k = 0; k < K; ++k) {
            z.xb[k] = b[k].m;
            z.eb[k] = b[k].e;
            z.xl[k] = l[k].m;
            z.el[k] = l[k].e;
        }
    }
    if constexpr (TASK == kMeet) {
        const float sum = sums_by_lane<R>(blanks);
        const int32_t f = min(lane, nf - 1);
        const int32_t t = t0 + (way.reversed ? nf - 1 - f : f);
        way.shares[(int64_t)t * way.share_row + way.U + (lane < nf ? wave : kShareBlanks)] = sum;
    }
}

// All blocks of this workgroup's two directions, a turn at a time: wavefront w of a direction is w blocks behind its
// first.
template <int K, int R, int TASK, bool TABLE>
__device__ inline void take_all(Lane<K, R, TABLE>& z, const Way& way, const Way& other, int32_t L, const Source& from,
                                int wave, int32_t used, const Lds<R>& lds) {
    double* const nowhere = lds.nowhere + ((way.reversed ? lds.W : 0) + wave) * (kWave + R);
    if (threadIdx.x < 4 * R) {
        Edge<R>& none = lds.edge(threadIdx.x >= 2 * R, 0, threadIdx.x / R);
        none.x[threadIdx.x & (R - 1)] = 0.0;
        none.e[threadIdx.x & (R - 1)] = kNoMass;
        none.E = kNoMass;
        none.least = -kNoMass;
        none.aligned = 0;
    }
    const int32_t first = way.lo / R;
    const int32_t blocks = way.hi > way.lo ? (way.hi + R - 1) / R - first : 0;
    const int32_t others = other.hi > other.lo ? (other.hi + R - 1) / R - other.lo / R : 0;
    const int32_t turns = max(blocks, others) + used - 1;
    constexpr bool kEarly = TASK == kMeet && K <= 2;   // registers for two blocks of the other direction
    Met<K, R> met, next;
    auto block = [&](int32_t n) { return way.reversed ? first + blocks - 1 - n : first + n; };
    const Places<K> at(way, z.i0, L);
    auto ask = [&](int32_t n) {
        const int32_t q = block(min(n, blocks - 1)), nf = min(R, way.hi - q * R);
        if constexpr (!TABLE) z.ask(from, q * R, nf, way.reversed);
        if constexpr (kEarly) next.ask(way, at, q * R, nf);
    };
    auto ask_table = [&](int32_t n) {
        const int32_t q = block(min(n, blocks - 1));
        z.ask_table(from, lds.stride, wave, lds.W, q * R, min(R, way.hi - q * R), way.reversed);
    };
    auto put_table = [&](int32_t n) { z.put_table(from, lds.table(way.reversed, n), lds.stride, wave, lds.W); };
    // The next block's exponentials; the block behind it is asked for.
    auto tabulate = [&](int32_t turn) {
        if constexpr (TABLE) {
            if (turn + 1 < blocks) {
                put_table(turn + 1);
                ask_table(turn + 2);
            }
        }
    };
    const bool works = wave < used && blocks > 0;
    if (works) ask(0);
    if constexpr (TABLE) {
        if (blocks > 0) {
            ask_table(0);
            put_table(0);
            ask_table(1);
        }
    }
    __syncthreads();
    // (three loops: with the idle turns in the loop of the blocks, a wait for a load would count on no store behind it)
    const int32_t before = works ? wave : turns, after = works ? wave + blocks : turns;
    for (int32_t turn = 0; turn < before; ++turn) {
        tabulate(turn);
        __syncthreads();
    }
    for (int32_t turn = before; turn < after; ++turn) {
        const int32_t n = turn - wave, q = block(n);
        tabulate(turn);
        if constexpr (!TABLE) z.got(from.type);
        if constexpr (kEarly) met = next;
        if constexpr (TASK == kMeet && !kEarly) met.ask(way, at, q * R, min(R, way.hi - q * R));
        ask(n + 1);
        if constexpr (TABLE) z.look_up(lds.table(way.reversed, n), lds.stride);
        take_block<K, R, TASK, TABLE>(z, way, met, at, L, q, wave, lds.edge(way.reversed, wave, turn - 1),
                                      lds.edge(way.reversed, wave + 1, turn), nowhere, from);
        __syncthreads();
    }
    for (int32_t turn = after; turn < turns; ++turn) {
        tabulate(turn);
        __syncthreads();
    }
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

// Scores, and the lattice up to the middle from both ends.  blockDim = 2 W wavefronts.
template <int K, int R, int THREADS, bool TABLE, int TASK>
__global__ __launch_bounds__(THREADS) void score_kernel(fltop_rows x, fltop_hypotheses h, double* out_scores,
                                                        ScoreSpace ws) {
    constexpr bool keep = TASK == kKeep;
    extern __shared__ char dynamic[];
    __shared__ Mass sums[2][kMostWaves];
    __shared__ Mass last[kMostWaves];
    const int64_t at = blockIdx.x;
    const int32_t b = (int32_t)(at / h.N), n = (int32_t)(at % h.N);
    const Hyp y = hypothesis(x, h, b, n);
    const int W = (int)blockDim.x / kWave / 2;
    const Lds<R> lds(dynamic, W, x.V, h.U);
    const int lane = threadIdx.x & (kWave - 1);
    const int wave_of_all = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    const bool reversed = wave_of_all >= W;
    const int wave = wave_of_all - (reversed ? W : 0);
    Lane<K, R, TABLE> z;
    const bool fine = y.L >= 0 && z.start(y, x.V, reversed, (wave * kWave + lane) * K);
    if (__syncthreads_or(!fine)) {
        if (threadIdx.x == 0) {
            out_scores[at] = y.L == -2 ? NAN : -INFINITY;
            if (keep) ws.total_m[at] = 0.0, ws.total_e[at] = kNoMass;
        }
        return;
    }
    const int32_t used = y.L / (kWave * K) + 1;
    const int32_t middle = middle_of<R>(y.frames);
    double* const rows = keep ? ws.rows + at * x.T * ws.row : nullptr;
    int32_t* const exps = keep ? ws.exps + at * blocks_of(x.T, R) * ws.row : nullptr;
    const Way ways[2] = {{0, middle, false, rows, exps, nullptr, 0, (int32_t)ws.row, share_row(h.U), h.U},
                         {middle, y.frames, true, rows, exps, nullptr, 0, (int32_t)ws.row, share_row(h.U), h.U}};
    const Way way = reversed ? ways[1] : ways[0], other = reversed ? ways[0] : ways[1];
    take_all<K, R, TASK, TABLE>(z, way, other, y.L, source_of(x, b), wave, used, lds);

    // P = sum over states of the forward mass after frame middle - 1 and the backward bracket at that frame
    if (reversed && lane == kWave - 1) last[wave] = normalized(z.xl[K - 1], z.el[K - 1]);
    __syncthreads();
    Mass on[K], stay[K];
    if (reversed) {
        Mass l[K], bl[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            l[k] = normalized(z.xl[k], z.el[k]);
            bl[k] = normalized(z.xb[k], z.eb[k]);
        }
        const Mass first = wave > 0 ? last[wave > 0 ? wave - 1 : 0] : no_mass();
        const Mass moved = {from_below(l[K - 1].m, first.m), from_below(l[K - 1].e, first.e)};
#pragma unroll
        for (int k = K - 1; k >= 0; --k) {
            const Mass prev = k > 0 ? l[k > 0 ? k - 1 : 0] : moved;
            stay[k] = plus(l[k], bl[k]);
            if (z.skip[k] != 0.0) stay[k] = plus(stay[k], prev);
            on[k] = plus(bl[k], prev);
        }
    }
#pragma unroll
    for (int part = 0; part < 2; ++part) {   // blanks, then tokens
        if (!reversed && wave < used) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int32_t i = z.i0 + k;
                const Mass m = part ? normalized(z.xl[k], z.el[k]) : normalized(z.xb[k], z.eb[k]);
                if (i < y.L + 1 - part) {
                    lds.half_m[i] = m.m;
                    lds.half_e[i] = m.e;
                }
            }
        }
        __syncthreads();
        if (reversed) {
            Mass sum = no_mass();
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int32_t i = z.i0 + k;
                if (i >= y.L + 1 - part) continue;
                const Mass m = part ? stay[k] : on[k];
                const int32_t s = y.L - part - i;
                sum = plus(sum, normalized(lds.half_m[s] * m.m, max(lds.half_e[s] + m.e, kNoMass)));
                sum = normalized(sum.m, sum.e);
            }
#pragma unroll
            for (int o = kWave / 2; o > 0; o >>= 1) {
                sum = plus(sum, {__shfl_xor(sum.m, o, kWave), __shfl_xor(sum.e, o, kWave)});
                sum = normalized(sum.m, sum.e);
            }
            if (lane == 0) sums[part][wave] = sum;
        }
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        Mass p = no_mass();
        for (int w = 0; w < W; ++w) {
            p = plus(p, plus(sums[0][w], sums[1][w]));
            p = normalized(p.m, p.e);
        }
        out_scores[at] = ln_of(p);
        if (keep) ws.total_m[at] = p.m, ws.total_e[at] = p.e;
    }
}

// From the middle on to both ends: occupancies, times the mantissa of P.
template <int K, int R, int THREADS, bool TABLE>
__global__ __launch_bounds__(THREADS) void shares_kernel(fltop_rows x, fltop_hypotheses h, ScoreSpace ws) {
    extern __shared__ char dynamic[];
    const int64_t at = blockIdx.x;
    const int32_t b = (int32_t)(at / h.N), n = (int32_t)(at % h.N);
    const int32_t total_e = ws.total_e[at];
    const Hyp y = hypothesis(x, h, b, n);
    if (total_e <= kNoMass || y.L < 0) return;
    const int W = (int)blockDim.x / kWave / 2;
    const Lds<R> lds(dynamic, W, x.V, h.U);
    const int lane = threadIdx.x & (kWave - 1);
    const int wave_of_all = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    const bool reversed = wave_of_all >= W;
    const int wave = wave_of_all - (reversed ? W : 0);
    Lane<K, R, TABLE> z;
    z.start(y, x.V, reversed, (wave * kWave + lane) * K);
    const int32_t used = y.L / (kWave * K) + 1;
    const int32_t middle = middle_of<R>(y.frames);
    double* const rows = ws.rows + at * x.T * ws.row;
    int32_t* const exps = ws.exps + at * blocks_of(x.T, R) * ws.row;
    float* const shares = ws.shares + at * x.T * share_row(h.U);
    const Way ways[2] = {{middle, y.frames, false, rows, exps, shares, total_e, (int32_t)ws.row, share_row(h.U), h.U},
                         {0, middle, true, rows, exps, shares, total_e, (int32_t)ws.row, share_row(h.U), h.U}};
    const int32_t from = reversed ? middle : middle - 1;   // the frame that this direction went to
    if (from >= 0 && from < y.frames) {
        double* row = rows + from * ws.row;
        int32_t* e = exps + from / R * ws.row;
        const Places<K> place(ways[reversed], z.i0, y.L);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int32_t i = z.i0 + k;
            const Mass mb = i <= y.L ? kept_mass(at_byte(row, place.b[k]), at_byte(e, place.b[k] / 2)) : no_mass();
            const Mass ml = i < y.L ? kept_mass(at_byte(row, place.l[k]), at_byte(e, place.l[k] / 2)) : no_mass();
            z.xb[k] = mb.m;
            z.eb[k] = mb.e;
            z.xl[k] = ml.m;
            z.el[k] = ml.e;
        }
    }
    const Way way = reversed ? ways[1] : ways[0], other = reversed ? ways[0] : ways[1];
    take_all<K, R, kMeet, TABLE>(z, way, other, y.L, source_of(x, b), wave, used, lds);
}

// Occupancies into rows of V sums, which are whole numbers so that the order in which lanes add does not matter.
// A wavefront takes `per_wave` frames of an utterance at a time: each token's place is read once for all of them.
constexpr int kGradWaves = 4;   // two where a frame's row takes 32 KB
constexpr int kGradFrames = 8;

// Orders a wavefront's accesses to its own part of LDS, lane by lane.
__device__ inline void wave_fence() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

template <typename T>
__global__ __launch_bounds__(kGradWaves* kWave) void score_grad_kernel(fltop_rows x, fltop_hypotheses h,
                                                                       const double* grad_scores, ScoreSpace ws,
                                                                       int32_t per_wave, int32_t chunks, int32_t per_used,
                                                                       T* grad) {
    extern __shared__ char dynamic[];
    const int lane = threadIdx.x & (kWave - 1);
    const int wave = threadIdx.x / kWave;
    unsigned long long* sums = reinterpret_cast<unsigned long long*>(dynamic) + (int64_t)wave * per_wave * x.V;
    const int64_t chunk = (int64_t)blockIdx.x * (blockDim.x / kWave) + wave;
    const int32_t b = (int32_t)(chunk / chunks), t0 = (int32_t)(chunk % chunks) * per_wave;
    if (b >= x.B) return;
    const int32_t frames = min(x.lengths[b], x.T);
    const int32_t nf = min(per_wave, x.T - t0), live = min(nf, frames - t0);
    T* out = grad + ((int64_t)b * x.T + t0) * x.V;
    double most = 0.0;
    bool odd = false;
    for (int32_t n = lane; n < h.N; n += kWave) {
        const int64_t at = (int64_t)b * h.N + n;
        if (ws.total_e[at] <= kNoMass) continue;
        const double w = fabs(grad_scores[at]);
        odd |= !(w <= 1.7976931348623157e308);
        most = fmax(most, w);
    }
    odd = __any(odd);
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) most = fmax(most, __shfl_xor(most, o, kWave));
    if (odd || most == 0.0 || live <= 0) {
        for (int32_t v = lane; v < nf * x.V; v += kWave)
            out[v] = from_float<T>(odd && v < (int64_t)live * x.V ? NAN : 0.0f);
        return;
    }
    for (int32_t v = lane; v < nf * x.V; v += kWave) sums[v] = 0;
    wave_fence();
    constexpr double kOne = 1125899906842624.0;       // 2^50
    constexpr double kShift = 6755399441055744.0;     // 1.5 * 2^52: its last bit is worth one
    const int64_t row = share_row(h.U);
    for (int32_t n = 0; n < h.N; ++n) {
        const int64_t at = (int64_t)b * h.N + n;
        if (ws.total_e[at] <= kNoMass) continue;
        // shares come times the mantissa of P, which is at least 1/2
        const double w = grad_scores[at] / most * (kOne / ws.total_m[at]);
        const Hyp y = hypothesis(x, h, b, n);
        const float* from = ws.shares + (at * x.T + t0) * row;
        for (int32_t i = lane; i < y.L; i += kWave) {
            const int32_t v = y.tokens[i];
            if ((uint32_t)v >= (uint32_t)x.V) continue;   // not the hypotheses that were scored
            float share[kGradFrames];
#pragma unroll
            for (int f = 0; f < kGradFrames; ++f) share[f] = f < live ? from[f * row + i] : 0.0f;
#pragma unroll
            for (int f = 0; f < kGradFrames; ++f) {
                if (f >= live) break;
                const long long a = __double_as_longlong(share[f] * w + kShift) - __double_as_longlong(kShift);
                atomicAdd(&sums[f * x.V + v], (unsigned long long)a);
            }
        }
        // the blanks: one partial sum from each wavefront that this hypothesis had
        const int32_t used = y.L / per_used + 1;
        for (int32_t i = lane; i < live * kShareBlanks; i += kWave) {
            const int32_t f = i / kShareBlanks, s = i % kShareBlanks;
            if (s >= used) continue;
            const long long a =
                __double_as_longlong(from[f * row + h.U + s] * w + kShift) - __double_as_longlong(kShift);
            atomicAdd(&sums[f * x.V], (unsigned long long)a);
        }
    }
    wave_fence();
    for (int32_t v = lane; v < nf * x.V; v += kWave)
        out[v] = from_float<T>((float)((double)(long long)sums[v] * (most / kOne)));
}

// Pairs of a lane, frames of a block, most threads.
template <int K, int R, int THREADS, bool TABLE>
struct Build {
    static hipError_t score(const fltop_rows& x, const fltop_hypotheses& h, double* out_scores, const ScoreSpace* keep,
                            hipStream_t stream) {
        const int W = waves_for(h.U, K);
        const dim3 grid((unsigned)(x.B * h.N)), block(2 * kWave * W);
        const size_t bytes = Lds<R>::bytes(W, x.V, h.U, true);
        if (keep)
            hipLaunchKernelGGL((score_kernel<K, R, THREADS, TABLE, kKeep>), grid, block, bytes, stream, x, h, out_scores,
                               *keep);
        else
            hipLaunchKernelGGL((score_kernel<K, R, THREADS, TABLE, kScore>), grid, block, bytes, stream, x, h, out_scores,
                               ScoreSpace{});
        return hipGetLastError();
    }
    static hipError_t shares(const fltop_rows& x, const fltop_hypotheses& h, const ScoreSpace& ws, hipStream_t stream) {
        const int W = waves_for(h.U, K);
        hipLaunchKernelGGL((shares_kernel<K, R, THREADS, TABLE>), dim3((unsigned)(x.B * h.N)), dim3(2 * kWave * W),
                           Lds<R>::bytes(W, x.V, h.U, false), stream, x, h, ws);
        return hipGetLastError();
    }
};

// Calls `f` with the build for these shapes.
template <typename F>
hipError_t with_build(const fltop_rows& x, const fltop_hypotheses& h, F f) {
    const bool table = x.V <= kTabulated;
    switch (lattice_pairs(x.B, h.N, h.U)) {
        case 1: return table ? f(Build<1, 8, 256, true>{}) : f(Build<1, 8, 256, false>{});
        case 2: return table ? f(Build<2, 8, 256, true>{}) : f(Build<2, 8, 256, false>{});
        case 4: return table ? f(Build<4, 4, 256, true>{}) : f(Build<4, 4, 256, false>{});
        default:
            if (waves_for(h.U, 8) <= 2) return table ? f(Build<8, 4, 256, true>{}) : f(Build<8, 4, 256, false>{});
            return table ? f(Build<8, 4, 1024, true>{}) : f(Build<8, 4, 1024, false>{});
    }
}

template <typename T>
hipError_t grad_of(const fltop_rows& x, const fltop_hypotheses& h, const double* grad_scores, const ScoreSpace& ws,
                   void* grad, hipStream_t stream) {
    // frames of a wavefront: as many as fit 16 KB (a workgroup's 64 KB leave room for two on a compute unit)
    int32_t per_wave = 2048 / x.V;
    per_wave = per_wave < 1 ? 1 : per_wave > kGradFrames ? kGradFrames : per_wave;
    const int32_t chunks = (x.T + per_wave - 1) / per_wave;
    const int waves = x.V > 2048 ? 2 : kGradWaves;
    const int64_t blocks = ((int64_t)x.B * chunks + waves - 1) / waves;
    hipLaunchKernelGGL(score_grad_kernel<T>, dim3((unsigned)blocks), dim3(waves * kWave),
                       (size_t)waves * per_wave * x.V * sizeof(unsigned long long), stream, x, h, grad_scores, ws,
                       per_wave, chunks, kWave * lattice_pairs(x.B, h.N, h.U), static_cast<T*>(grad));
    return hipGetLastError();
}

}  // namespace

hipError_t launch_score(const fltop_rows& x, const fltop_hypotheses& h, double* out_scores, const ScoreSpace* keep,
                        hipStream_t stream) {
    return with_build(x, h, [&](auto build) { return decltype(build)::score(x, h, out_scores, keep, stream); });
}

hipError_t launch_score_grad(const fltop_rows& x, const fltop_hypotheses& h, const double* grad_scores,
                             const ScoreSpace& ws, void* grad, hipStream_t stream) {
    const hipError_t e = with_build(x, h, [&](auto build) { return decltype(build)::shares(x, h, ws, stream); });
    if (e != hipSuccess) return e;
    if (x.type == FLTOP_TYPE_BF16) return grad_of<__hip_bfloat16>(x, h, grad_scores, ws, grad, stream);
    if (x.type == FLTOP_TYPE_F16) return grad_of<__half>(x, h, grad_scores, ws, grad, stream);
    return grad_of<float>(x, h, grad_scores, ws, grad, stream);
}

}  // namespace fltop
