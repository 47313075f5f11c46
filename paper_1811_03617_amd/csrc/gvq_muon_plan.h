// The units in which the Newton-Schulz steps keep their numbers, and the tiles that their products take.  Plain C++: nothing here needs HIP.
#pragma once
#include <cmath>
#include <cstdint>

#if defined(__HIPCC__)
#define NS_BOTH __host__ __device__ inline
#else
#define NS_BOTH inline
#endif

// X, A = X X^T and the polynomial P = b A + c A A are kept as two f16 terms per number, 22 bits down to a smallest step and up to 65504:
// X in units of 2^-(12 + k), A in 2^-(12 + 2 k), P in 2^-(10 + j).  With k = j = 0, the ordinary case, that is |X| and |A| below 16, which singular values
// below 4 keep, and |P| below 64; what goes beyond becomes NaN.  Small numbers would lose their last bits (of |U| = 1e-11 beside eps = 1e-7
// 3e-5, of 1e-13 all but three digits), so k and j follow the numbers' bounds downwards: singular values are at most the
// Frobenius norm r = |U| / (|U| + eps) at the start and the largest |a s + b s^3 + c s^5| over [0, S] behind a step from at most S; A's entries are
// at most S^2, P's the largest |b x + c x^2| over [0, S^2].  Never upwards: a bound that is far above the numbers themselves, as behind coefficients that
// would let X grow, would cost the bits that it is to save.
#define NS_X_BITS 12
#define NS_P_BITS 10

// The largest |a s + b s^3 + c s^5| for s from 0 to S: at S or where the derivative a + 3 b x + 5 c x^2, x = s^2, is 0.
NS_BOTH double ns_step_bound(double a, double b, double c, double S)
{
    auto at = [=](double x) { return std::fabs(std::sqrt(x) * (a + x * (b + x * c))); };
    const double top = S * S;
    double most = at(top);
    auto look = [&](double x) {
        if (x > 0.0 && x < top) {
            const double v = at(x);
            most = v > most ? v : most;
        }
    };
    const double d = 9.0 * b * b - 20.0 * a * c;
    if (d >= 0.0) {
        const double q = -0.5 * (3.0 * b + (b < 0.0 ? -std::sqrt(d) : std::sqrt(d)));
        if (c != 0.0) look(q / (5.0 * c));
        if (q != 0.0) look(a / q);
    }
    return most;
}
// The largest |b x + c x^2| for x from 0 to S^2.
NS_BOTH double ns_poly_bound(double b, double c, double S)
{
    const double top = S * S;
    double most = std::fabs(top * (b + top * c));
    if (c != 0.0) {
        const double x = -b / (2.0 * c);
        if (x > 0.0 && x < top && std::fabs(0.5 * b * x) > most) most = std::fabs(0.5 * b * x);
    }
    return most;
}

// k for a bound S: 0 above 1/2, otherwise S 2^k is in [1/2, 1).
NS_BOTH int ns_unit_x(double S)
{
    if (!(S > 0.0 && S <= 0.5)) return 0;
    int e;
    std::frexp(S, &e);
    return -e;
}
// j for a bound B: 0 from 1/16 on and for B = 0, otherwise B 2^j is in [1, 2).
NS_BOTH int ns_unit_p(double B)
{
    if (!(B > 0.0 && B < 0.0625)) return 0;
    int e;
    std::frexp(B, &e);
    return 1 - e;
}

// What a step's kernels multiply with: P = pa A + pc (A A), X' = sa X + ss (P X), all in their units; out X' is the result.
struct NsFactors {
    float pa, pc, sa, ss, out;
};

// Norms above this share of |U| + eps are taken for all of it: the usual case, for which the factors are known beforehand.
#define NS_WHOLE 0.5

NS_BOTH bool ns_is_whole(double r) { return !(r > 0.0 && r <= NS_WHOLE); }   // (NaN: whatever the factors are, X is NaN; 0: X is 0)

// Factors of all steps from singular values of at most S.  coef: [steps][3].
NS_BOTH void ns_factors(const float* coef, int steps, double S, NsFactors* f)
{
    int k = ns_unit_x(S);
    for (int t = 0; t < steps; ++t) {
        const double a = coef[3 * t], b = coef[3 * t + 1], c = coef[3 * t + 2];
        const int j = ns_unit_p(ns_poly_bound(b, c, S));
        S = ns_step_bound(a, b, c, S);
        const int next = t + 1 < steps ? ns_unit_x(S) : k;
        f[t].pa = (float)std::ldexp(b, NS_P_BITS + j - NS_X_BITS - 2 * k);
        f[t].pc = (float)std::ldexp(c, NS_P_BITS + j - 2 * NS_X_BITS - 4 * k);
        f[t].sa = (float)std::ldexp(a, next - k);
        f[t].ss = (float)std::ldexp(1.0, next - k - NS_P_BITS - j);
        f[t].out = (float)std::ldexp(1.0, -NS_X_BITS - next);
        k = next;
    }
}

// ---- tiles ------------------------------------------------------------------------------------------------------------

inline int64_t ns_padded(int64_t n) { return (n + 31) / 32 * 32; }

// Which tiles a product takes, and in how many parts its sum is cut.
struct NsChoice {
    int shape = 0, splits = 1;
};

// Tile shapes: 256, 128 and 64 on both sides, and 192 for products whose operands both run along the sum.  The times are fitted to 43
// products of single matrices (64 to 4096 rows, 64 to 16384 columns) each measured with every shape and up to 8 parts: of those what they pick is the fastest
// or at most 4 % (of the iteration) behind it.  They rank the ways and are no forecast: they know neither the clock under a full chip's load nor
// the bytes of X that a step reads and writes (4096 x 4096 227 us for a step that takes 338, 1000 x 4096 23 for 38, 5 of 512 x 4608 36 for 67).
struct NsShape {
    int size;
    double step_us, start_us;   // of one work-group on a compute unit: a step, and what a tile costs beside its steps
    int per_cu;                 // work-groups that share a compute unit (step_us is that of the pair)
};
static const NsShape ns_shapes[4] = {{256, 1.7, 9.0, 1}, {192, 1.08, 4.5, 1}, {128, 0.62, 3.3, 1}, {64, 0.48, 2.9, 2}};

// Whether tiles of a size come in parts: 64 x 64 for the Gram matrix of long rows alone (no size has them the fastest way elsewhere).
constexpr bool ns_in_parts(int size, bool gram) { return gram || size > 64; }

// Rounds of tiles over 256 compute units, with the sum cut in up to 8 parts where there are few tiles.  The parts go by one
// matrix alone: the tiles' shape does not change a result's bits, the parts do, and a matrix has the same result in every batch.
inline double ns_time(const NsShape& s, int64_t batch, int64_t rows, int64_t cols, int64_t steps, int splits, bool sym)
{
    const int64_t nm = (rows + s.size - 1) / s.size, nn = (cols + s.size - 1) / s.size;
    const int64_t tiles = batch * (sym ? nm * (nm + 1) / 2 : nm * nn) * splits;
    const int64_t rounds = (tiles + 256 * s.per_cu - 1) / (256 * s.per_cu);
    const double join = splits > 1 ? 10.0 + 0.56e-6 * batch * rows * cols * (splits + 1) * (sym ? 0.5 : 1.0) : 0.0;
    return rounds * (s.start_us + s.step_us * ((steps + splits - 1) / splits)) + join;
}

// sym: a symmetric product; gram: X X^T.
inline NsChoice ns_choose(int64_t batch, int64_t rows, int64_t cols, int64_t steps, bool sym, bool gram)
{
    NsChoice best;
    double least = 1e300;
    auto look = [&](int64_t of, int k, int splits) {
        if ((k == 1 && !sym) || (splits > 1 && !ns_in_parts(ns_shapes[k].size, gram))) return;
        const double t = ns_time(ns_shapes[k], of, rows, cols, steps, splits, sym);
        if (t < least) { least = t; best.shape = k; best.splits = splits; }
    };
    for (int splits = 1; splits <= 8 && (splits == 1 || splits * 2 <= steps); ++splits)
        for (int k = 0; k < 4; ++k) look(1, k, splits);
    if (batch > 1) {
        const int splits = best.splits;
        least = 1e300;
        for (int k = 0; k < 4; ++k) look(batch, k, splits);
    }
    return best;
}

// The three products of a step for X of m rows and n columns, m <= n.
struct NsWays {
    NsChoice gram, poly, step;
};
inline NsWays ns_ways(int64_t batch, int64_t m, int64_t n)
{
    return {ns_choose(batch, m, m, ns_padded(n) / 32, true, true), ns_choose(batch, m, m, ns_padded(m) / 32, true, false),
            ns_choose(batch, m, n, ns_padded(m) / 32, false, false)};
}

inline int64_t ns_part_numbers(const NsChoice& c, int64_t rows, int64_t cols)
{
    const int64_t s = ns_shapes[c.shape].size;
    return c.splits == 1 ? 0 : c.splits * ((rows + s - 1) / s * s) * ((cols + s - 1) / s * s);
}
