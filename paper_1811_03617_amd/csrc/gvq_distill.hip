// Divergence of a teacher's top logits from a student's softmax over all of its logits, for every row, and its gradient.
//
//   p = softmax(a / t) over the row's entries, q = softmax(z / t):  l = w t^2 sum_j p_j (log p_j - log q_j),  dz = w t (q - p).
//
// Powers are of 2, of (z - largest) c with c = log2(e) / t: the difference first, since z c alone may leave fp32 (masks of the type's lowest
// value) and loses bits that the difference keeps.  With e_j = 2^((a_j - top_a) c), A = sum e_j, S = sum_v 2^((z_v - top_z) c):
//   l = w t (sum_j e_j ((a_j - top_a) - (z_j - top_z)) / A + t ln 2 (log2 S - log2 A)),
// so that two rounds of joining are enough: the largest, then A, S and that sum, D.  D is held in 64 bits: at an entry that the student's mask
// covers the difference may be twice the type's largest number, and the loss of it, times w p, is a number still.
//
// A row to a wave, to four or to sixteen; each thread keeps its first words of the row in registers and reads only the rest a second
// time, for the gradient.  Bound: memory, each logit in and out once: 4096 x 131072 bf16 445 us (4.8 TB/s, a plain copy's 5.1), the losses alone 179 (6.0);
// 16384 x 4096 bf16 51; below that a launch and two joins, 2048 x 1000 fp32 7.6.
#include "gvq_distill.h"

// Eight neighbouring logits of a row, as they lie in memory.
template <typename T>
struct DistillWord {
    u4 v[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T* p)
    {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) v[i] = *((const u4*)p + i);
    }
    __device__ __forceinline__ void numbers(float (&f)[8]) const
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (sizeof(T) == 4) f[i] = __uint_as_float(v[i >> 2][i & 3]);
            else f[i] = __uint_as_float(i & 1 ? v[0][i >> 1] & 0xffff0000u : v[0][i >> 1] << 16);
        }
    }
};
__device__ __forceinline__ void distill_store8(float* p, const float (&v)[8])
{
    stream_store((f4*)p, f4{v[0], v[1], v[2], v[3]});
    stream_store((f4*)p + 1, f4{v[4], v[5], v[6], v[7]});
}
__device__ __forceinline__ void distill_store8(unsigned short* p, const float (&v)[8])
{
    stream_store((u4*)p, u4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])});
}
__device__ __forceinline__ float distill_load(const float* p) { return *p; }
__device__ __forceinline__ float distill_load(const unsigned short* p) { return bf16_to_f32(*p); }
__device__ __forceinline__ void distill_store(float* p, float v) { *p = v; }
__device__ __forceinline__ void distill_store(unsigned short* p, float v) { *p = (unsigned short)f32_to_bf16_rne(v); }

// Largest z so far and the sum of 2^((z - largest) c).  As long as there is nothing but -inf, `top` is -inf and differences are taken from 0.
__device__ __forceinline__ float distill_from(float top) { return top == -INFINITY ? 0.f : top; }
__device__ __forceinline__ float distill_power(float z, float from, float c) { return __builtin_amdgcn_exp2f((z - from) * c); }
template <bool WARM>
struct DistillSum {
    typedef float Number;
    float top = -INFINITY, sum = 0.f;
    template <int N>
    __device__ __forceinline__ void add(const DistillArgs& a, const float (&v)[N])
    {
        const float c = a.log2_t;
        float m = v[0];
#pragma unroll
        for (int i = 1; i < N; ++i) m = fmaxf(m, v[i]);
        m = fmaxf(top, m);
        const float from = distill_from(m);
        float s = sum * distill_power(top, from, c);
#pragma unroll
        for (int i = 0; i < N; ++i) s += distill_power(v[i], from, c);
        sum = s;
        top = m;
    }
    __device__ __forceinline__ float seen_from(const DistillArgs& a, float from) const { return sum * distill_power(top, from, a.log2_t); }
};

// High temperatures.  The loss is t^2 times a difference of logarithms, which are near each other where the entries hold most of the softmax: an
// error of 2^-24 in S or A counts t^2 times, while the loss does not grow with t (1000 logits, all of them entries, off by, relative: 6e-6 at t = 8,
// 3e-5 at 20, 9e-4 at 100, 8 % at 1000; this way 3e-7 at any).  Above DISTILL_WARM therefore, with x = (z - from) / t from a number `from` near z's,
//   sum of e^x = sum of 1 + x + r(x) where |x| < 1, and of e^x elsewhere,   r(x) = e^x - 1 - x = x^2 P(x),
// the number of the first and their sum of z in 64 bits, which holds that sum exactly where |z| is large against t.  What is left in 32 bits, r and
// the other powers, is off by a few 2^-24 of x^2 at most, and that times t^2 is (z - from)^2, whatever t is.  `from` is a thread's first
// word's largest, and moves only where powers would leave fp32.  Entries, logarithms and joined sums are in 64 bits.
// Its price is arithmetic, and why it is not the way for all (us, the other way and this): 4096 x 131072 bf16 444 and 640, the losses alone 178 and 318, 2048 x
// 131072 fp32 517 and 530, 8192 x 2048 bf16 18.6 and 28, 16 x 50021 fp32 12.0 and 18.1.
#define DISTILL_WARM 8.0
template <>
struct DistillSum<true> {
    typedef double Number;
    float top = -INFINITY, ref = -INFINITY;
    double z = 0.0, more = 0.0;   // of the near ones; r and the other powers
    int near = 0;
    template <int N>
    __device__ __forceinline__ void add(const DistillArgs& a, const float (&v)[N])
    {
        float m = v[0];
#pragma unroll
        for (int i = 1; i < N; ++i) m = fmaxf(m, v[i]);
        top = fmaxf(top, m);
        if ((m - ref) * a.per_t > 60.f) {   // (-inf - -inf is no number)
            more = seen_from(a, m);
            z = 0.0;
            near = 0;
            ref = m;
        }
        const float from = distill_from(ref);
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float x = (v[i] - from) * a.per_t;
            const bool is_near = fabsf(x) < 1.f;   // (not so of a NaN)
            float p = 1.f / 3628800;               // (x^9 / 11! is 7e-8 of P at most)
            p = __builtin_fmaf(p, x, 1.f / 362880);
            p = __builtin_fmaf(p, x, 1.f / 40320);
            p = __builtin_fmaf(p, x, 1.f / 5040);
            p = __builtin_fmaf(p, x, 1.f / 720);
            p = __builtin_fmaf(p, x, 1.f / 120);
            p = __builtin_fmaf(p, x, 1.f / 24);
            p = __builtin_fmaf(p, x, 1.f / 6);
            p = __builtin_fmaf(p, x, 0.5f);
            s += is_near ? x * x * p : distill_power(v[i], from, a.log2_t);
            z += is_near ? (double)v[i] : 0.0;
            near += is_near;
        }
        more += (double)s;
    }
    __device__ __forceinline__ double seen_from(const DistillArgs& a, float from) const
    {
        if (ref == -INFINITY) return more;   // nothing but -inf and NaN
        const double per = 1.0 / a.t64, sum = near == 0 ? more : more + (double)near + (z - (double)near * (double)ref) * per;
        return ref == from ? sum : sum * exp(((double)ref - (double)from) * per);
    }
};

// A row's numbers before the first whole word of 16 bytes.
template <typename T>
__device__ __forceinline__ int distill_head(const T* p, int n)
{
    const int h = (int)((16 - ((uintptr_t)p & 15)) & 15) / (int)sizeof(T);
    return h < n ? h : n;
}

// What all lanes of a wave hold, joined, for every lane: along rows of 16 lanes, then the rows.  `none` joins without effect.
template <int CTRL, int ROWS>
__device__ __forceinline__ float distill_lane(float none, float v)
{
    return __uint_as_float((unsigned int)__builtin_amdgcn_update_dpp((int)__float_as_uint(none), (int)__float_as_uint(v), CTRL, ROWS, 0xf, false));
}
template <typename F>
__device__ __forceinline__ float wave_all(float v, float none, F join)
{
    v = join(v, distill_lane<0x111, 0xf>(none, v));   // row_shr 1, 2, 4, 8
    v = join(v, distill_lane<0x112, 0xf>(none, v));
    v = join(v, distill_lane<0x114, 0xf>(none, v));
    v = join(v, distill_lane<0x118, 0xf>(none, v));
    v = join(v, distill_lane<0x142, 0xa>(none, v));   // row_bcast 15, 31
    v = join(v, distill_lane<0x143, 0xc>(none, v));
    return __uint_as_float((unsigned int)__builtin_amdgcn_readlane((int)__float_as_uint(v), 63));
}
// Three values over a row's team of threads.  part: [3][TEAM / 64], of this call alone.
template <int TEAM, typename F>
__device__ __forceinline__ void team_all(float (&v)[3], float none, float* part, F join)
{
    constexpr int WAVES = TEAM / 64;
#pragma unroll
    for (int k = 0; k < 3; ++k) v[k] = wave_all(v[k], none, join);
    if constexpr (WAVES > 1) {
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < 3; ++k) part[k * WAVES + (threadIdx.x >> 6)] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            v[k] = part[k * WAVES];
#pragma unroll
            for (int i = 1; i < WAVES; ++i) v[k] = join(v[k], part[k * WAVES + i]);
        }
    }
}
// Two values of 32 bits, summed for everybody, and one of 64 bits, summed for the first thread: only the loss needs it.  part: [2][TEAM / 64], part_d: [TEAM / 64].
__device__ __forceinline__ double wave_sum(double v)
{
    auto from = [&](auto ctrl, auto rows) {   // (lanes that nothing comes to get 0.0)
        const uint64_t b = __builtin_bit_cast(uint64_t, v);
        const unsigned int lo = (unsigned int)__builtin_amdgcn_update_dpp(0, (int)b, decltype(ctrl)::value, decltype(rows)::value, 0xf, false),
                           hi = (unsigned int)__builtin_amdgcn_update_dpp(0, (int)(b >> 32), decltype(ctrl)::value, decltype(rows)::value, 0xf, false);
        v += __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
    };
    typedef std::integral_constant<int, 0xf> All;
    from(std::integral_constant<int, 0x111>{}, All{});
    from(std::integral_constant<int, 0x112>{}, All{});
    from(std::integral_constant<int, 0x114>{}, All{});
    from(std::integral_constant<int, 0x118>{}, All{});
    from(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});
    from(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const unsigned int lo = (unsigned int)__builtin_amdgcn_readlane((int)b, 63), hi = (unsigned int)__builtin_amdgcn_readlane((int)(b >> 32), 63);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
template <int TEAM>
__device__ __forceinline__ void team_sums(float (&v)[2], double& d, float* part, double* part_d)
{
    constexpr int WAVES = TEAM / 64;
#pragma unroll
    for (int k = 0; k < 2; ++k) v[k] = wave_all(v[k], 0.f, [](float a, float b) { return a + b; });
    d = wave_sum(d);
    if constexpr (WAVES > 1) {
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int k = 0; k < 2; ++k) part[k * WAVES + (threadIdx.x >> 6)] = v[k];
            part_d[threadIdx.x >> 6] = d;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            v[k] = part[k * WAVES];
#pragma unroll
            for (int i = 1; i < WAVES; ++i) v[k] += part[k * WAVES + i];
        }
        if (threadIdx.x == 0)
#pragma unroll
            for (int i = 1; i < WAVES; ++i) d += part_d[i];
    }
}
template <int TEAM>
__device__ __forceinline__ void team_sums(double (&v)[2], double& d, double* part, double* part_d)
{
    constexpr int WAVES = TEAM / 64;
#pragma unroll
    for (int k = 0; k < 2; ++k) v[k] = wave_sum(v[k]);
    d = wave_sum(d);
    if constexpr (WAVES > 1) {
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int k = 0; k < 2; ++k) part[k * WAVES + (threadIdx.x >> 6)] = v[k];
            part_d[threadIdx.x >> 6] = d;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            v[k] = part[k * WAVES];
            for (int i = 1; i < WAVES; ++i) v[k] += part[k * WAVES + i];
        }
        if (threadIdx.x == 0)
            for (int i = 1; i < WAVES; ++i) d += part_d[i];
    }
}
struct JoinMax {
    __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
template <int TEAM>
__device__ __forceinline__ void team_sync()
{
    if constexpr (TEAM > 64) __syncthreads();
    else wave_lds_sync();
}

// A row's entries in LDS: the teacher's logits and then e, the student's logits there, their places (-1: absent).
struct DistillEntries {
    float *e, *z;
    int* at;
};
template <int TEAM, typename T>
__device__ __forceinline__ void distill_entries(const DistillArgs& a, int64_t row, int t, const T* z, const DistillEntries& n, float& any, float& top)
{
    any = 0.f;
    top = -INFINITY;
    for (int j = t; j < a.n_top; j += TEAM) {
        const int64_t i = a.index[row * a.ld_index + j], at = row * a.ld_top + j;
        const bool there = i >= 0 && i < a.vocab;
        float v = -INFINITY, s = 0.f;
        if (there) {
            v = a.top_bf16 ? bf16_to_f32(((const unsigned short*)a.top)[at]) : ((const float*)a.top)[at];
            s = distill_load(z + i);
            any = 1.f;
        }
        n.at[j] = there ? (int)i : -1;
        n.e[j] = v;
        n.z[j] = s;
        top = fmaxf(top, v);
    }
}
// A and the sum of the loss.
__device__ __forceinline__ float distill_entry(const DistillArgs& a, float v, float top, float) { return __builtin_amdgcn_exp2f((v - top) * a.log2_t); }
__device__ __forceinline__ double distill_entry(const DistillArgs& a, float v, float top, double) { return exp(((double)v - (double)top) / a.t64); }
template <int TEAM, typename N>
__device__ __forceinline__ void distill_sums(const DistillArgs& a, int t, const DistillEntries& n, float top, float from, N& A, double& D)
{
    A = 0;
    D = 0.0;
    for (int j = t; j < a.n_top; j += TEAM)
        if (n.at[j] >= 0) {
            const float v = n.e[j];
            const N e = distill_entry(a, v, top, N());
            n.e[j] = (float)e;
            A += e;
            if (e != 0) D += (double)e * (((double)v - (double)top) - ((double)n.z[j] - (double)from));   // (0 log 0 is 0)
        }
}
__device__ __forceinline__ float distill_loss(const DistillArgs& a, float w, const float (&s)[2], double D)   // s: A and S
{
    const double logs = (double)(__builtin_amdgcn_logf(s[1]) - __builtin_amdgcn_logf(s[0])) * 0.69314718055994531;
    return (float)((double)w * (double)a.t * (D * (double)(1.f / s[0]) + (double)a.t * logs));
}
__device__ __forceinline__ float distill_loss(const DistillArgs& a, float w, const double (&s)[2], double D)
{
    return (float)((double)w * a.t64 * (D / s[0] + a.t64 * (log(s[1]) - log(s[0]))));
}
// The gradient at the entries' places in [lo, hi), once the rest has been written; the first of several entries of one place has the
// sum of all.
template <int TEAM, typename T>
__device__ __forceinline__ void distill_places(const DistillArgs& a, int t, const DistillEntries& n, T* g, int lo, int hi, float from, float scale, float per)
{
    for (int j = t; j < a.n_top; j += TEAM) {
        const int at = n.at[j];
        if (at < lo || at >= hi) continue;
        float sum = 0.f;
        bool first = true;
        for (int k = 0; k < a.n_top; ++k)
            if (n.at[k] == at) {
                if (k < j) first = false;
                sum += n.e[k];
            }
        if (first) distill_store(g + at, distill_power(n.z[j], from, a.log2_t) * scale - sum * per);
    }
}

// The gradient of eight neighbours.
template <typename T>
__device__ __forceinline__ void distill_out(const DistillWord<T>& word, T* g, bool same, float from, float c, float scale)
{
    float v[8];
    word.numbers(v);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = distill_power(v[k], from, c) * scale;
    if (same) distill_store8(g, v);
    else
#pragma unroll
        for (int k = 0; k < 8; ++k) distill_store(g + k, v[k]);
}

// TEAM threads a row (64: four rows a work-group), HOLD times eight logits of each in registers.
template <typename T, int TEAM, int HOLD, bool GRAD, bool WARM>
__global__ __launch_bounds__(TEAM > 64 ? TEAM : 256, TEAM > 256 && !WARM ? 8 : 4) void distill_row_kernel(DistillArgs a)
{
    typedef typename DistillSum<WARM>::Number Number;
    constexpr int ROWS = TEAM > 64 ? 1 : 4;
    extern __shared__ __attribute__((aligned(16))) char lds[];   // [ROWS][3][n_top]
    __shared__ float part[3 * TEAM / 64];
    __shared__ Number part_s[2 * TEAM / 64];
    __shared__ double part_d[TEAM / 64];
    const int t = threadIdx.x % TEAM, which = threadIdx.x / TEAM;
    const int64_t row = (int64_t)blockIdx.x * ROWS + which;
    if (ROWS > 1 && row >= a.rows) return;
    const T* z = (const T*)a.logits + row * a.ld;
    T* g = GRAD ? (T*)a.grad + row * a.ld_grad : nullptr;
    const float w = a.weight ? a.weight[row] : 1.f, c = a.log2_t;
    DistillEntries n;
    n.e = (float*)lds + which * 3 * a.n_top;
    n.z = n.e + a.n_top;
    n.at = (int*)(n.z + a.n_top);
    float round[3] = {0.f, -INFINITY, -INFINITY};   // any entries, the largest of them, the largest logit
    const int head = distill_head(z, a.vocab), words = (a.vocab - head) / 8, rest = a.vocab - 8 * words;
    DistillWord<T> held[HOLD];
    DistillSum<WARM> sum;
    if (w != 0.f) {
#pragma unroll
        for (int i = 0; i < HOLD; ++i)
            if (t + i * TEAM < words) held[i].load(z + head + 8 * (t + i * TEAM));
        distill_entries<TEAM>(a, row, t, z, n, round[0], round[1]);
#pragma unroll
        for (int i = 0; i < HOLD; ++i)
            if (t + i * TEAM < words) {
                float v[8];
                held[i].numbers(v);
                sum.add(a, v);
            }
        for (int i = t + HOLD * TEAM; i < words; i += TEAM) {
            DistillWord<T> word;
            float v[8];
            word.load(z + head + 8 * i);
            word.numbers(v);
            sum.add(a, v);
        }
        for (int i = t; i < rest; i += TEAM) {
            const float v[1] = {distill_load(z + (i < head ? i : 8 * words + i))};
            sum.add(a, v);
        }
        round[2] = sum.top;
    }
    team_all<TEAM>(round, -INFINITY, part, JoinMax());
    if (!(round[0] > 0.f)) {   // weight 0 or no entries
        if (t == 0) a.loss[row] = 0.f;
        if (GRAD)
            for (int i = t; i < a.vocab; i += TEAM) distill_store(g + i, 0.f);
        return;
    }
    const float from = distill_from(round[2]);
    Number sums[2];   // A, S
    double D;
    distill_sums<TEAM>(a, t, n, round[1], from, sums[0], D);
    sums[1] = sum.seen_from(a, from);
    team_sums<TEAM>(sums, D, part_s, part_d);
    if (t == 0) a.loss[row] = distill_loss(a, w, sums, D);
    if constexpr (GRAD) {
        const float scale = w * a.t / (float)sums[1];
        const bool same = (((uintptr_t)g ^ (uintptr_t)z) & 15) == 0;
        // the rest backwards: what was read last is in the caches still (2048 x 131072 fp32 596 us forwards, 502 so, 4096 x 65536 544 and 448; bf16, a
        // row's rest being shorter, 422 and 417)
        const int rest_words = words - t - HOLD * TEAM;
        for (int i = rest_words > 0 ? (rest_words - 1) / TEAM : -1; i >= 0; --i) {
            const int at = head + 8 * (t + (HOLD + i) * TEAM);
            DistillWord<T> word;
            word.load(z + at);
            distill_out(word, g + at, same, from, c, scale);
        }
#pragma unroll
        for (int i = 0; i < HOLD; ++i)
            if (t + i * TEAM < words) distill_out(held[i], g + head + 8 * (t + i * TEAM), same, from, c, scale);
        for (int i = t; i < rest; i += TEAM) {
            const int at = i < head ? i : 8 * words + i;
            distill_store(g + at, distill_power(distill_load(z + at), from, c) * scale);
        }
        team_sync<TEAM>();
        distill_places<TEAM>(a, t, n, g, 0, a.vocab, from, scale, w * a.t / (float)sums[0]);
    }
}

// ---- few rows of many logits -----------------------------------------------------------------------------------------

// A row in `parts` pieces of whole words; its sums and largest logits go into sums [rows][parts][2], and a second launch joins them.
struct DistillPiece {
    int lo, hi;
};
__device__ __forceinline__ DistillPiece distill_piece(int vocab, int parts, int part)
{
    const int per = ((vocab + parts - 1) / parts + 7) / 8 * 8;
    const int lo = per * part < vocab ? per * part : vocab;
    return {lo, vocab - lo < per ? vocab : lo + per};
}
// Each number of the piece that is this thread's, by words where they can be.
template <int TEAM, typename T, typename F8, typename F1>
__device__ __forceinline__ void distill_each(const T* z, DistillPiece p, F8 word, F1 one)
{
    const int n = p.hi - p.lo, head = distill_head(z + p.lo, n), words = (n - head) / 8, rest = n - 8 * words;
    for (int i = threadIdx.x; i < words; i += TEAM) word(p.lo + head + 8 * i);
    for (int i = threadIdx.x; i < rest; i += TEAM) one(p.lo + (i < head ? i : 8 * words + i));
}

template <typename T, int TEAM, bool WARM>
__global__ __launch_bounds__(TEAM) void distill_part_kernel(DistillArgs a, int parts, typename DistillSum<WARM>::Number* sums)
{
    typedef typename DistillSum<WARM>::Number Number;
    __shared__ float shared[3 * TEAM / 64];
    __shared__ Number shared_s[2 * TEAM / 64];
    __shared__ double shared_d[TEAM / 64];
    const int64_t row = blockIdx.x / parts;
    const int part = blockIdx.x % parts;
    if (a.weight && a.weight[row] == 0.f) return;   // (nobody reads its sums)
    const T* z = (const T*)a.logits + row * a.ld;
    DistillSum<WARM> sum;
    distill_each<TEAM>(z, distill_piece(a.vocab, parts, part), [&](int i) {
        DistillWord<T> word;
        float v[8];
        word.load(z + i);
        word.numbers(v);
        sum.add(a, v);
    }, [&](int i) {
        const float v[1] = {distill_load(z + i)};
        sum.add(a, v);
    });
    float top[3] = {sum.top, -INFINITY, -INFINITY};
    team_all<TEAM>(top, -INFINITY, shared, JoinMax());
    Number s[2] = {sum.seen_from(a, distill_from(top[0])), 0};
    double none = 0.0;
    team_sums<TEAM>(s, none, shared_s, shared_d);
    if (threadIdx.x == 0) {
        sums[2 * (row * parts + part)] = s[0];
        sums[2 * (row * parts + part) + 1] = top[0];
    }
}

// A piece's sum from the largest logit of the row.
__device__ __forceinline__ float distill_join(const DistillArgs& a, float sum, float top, float from) { return sum * distill_power(top, from, a.log2_t); }
__device__ __forceinline__ double distill_join(const DistillArgs& a, double sum, float top, float from)
{
    return sum * exp(((double)top - (double)from) / a.t64);
}

template <typename T, int TEAM, bool GRAD, bool WARM>
__global__ __launch_bounds__(TEAM) void distill_join_kernel(DistillArgs a, int parts, const typename DistillSum<WARM>::Number* sums)
{
    typedef typename DistillSum<WARM>::Number Number;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ float shared[3 * TEAM / 64];
    __shared__ Number shared_s[2 * TEAM / 64];
    __shared__ double shared_d[TEAM / 64];
    const int pieces = GRAD ? parts : 1, t = threadIdx.x;
    const int64_t row = blockIdx.x / pieces;
    const DistillPiece piece = distill_piece(a.vocab, parts, blockIdx.x % pieces);
    const T* z = (const T*)a.logits + row * a.ld;
    T* g = GRAD ? (T*)a.grad + row * a.ld_grad : nullptr;
    const float w = a.weight ? a.weight[row] : 1.f, c = a.log2_t;
    DistillEntries n;
    n.e = (float*)lds;
    n.z = n.e + a.n_top;
    n.at = (int*)(n.z + a.n_top);
    float round[3] = {0.f, -INFINITY, -INFINITY};
    Number sum = 0;
    float top = -INFINITY;
    if (w != 0.f) {
        distill_entries<TEAM>(a, row, t, z, n, round[0], round[1]);
        if (t < parts) {
            sum = sums[2 * (row * parts + t)];
            top = (float)sums[2 * (row * parts + t) + 1];
        }
        round[2] = top;
    }
    team_all<TEAM>(round, -INFINITY, shared, JoinMax());
    if (!(round[0] > 0.f)) {
        if (t == 0 && piece.lo == 0) a.loss[row] = 0.f;
        if (GRAD)
            for (int i = piece.lo + t; i < piece.hi; i += TEAM) distill_store(g + i, 0.f);
        return;
    }
    const float from = distill_from(round[2]);
    Number s[2];
    double D;
    distill_sums<TEAM>(a, t, n, round[1], from, s[0], D);
    s[1] = distill_join(a, sum, top, from);
    team_sums<TEAM>(s, D, shared_s, shared_d);
    if (t == 0 && piece.lo == 0) a.loss[row] = distill_loss(a, w, s, D);
    if constexpr (GRAD) {
        const float scale = w * a.t / (float)s[1];
        const bool same = (((uintptr_t)g ^ (uintptr_t)z) & 15) == 0;
        distill_each<TEAM>(z, piece, [&](int i) {
            DistillWord<T> word;
            word.load(z + i);
            distill_out(word, g + i, same, from, c, scale);
        }, [&](int i) { distill_store(g + i, distill_power(distill_load(z + i), from, c) * scale); });
        __syncthreads();
        distill_places<TEAM>(a, t, n, g, piece.lo, piece.hi, from, scale, w * a.t / (float)s[0]);
    }
}

template <typename T, int TEAM, int HOLD, bool WARM>
static int launch_rows(const DistillArgs& a, hipStream_t st)
{
    constexpr int ROWS = TEAM > 64 ? 1 : 4;
    const unsigned lds = (unsigned)(ROWS * 12 * a.n_top);
    const dim3 grid((unsigned)((a.rows + ROWS - 1) / ROWS)), threads(TEAM > 64 ? TEAM : 256);
    if (a.grad) hipLaunchKernelGGL((distill_row_kernel<T, TEAM, HOLD, true, WARM>), grid, threads, lds, st, a);
    else hipLaunchKernelGGL((distill_row_kernel<T, TEAM, HOLD, false, WARM>), grid, threads, lds, st, a);
    GVQ_HIP(hipGetLastError());
    return GVQ_OK;
}

#define DISTILL_TEAM 256   // of a piece

// Few rows of many logits leave most of the chip idle while each waits for its own loads; in pieces of at least 2048 they fill it, for a second
// launch (whole and in pieces, us with the gradient: 1 x 65536 bf16 12.1 and 7.9, 1 x 131072 18.7 and 7.8, 64 x 131072 20.1 and 13.1, 96 x 65536 13.4 and
// 13.0, 96 x 262144 39 and 35; 112 x 131072 20.5 and 21.4).  That launch and its workspace are 4 us of the host's time: 16 x 50021 fp32 takes
// 12.1 whole and 9.8 in pieces, but 11.3 and 14.5 where Python makes one call after the other, so that shorter rows stay whole.  Pieces of at least 8192
// instead: 1.5 us more for one row, nothing from 64 on.
int gvq_distill_parts(int64_t rows, int64_t vocab)
{
    if (rows > 96 || vocab < 65536) return 1;
    const int64_t want = (512 + rows - 1) / rows, most = vocab / 2048 < DISTILL_TEAM ? vocab / 2048 : DISTILL_TEAM;   // (a thread each joins them)
    return (int)(want < most ? want : most);
}

template <typename T, bool WARM>
static int launch_distill(const DistillArgs& a, void* workspace, hipStream_t st)
{
    // in place the second launch's work-groups would read the student's logits at entries that another piece's have replaced: rows stay whole.  Warm: a
    // piece's numbers are of 64 bits, and there are half as many for the same workspace.
    const int parts = a.grad == a.logits ? 1 : gvq_distill_parts(a.rows, a.vocab) / (WARM ? 2 : 1);
    if (parts > 1) {
        auto* sums = (typename DistillSum<WARM>::Number*)workspace;
        const unsigned lds = (unsigned)(12 * a.n_top);
        const dim3 grid((unsigned)(a.rows * parts)), threads(DISTILL_TEAM);
        hipLaunchKernelGGL((distill_part_kernel<T, DISTILL_TEAM, WARM>), grid, threads, 0, st, a, parts, sums);
        GVQ_HIP(hipGetLastError());
        if (a.grad) hipLaunchKernelGGL((distill_join_kernel<T, DISTILL_TEAM, true, WARM>), grid, threads, lds, st, a, parts, sums);
        else hipLaunchKernelGGL((distill_join_kernel<T, DISTILL_TEAM, false, WARM>), dim3((unsigned)a.rows), threads, lds, st, a, parts, sums);
        GVQ_HIP(hipGetLastError());
        return GVQ_OK;
    }
    // by a row's bytes.  A wave, four and sixteen of them (us with the gradient): 16384 x 1000 bf16 23, 37; 8192 x 2048 bf16 19, 23; 8192 x 2048 fp32
    // 36, 30; 4096 x 8192 bf16 35, 28, 48; 8192 x 4096 fp32 77, 54, 81; 4096 x 16384 bf16 -, 50, 60; 4096 x 32000 bf16 -, 112, 107; 64 x 32000 -, 13,
    // 9.2.  Many entries would take a wave's row too much LDS, and a launch has fewer than 2^32 threads.
    const int64_t bytes = (int64_t)a.vocab * (int64_t)sizeof(T);
    if (bytes <= 4096 && a.n_top <= 256) return launch_rows<T, 64, sizeof(T) == 2 ? 4 : 2, WARM>(a, st);
    if (bytes <= (a.rows >= 1024 ? 32768 : 16384) || a.rows * 1024 > 0xffffffffll) return launch_rows<T, 256, 4, WARM>(a, st);
    return launch_rows<T, 1024, sizeof(T) == 2 ? 6 : 3, WARM>(a, st);
}

int gvq_launch_distill(const DistillArgs& a, gvq_dtype_t dtype, void* workspace, hipStream_t st)
{
    const bool warm = a.t64 > DISTILL_WARM;
    if (dtype == GVQ_BF16) return warm ? launch_distill<unsigned short, true>(a, workspace, st) : launch_distill<unsigned short, false>(a, workspace, st);
    return warm ? launch_distill<float, true>(a, workspace, st) : launch_distill<float, false>(a, workspace, st);
}
