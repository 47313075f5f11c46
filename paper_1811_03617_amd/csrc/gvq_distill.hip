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
struct DistillSum {
    float top, sum;
};
__device__ __forceinline__ float distill_from(float top) { return top == -INFINITY ? 0.f : top; }
__device__ __forceinline__ float distill_power(float z, float from, float c) { return __builtin_amdgcn_exp2f((z - from) * c); }
template <int N>
__device__ __forceinline__ void distill_add(DistillSum& a, const float (&v)[N], float c)
{
    float m = v[0];
#pragma unroll
    for (int i = 1; i < N; ++i) m = fmaxf(m, v[i]);
    m = fmaxf(a.top, m);
    const float from = distill_from(m);
    float s = a.sum * distill_power(a.top, from, c);
#pragma unroll
    for (int i = 0; i < N; ++i) s += distill_power(v[i], from, c);
    a.sum = s;
    a.top = m;
}

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
struct JoinMax {
    __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
struct JoinSum {
    __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
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
template <int TEAM>
__device__ __forceinline__ void distill_sums(const DistillArgs& a, int t, const DistillEntries& n, float top, float from, float& A, double& D)
{
    A = 0.f;
    D = 0.0;
    for (int j = t; j < a.n_top; j += TEAM)
        if (n.at[j] >= 0) {
            const float v = n.e[j], e = __builtin_amdgcn_exp2f((v - top) * a.log2_t);
            n.e[j] = e;
            A += e;
            if (e != 0.f) D += (double)e * (((double)v - (double)top) - ((double)n.z[j] - (double)from));   // (0 log 0 is 0)
        }
}
__device__ __forceinline__ float distill_loss(float w, float t, float A, float S, double D)
{
    const double logs = (double)(__builtin_amdgcn_logf(S) - __builtin_amdgcn_logf(A)) * 0.69314718055994531;
    return (float)((double)w * (double)t * (D * (double)(1.f / A) + (double)t * logs));
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
template <typename T, int TEAM, int HOLD, bool GRAD>
__global__ __launch_bounds__(TEAM > 64 ? TEAM : 256, TEAM > 256 ? 8 : 4) void distill_row_kernel(DistillArgs a)
{
    constexpr int ROWS = TEAM > 64 ? 1 : 4;
    extern __shared__ __attribute__((aligned(16))) char lds[];   // [ROWS][3][n_top]
    __shared__ float part[2][3 * TEAM / 64];
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
    DistillSum sum = {-INFINITY, 0.f};
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
                distill_add(sum, v, c);
            }
        for (int i = t + HOLD * TEAM; i < words; i += TEAM) {
            DistillWord<T> word;
            float v[8];
            word.load(z + head + 8 * i);
            word.numbers(v);
            distill_add(sum, v, c);
        }
        for (int i = t; i < rest; i += TEAM) {
            const float v[1] = {distill_load(z + (i < head ? i : 8 * words + i))};
            distill_add(sum, v, c);
        }
        round[2] = sum.top;
    }
    team_all<TEAM>(round, -INFINITY, part[0], JoinMax());
    if (!(round[0] > 0.f)) {   // weight 0 or no entries
        if (t == 0) a.loss[row] = 0.f;
        if (GRAD)
            for (int i = t; i < a.vocab; i += TEAM) distill_store(g + i, 0.f);
        return;
    }
    const float from = distill_from(round[2]);
    float sums[2];   // A, S
    double D;
    distill_sums<TEAM>(a, t, n, round[1], from, sums[0], D);
    sums[1] = sum.sum * distill_power(sum.top, from, c);
    team_sums<TEAM>(sums, D, part[1], part_d);
    if (t == 0) a.loss[row] = distill_loss(w, a.t, sums[0], sums[1], D);
    if constexpr (GRAD) {
        const float scale = w * a.t / sums[1];
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
        distill_places<TEAM>(a, t, n, g, 0, a.vocab, from, scale, w * a.t / sums[0]);
    }
}

// ---- few rows of many logits -----------------------------------------------------------------------------------------

// A row in `parts` pieces of whole words; its largest logits and sums go into sums [rows][parts][2], and a second launch joins them.
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

template <typename T, int TEAM>
__global__ __launch_bounds__(TEAM) void distill_part_kernel(DistillArgs a, int parts, float* sums)
{
    __shared__ float shared[2][3 * TEAM / 64];
    const int64_t row = blockIdx.x / parts;
    const int part = blockIdx.x % parts;
    if (a.weight && a.weight[row] == 0.f) return;   // (nobody reads its sums)
    const T* z = (const T*)a.logits + row * a.ld;
    const float c = a.log2_t;
    DistillSum sum = {-INFINITY, 0.f};
    distill_each<TEAM>(z, distill_piece(a.vocab, parts, part), [&](int i) {
        DistillWord<T> word;
        float v[8];
        word.load(z + i);
        word.numbers(v);
        distill_add(sum, v, c);
    }, [&](int i) {
        const float v[1] = {distill_load(z + i)};
        distill_add(sum, v, c);
    });
    float top[3] = {sum.top, -INFINITY, -INFINITY};
    team_all<TEAM>(top, -INFINITY, shared[0], JoinMax());
    float s[3] = {sum.sum * distill_power(sum.top, distill_from(top[0]), c), 0.f, 0.f};
    team_all<TEAM>(s, 0.f, shared[1], JoinSum());
    if (threadIdx.x == 0) {
        sums[2 * (row * parts + part)] = top[0];
        sums[2 * (row * parts + part) + 1] = s[0];
    }
}

template <typename T, int TEAM, bool GRAD>
__global__ __launch_bounds__(TEAM) void distill_join_kernel(DistillArgs a, int parts, const float* sums)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ float shared[2][3 * TEAM / 64];
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
    DistillSum mine = {-INFINITY, 0.f};
    if (w != 0.f) {
        distill_entries<TEAM>(a, row, t, z, n, round[0], round[1]);
        if (t < parts) mine = {sums[2 * (row * parts + t)], sums[2 * (row * parts + t) + 1]};
        round[2] = mine.top;
    }
    team_all<TEAM>(round, -INFINITY, shared[0], JoinMax());
    if (!(round[0] > 0.f)) {
        if (t == 0 && piece.lo == 0) a.loss[row] = 0.f;
        if (GRAD)
            for (int i = piece.lo + t; i < piece.hi; i += TEAM) distill_store(g + i, 0.f);
        return;
    }
    const float from = distill_from(round[2]);
    float s[2];
    double D;
    distill_sums<TEAM>(a, t, n, round[1], from, s[0], D);
    s[1] = mine.sum * distill_power(mine.top, from, c);
    team_sums<TEAM>(s, D, shared[1], shared_d);
    if (t == 0 && piece.lo == 0) a.loss[row] = distill_loss(w, a.t, s[0], s[1], D);
    if constexpr (GRAD) {
        const float scale = w * a.t / s[1];
        const bool same = (((uintptr_t)g ^ (uintptr_t)z) & 15) == 0;
        distill_each<TEAM>(z, piece, [&](int i) {
            DistillWord<T> word;
            word.load(z + i);
            distill_out(word, g + i, same, from, c, scale);
        }, [&](int i) { distill_store(g + i, distill_power(distill_load(z + i), from, c) * scale); });
        __syncthreads();
        distill_places<TEAM>(a, t, n, g, piece.lo, piece.hi, from, scale, w * a.t / s[0]);
    }
}

template <typename T, int TEAM, int HOLD>
static int launch_rows(const DistillArgs& a, hipStream_t st)
{
    constexpr int ROWS = TEAM > 64 ? 1 : 4;
    const unsigned lds = (unsigned)(ROWS * 12 * a.n_top);
    const dim3 grid((unsigned)((a.rows + ROWS - 1) / ROWS)), threads(TEAM > 64 ? TEAM : 256);
    if (a.grad) hipLaunchKernelGGL((distill_row_kernel<T, TEAM, HOLD, true>), grid, threads, lds, st, a);
    else hipLaunchKernelGGL((distill_row_kernel<T, TEAM, HOLD, false>), grid, threads, lds, st, a);
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

template <typename T>
static int launch_distill(const DistillArgs& a, float* sums, hipStream_t st)
{
    // in place the second launch's work-groups would read the student's logits at entries that another piece's have replaced: rows stay whole
    const int parts = a.grad == a.logits ? 1 : gvq_distill_parts(a.rows, a.vocab);
    if (parts > 1) {
        const unsigned lds = (unsigned)(12 * a.n_top);
        const dim3 grid((unsigned)(a.rows * parts)), threads(DISTILL_TEAM);
        hipLaunchKernelGGL((distill_part_kernel<T, DISTILL_TEAM>), grid, threads, 0, st, a, parts, sums);
        GVQ_HIP(hipGetLastError());
        if (a.grad) hipLaunchKernelGGL((distill_join_kernel<T, DISTILL_TEAM, true>), grid, threads, lds, st, a, parts, sums);
        else hipLaunchKernelGGL((distill_join_kernel<T, DISTILL_TEAM, false>), dim3((unsigned)a.rows), threads, lds, st, a, parts, sums);
        GVQ_HIP(hipGetLastError());
        return GVQ_OK;
    }
    // by a row's bytes.  A wave, four and sixteen of them (us with the gradient): 16384 x 1000 bf16 23, 37; 8192 x 2048 bf16 19, 23; 8192 x 2048 fp32
    // 36, 30; 4096 x 8192 bf16 35, 28, 48; 8192 x 4096 fp32 77, 54, 81; 4096 x 16384 bf16 -, 50, 60; 4096 x 32000 bf16 -, 112, 107; 64 x 32000 -, 13,
    // 9.2.  Many entries would take a wave's row too much LDS.
    const int64_t bytes = (int64_t)a.vocab * (int64_t)sizeof(T);
    if (bytes <= 4096 && a.n_top <= 256) return launch_rows<T, 64, sizeof(T) == 2 ? 4 : 2>(a, st);
    if (bytes <= (a.rows >= 1024 ? 32768 : 16384)) return launch_rows<T, 256, 4>(a, st);
    return launch_rows<T, 1024, sizeof(T) == 2 ? 6 : 3>(a, st);
}

int gvq_launch_distill(const DistillArgs& a, gvq_dtype_t dtype, void* workspace, hipStream_t st)
{
    return dtype == GVQ_BF16 ? launch_distill<unsigned short>(a, (float*)workspace, st) : launch_distill<float>(a, (float*)workspace, st);
}
