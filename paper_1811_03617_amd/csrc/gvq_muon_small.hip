// Newton-Schulz for matrices with at most 64 rows or columns (X has m <= 64 rows here, the transpose if need be): what such a
// matrix costs elsewhere is launches, 17 and more of 3.5 us each.
//
// Up to MS_ONE columns the whole of X stays in the LDS of one work-group, momentum, norm, steps and result in one launch.  Wider
// ones are cut into up to MS_GROUPS runs of columns, a launch per step: every work-group adds up the partial Gram matrices of the
// launch before, makes the polynomial for itself (a 64 x 64 product), takes its columns through the step and leaves its part of
// the next Gram matrix.  Same numbers and products as in gvq_muon.hip: two f16 terms, three products, fp32 sums.
// Bound: latency, from barrier to barrier, and at many columns the LDS, whose fragments every tile reads for itself, on the 32 compute units that
// have columns.  64 x 27 16 us, 64 x 384 59, 64 x 4096 87, 64 x 25088 208 (one launch per product: 68, 99, 129, 251).
#include "gvq_muon_device.h"

#define MS_THREADS 512
#define MS_M 64
#define MS_LDM (MS_M + 8)      // padded rows: 16 rows' 16-byte words in different banks (an odd number of them per row)
#define MS_ONE 384             // columns of the one-launch kernel
#define MS_SLAB 384            // most columns a work-group has in LDS at a time otherwise
#define MS_GROUPS 32

struct MuonSmallArgs {
    MuonPrep p;
    int m, n;
    int steps;
    const double* sums;            // of squares, [matrix][parts]: slabs only
    NsFactors* factors;            // slabs: this step's of the first matrix (FIRST: all of them), GVQ_MAX_STEPS further for each next one
    _Float16* x;                   // slabs: planes of the first matrix, `per` bytes further for each next one
    int64_t per, plane, ldn;
    float *from, *to;              // slabs: partial Gram matrices, [matrix][group][64][64]
    int run, slab;                 // slabs: columns of a work-group, and at a time; multiples of 32
    void* out;
    int64_t ld_out, stride_out;
    int update;
    float keep, rate;
};

// Two planes in LDS, `plane` numbers apart, rows of ld.
struct Slab {
    _Float16* hi;
    int plane, ld;
};

__device__ __forceinline__ void frag_rows(const Slab& s, int row, int k, h8& hi, h8& lo)   // 16 rows from `row`, 32 numbers from k
{
    const int lane = threadIdx.x & 63;
    const _Float16* p = s.hi + (row + (lane & 15)) * s.ld + k + 8 * (lane >> 4);
    hi = *(const h8*)p;
    lo = *(const h8*)(p + s.plane);
}
__device__ __forceinline__ void frag_cols(const Slab& s, int k, int col, h8& hi, h8& lo)   // 32 rows from k, 16 columns from `col`
{
    const int lane = threadIdx.x & 63;
    const _Float16* p = s.hi + (k + 8 * (lane >> 4) + ((lane & 15) >> 2)) * s.ld + col + 4 * (lane & 3);
    const h4 a = turned4(p), b = turned4(p + 4 * s.ld), c = turned4(p + s.plane), d = turned4(p + s.plane + 4 * s.ld);
    hi = h8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    lo = h8{c[0], c[1], c[2], c[3], d[0], d[1], d[2], d[3]};
}
// Four neighbouring numbers of a row into the planes.
__device__ __forceinline__ void put4(const Slab& s, int row, int col, f4 v)
{
    h4 hi, lo;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        _Float16 h, l;
        split_f16(v[i], h, l);
        hi[i] = h; lo[i] = l;
    }
    *(h4*)(s.hi + row * s.ld + col) = hi;
    *(h4*)(s.hi + s.plane + row * s.ld + col) = lo;
}
__device__ __forceinline__ f4 get4(const Slab& s, int row, int col)
{
    const h4 hi = *(const h4*)(s.hi + row * s.ld + col), lo = *(const h4*)(s.hi + s.plane + row * s.ld + col);
    return f4{(float)hi[0] + (float)lo[0], (float)hi[1] + (float)lo[1], (float)hi[2] + (float)lo[2], (float)hi[3] + (float)lo[3]};
}

// Sums of the three products of two terms each, the small ones apart: a product's latency is not another's.
struct Sum3 {
    f4 big = {0.f, 0.f, 0.f, 0.f}, small = {0.f, 0.f, 0.f, 0.f};
    __device__ __forceinline__ void add(const h8& ahi, const h8& alo, const h8& bhi, const h8& blo)
    {
        small = __builtin_amdgcn_mfma_f32_16x16x32_f16(blo, ahi, small, 0, 0, 0);
        big = __builtin_amdgcn_mfma_f32_16x16x32_f16(bhi, ahi, big, 0, 0, 0);
        small = __builtin_amdgcn_mfma_f32_16x16x32_f16(bhi, alo, small, 0, 0, 0);
    }
    __device__ __forceinline__ f4 value() const { return big + small; }
};

// Tile t of the 4 x 4 of a 64 x 64 matrix: wave w has the columns 16 (w % 4) and, for t = 0 and 1, the rows 16 (w / 4) and 32 more.
__device__ __forceinline__ void gram_add(const Slab& X, int cols, int m, Sum3 (&acc)[2])
{
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), r = 16 * (wave >> 2), c = 16 * (wave & 3);
    if (r >= m || c >= m) return;
    const bool two = r + 32 < m;
    for (int k = 0; k < cols; k += 32) {
        h8 bh, bl, ah, al, ch, cl;
        frag_rows(X, c, k, bh, bl);
        frag_rows(X, r, k, ah, al);
        if (two) frag_rows(X, r + 32, k, ch, cl);
        acc[0].add(ah, al, bh, bl);
        if (two) acc[1].add(ch, cl, bh, bl);
    }
}

// P = b A + c A A from the planes of A.
__device__ __forceinline__ void poly(const Slab& A, const Slab& P, int m, const NsFactors& f)
{
    const int lane = threadIdx.x & 63;
    Sum3 acc[2];
    gram_add(A, m, m, acc);
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), r = 16 * (wave >> 2), q = 16 * (wave & 3);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        if (r + 32 * t >= m || q >= m) continue;
        const int row = r + 32 * t + (lane & 15), col = q + 4 * (lane >> 4);
        put4(P, row, col, f.pa * get4(A, row, col) + f.pc * acc[t].value());
    }
}

// The polynomial as a wave keeps it: all of it.
struct PolyFrags {
    h8 hi[2][4], lo[2][4];
    __device__ __forceinline__ void load(const Slab& P, int m)
    {
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (16 * r < m && 32 * k < m) frag_rows(P, 16 * r, 32 * k, hi[k][r], lo[k][r]);
    }
};

// a X + P X for the column tiles wave, wave + 8, .. of a slab of `cols` columns: TILES of them at most, four row tiles each.
template <int TILES>
__device__ __forceinline__ void step(const Slab& X, const PolyFrags& P, int cols, int m, const NsFactors& f, f4 (&v)[TILES][4])
{
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63;
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
        const int c = 16 * (wave + 8 * t);
        if (c >= cols) continue;
        h8 bh[2], bl[2];
        frag_cols(X, 0, c, bh[0], bl[0]);
        if (m > 32) frag_cols(X, 32, c, bh[1], bl[1]);
        Sum3 acc[4];
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (16 * r < m && 32 * k < m) acc[r].add(P.hi[k][r], P.lo[k][r], bh[k], bl[k]);
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (16 * r < m) v[t][r] = f.sa * get4(X, 16 * r + (lane & 15), c + 4 * (lane >> 4)) + f.ss * acc[r].value();
    }
}

// Every number of R x C, rows over the waves and columns over the lanes: `load` for eight of them first (at places inside), then
// `use`.  One at a time each would wait for memory: 1 us a number.
template <typename L, typename U>
__device__ __forceinline__ void for_numbers(int R, int C, L load, U use)
{
    const int lane = threadIdx.x & 63;
    int r = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), c = 0;
    while (r < R) {
        int row[8], col[8];
        decltype(load(0, 0)) v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            row[i] = r;
            col[i] = c + lane;
            c += 64;
            if (c >= C) { c = 0; r += MS_THREADS / 64; }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = load(row[i] < R ? row[i] : R - 1, col[i] < C ? col[i] : C - 1);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (row[i] < R && col[i] < C) use(row[i], col[i], v[i]);
    }
}

struct GradAndMomentum {
    float g, m;
};
template <typename G>
__device__ __forceinline__ GradAndMomentum both_at(const MuonPrep& a, const G* g, int64_t r, int64_t c)
{
    return {number_at(g, r * a.ld_grad + c), a.momentum ? a.momentum[r * a.ld_momentum + c] : 0.f};
}

// The result, `at(r, c)` being its number of row r and column c (in natural order).
template <typename OUT, typename F>
__device__ __forceinline__ void results(const MuonSmallArgs& a, OUT* out, int R, int C, F at)
{
    for_numbers(R, C, [&](int r, int c) { return a.update ? number_at((const OUT*)out, r * a.ld_out + c) : 0.f; },
                [&](int r, int c, float old) {
                    const float x = at(r, c), v = a.update ? a.keep * old - a.rate * x : x;
                    if constexpr (sizeof(OUT) == 2) out[r * a.ld_out + c] = (OUT)f32_to_bf16_rne(v);
                    else out[r * a.ld_out + c] = v;
                });
}

// ---- the whole matrix in one work-group -------------------------------------------------------------------------------

// LDS: the planes of X ([2][64][ld], ld = n rounded up to 32 plus 8), which are one array of fp32 numbers of the same rows before
// and after the steps; those of A and P.  WIDTH: the most columns.
template <typename G, typename OUT, int WIDTH>
__global__ __launch_bounds__(MS_THREADS) void muon_one_kernel(MuonSmallArgs a, MuonCoef coef)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ double red[MS_THREADS / 64];
    __shared__ NsFactors factors[GVQ_MAX_STEPS];
    const int cols = (a.n + 31) & ~31, ld = cols + 8, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const Slab X = {(_Float16*)lds, MS_M * ld, ld};
    const Slab A = {(_Float16*)lds + 2 * MS_M * ld, MS_M * MS_LDM, MS_LDM}, P = {A.hi + 2 * MS_M * MS_LDM, MS_M * MS_LDM, MS_LDM};
    float* F = (float*)lds;
    const G* g = (const G*)a.p.grad + blockIdx.x * a.p.stride_grad;
    double s = 0;
    const int R = (int)a.p.rows, C = (int)a.p.cols;
    for_numbers(R, C, [&](int r, int c) { return both_at<G>(a.p, g, r, c); },
                [&](int r, int c, GradAndMomentum v) {
                    float u = v.g;
                    if (a.p.momentum) {
                        const float m = a.p.beta * v.m + v.g;
                        a.p.momentum[r * a.p.ld_momentum + c] = m;
                        u = a.p.nesterov ? v.g + a.p.beta * m : m;
                    }
                    s += (double)u * u;
                    F[a.p.turn ? c * ld + r : r * ld + c] = u;
                });
    double norm;
    const double inv = scale_to_x(group_sum<MS_THREADS>(s, red), a.p.eps, norm);   // (its barriers are behind all of F)
    leave_factors(coef, norm, factors);
    // wave w has the rows w, w + 8, ..
    constexpr int ACROSS = WIDTH / 64;
    float v[MS_M / 8][ACROSS];
#pragma unroll
    for (int y = 0; y < MS_M / 8; ++y)
#pragma unroll
        for (int x = 0; x < ACROSS; ++x) {
            const int r = wave + 8 * y, c = lane + 64 * x;
            v[y][x] = r < a.m && c < a.n ? (float)((double)F[r * ld + c] * inv) : 0.f;
        }
    __syncthreads();
#pragma unroll
    for (int y = 0; y < MS_M / 8; ++y)
#pragma unroll
        for (int x = 0; x < ACROSS; ++x) {
            const int r = wave + 8 * y, c = lane + 64 * x;
            if (c < cols) {
                _Float16 h, l;
                split_f16(v[y][x], h, l);
                X.hi[r * ld + c] = h;
                X.hi[X.plane + r * ld + c] = l;
            }
        }
    const int m = (a.m + 31) & ~31;   // rows and columns up to there are zeros
    for (int t = 0; t < a.steps; ++t) {
        __syncthreads();
        Sum3 acc[2];
        gram_add(X, cols, m, acc);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int r = 16 * (wave >> 2) + 32 * i, c = 16 * (wave & 3);
            if (r < m && c < m) put4(A, r + (lane & 15), c + 4 * (lane >> 4), acc[i].value() * NS_GRAM_SCALE);
        }
        const NsFactors f = factors[t];
        __syncthreads();
        poly(A, P, m, f);
        __syncthreads();
        constexpr int TILES = (WIDTH + 127) / 128;
        f4 x[TILES][4];
        PolyFrags frags;
        frags.load(P, m);
        step<TILES>(X, frags, cols, m, f, x);
        __syncthreads();
        const bool last = t + 1 == a.steps;
#pragma unroll
        for (int i = 0; i < TILES; ++i) {
            const int c = 16 * (wave + 8 * i) + 4 * (lane >> 4);
            if (c >= cols) continue;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 16 * r + (lane & 15);
                if (16 * r >= m) continue;
                if (last) *(f4*)(F + row * ld + c) = x[i][r] * f.out;
                else put4(X, row, c, x[i][r]);
            }
        }
    }
    __syncthreads();
    results(a, (OUT*)a.out + blockIdx.x * a.stride_out, R, C, [&](int r, int c) { return F[a.p.turn ? c * ld + r : r * ld + c]; });
}

// ---- columns over several work-groups -----------------------------------------------------------------------------------

// The words of a slab's planes, `load` for all of a thread's first; `in`: in the matrix.
template <typename L, typename U>
__device__ __forceinline__ void slab_words(const MuonSmallArgs& a, int cols, L load, U use)
{
    constexpr int PER_ROW = MS_SLAB / 8, N = 2 * MS_M * PER_ROW / MS_THREADS;
    u4 v[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int e = threadIdx.x + i * MS_THREADS, pl = e / (MS_M * PER_ROW), r = e / PER_ROW % MS_M, c = e % PER_ROW * 8;
        v[i] = load(pl, r, c, r < a.m && c < cols);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int e = threadIdx.x + i * MS_THREADS, pl = e / (MS_M * PER_ROW), r = e / PER_ROW % MS_M, c = e % PER_ROW * 8;
        use(pl, r, c, r < a.m && c < cols, v[i]);
    }
}

struct MuonNone {};

// FIRST: U / (|U| + eps) into the planes and its part of A.  Otherwise a step, the result if LAST.
// LDS: the planes of a slab of MS_SLAB columns (fp32 numbers of the same rows on the way out), those of A and P.
template <typename G, typename OUT, bool FIRST, bool LAST>
__global__ __launch_bounds__(MS_THREADS) void muon_slab_kernel(MuonSmallArgs a, typename std::conditional<FIRST, MuonCoef, MuonNone>::type coef)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ double red[MS_THREADS / 64];
    constexpr int LD = MS_SLAB + 8, TILES = MS_SLAB / 128;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const Slab X = {(_Float16*)lds, MS_M * LD, LD};
    const Slab A = {(_Float16*)lds + 2 * MS_M * LD, MS_M * MS_LDM, MS_LDM}, P = {A.hi + 2 * MS_M * MS_LDM, MS_M * MS_LDM, MS_LDM};
    float* F = (float*)lds;
    const int m = (a.m + 31) & ~31, groups = gridDim.x;
    const G* g = (const G*)a.p.grad + blockIdx.y * a.p.stride_grad;
    OUT* out = (OUT*)a.out + blockIdx.y * a.stride_out;
    _Float16* gx = (_Float16*)((char*)a.x + blockIdx.y * a.per);
    double inv = 0;
    NsFactors* fs = a.factors + blockIdx.y * GVQ_MAX_STEPS;
    NsFactors f{};
    if (!FIRST) f = *fs;
    if constexpr (FIRST) {
        double s = 0, norm;
        for (int i = threadIdx.x; i < a.p.parts; i += MS_THREADS) s += a.sums[blockIdx.y * a.p.parts + i];
        inv = scale_to_x(group_sum<MS_THREADS>(s, red), a.p.eps, norm);
        if (blockIdx.x == 0) leave_factors(coef, norm, fs);
    } else {
        const float* p = a.from + (int64_t)blockIdx.y * groups * MS_M * MS_M;
        f4 v[2] = {f4{0.f, 0.f, 0.f, 0.f}, f4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll 16
        for (int q = 0; q < groups; ++q)
#pragma unroll
            for (int i = 0; i < 2; ++i) v[i] += *(const f4*)(p + q * MS_M * MS_M + 4 * (threadIdx.x + i * MS_THREADS));
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int e = 4 * (threadIdx.x + i * MS_THREADS);
            put4(A, e / MS_M, e % MS_M, v[i] * NS_GRAM_SCALE);
        }
        __syncthreads();
        poly(A, P, m, f);
    }
    Sum3 acc[2];
    PolyFrags frags;
    if (!FIRST) {
        __syncthreads();
        frags.load(P, m);
    }
    const int begin = blockIdx.x * a.run, end = begin + a.run < a.n ? begin + a.run : a.n;
    for (int c0 = begin; c0 < end; c0 += a.slab) {
        const int w = end - c0 < a.slab ? end - c0 : a.slab, cols = (w + 31) & ~31;
        __syncthreads();
        if (FIRST) {
            // in natural order, so that neighbouring lanes read neighbouring numbers; zeros behind the matrix
            const int R = a.p.turn ? w : a.m, C = a.p.turn ? a.m : w;
            for (int i = threadIdx.x; i < MS_M * (LD / 8); i += MS_THREADS) {
                *(u4*)(X.hi + 8 * i) = u4{0, 0, 0, 0};
                *(u4*)(X.hi + X.plane + 8 * i) = u4{0, 0, 0, 0};
            }
            __syncthreads();
            for_numbers(R, C, [&](int r, int c) { return both_at<G>(a.p, g, a.p.turn ? c0 + r : r, a.p.turn ? c : c0 + c); },
                        [&](int r, int c, GradAndMomentum b) {
                            const float u = a.p.momentum ? a.p.nesterov ? b.g + a.p.beta * b.m : b.m : b.g;
                            _Float16 h, l;
                            split_f16((float)((double)u * inv), h, l);
                            const int at = a.p.turn ? c * LD + r : r * LD + c;
                            X.hi[at] = h;
                            X.hi[X.plane + at] = l;
                        });
        } else {
            slab_words(a, cols, [&](int pl, int r, int c, bool in) { return in ? *(const u4*)(gx + pl * a.plane + r * a.ldn + c0 + c) : u4{0, 0, 0, 0}; },
                       [&](int pl, int r, int c, bool, u4 v) { *(u4*)(X.hi + pl * X.plane + r * LD + c) = v; });
        }
        __syncthreads();
        if (!FIRST) {
            f4 x[TILES][4];
            step<TILES>(X, frags, cols, m, f, x);
            __syncthreads();
#pragma unroll
            for (int i = 0; i < TILES; ++i) {
                const int c = 16 * (wave + 8 * i) + 4 * (lane >> 4);
                if (c >= cols) continue;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int row = 16 * r + (lane & 15);
                    if (16 * r >= m) continue;
                    if (LAST) *(f4*)(F + row * LD + c) = x[i][r] * f.out;
                    else put4(X, row, c, x[i][r]);
                }
            }
            __syncthreads();
        }
        if (LAST) {
            results(a, out + (a.p.turn ? c0 * a.ld_out : c0), a.p.turn ? w : a.m, a.p.turn ? a.m : w,
                    [&](int r, int c) { return F[a.p.turn ? c * LD + r : r * LD + c]; });
        } else {
            slab_words(a, cols, [&](int pl, int r, int c, bool) { return *(const u4*)(X.hi + pl * X.plane + r * LD + c); },
                       [&](int pl, int r, int c, bool in, u4 v) { if (in) *(u4*)(gx + pl * a.plane + r * a.ldn + c0 + c) = v; });
            gram_add(X, cols, m, acc);
        }
    }
    if (!LAST) {
        float* to = a.to + ((int64_t)blockIdx.y * groups + blockIdx.x) * MS_M * MS_M;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int r = 16 * (wave >> 2) + 32 * i + (lane & 15), c = 16 * (wave & 3) + 4 * (lane >> 4);
            *(f4*)(to + r * MS_M + c) = acc[i].value();
        }
    }
}

// ---- launchers ------------------------------------------------------------------------------------------------------------

bool gvq_muon_small_takes(const MuonMatrix& x) { return (x.rows < x.cols ? x.rows : x.cols) <= MS_M; }

// Columns of a work-group.
static int64_t small_run(int64_t n)
{
    const int64_t run = ns_padded((n + MS_GROUPS - 1) / MS_GROUPS);
    return run < 128 ? 128 : run;
}

int64_t gvq_muon_small_plan(const MuonMatrix& x, MuonSmallPlan* p)
{
    p->m = x.rows < x.cols ? x.rows : x.cols;
    p->n = x.rows < x.cols ? x.cols : x.rows;
    p->one = p->n <= MS_ONE;
    p->bytes = 256;   // (a workspace of its own, however small, from every caller)
    if (p->one) return p->bytes;
    int64_t at = 0;
    auto take = [&](int64_t bytes) { const int64_t was = at; at += (bytes + 255) / 256 * 256; return was; };
    p->ldn = ns_padded(p->n);
    p->run = small_run(p->n);
    p->groups = (p->n + p->run - 1) / p->run;
    p->per = p->m * p->ldn * 4;
    p->x = take(x.batch * p->per);
    for (int i = 0; i < 2; ++i) p->grams[i] = take(x.batch * p->groups * MS_M * MS_M * 4);
    p->parts = gvq_muon_parts(x);
    p->sums = take(x.batch * p->parts * (int64_t)sizeof(double));
    p->factors = take(x.batch * GVQ_MAX_STEPS * (int64_t)sizeof(NsFactors));
    return p->bytes = at;
}

template <typename K>
static int raise_lds(gvq_once_per_device& once, K kernel, int bytes)
{
    int dev;
    GVQ_HIP(hipGetDevice(&dev));
    return once.call(dev, [&] {
        GVQ_HIP(hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes));
        return (int)GVQ_OK;
    });
}

static constexpr int lds_of(int cols) { return 4 * MS_M * (cols + 8) + 8 * MS_M * MS_LDM; }

template <typename G, typename OUT, int WIDTH>
static int launch_one(const MuonSmallArgs& a, const MuonCoef& coef, int64_t batch, hipStream_t st)
{
    static gvq_once_per_device once;
    const int rc = raise_lds(once, muon_one_kernel<G, OUT, WIDTH>, lds_of(WIDTH));
    if (rc != GVQ_OK) return rc;
    hipLaunchKernelGGL((muon_one_kernel<G, OUT, WIDTH>), dim3((unsigned)batch), dim3(MS_THREADS), lds_of((int)ns_padded(a.n)), st, a, coef);
    GVQ_HIP(hipGetLastError());
    return GVQ_OK;
}

template <typename G, typename OUT, bool FIRST, bool LAST>
static int launch_slab(const MuonSmallArgs& a, const typename std::conditional<FIRST, MuonCoef, MuonNone>::type& coef, int64_t groups, int64_t batch,
                       hipStream_t st)
{
    static gvq_once_per_device once;
    const int rc = raise_lds(once, muon_slab_kernel<G, OUT, FIRST, LAST>, lds_of(MS_SLAB));
    if (rc != GVQ_OK) return rc;
    hipLaunchKernelGGL((muon_slab_kernel<G, OUT, FIRST, LAST>), dim3((unsigned)groups, (unsigned)batch), dim3(MS_THREADS), lds_of(MS_SLAB), st, a, coef);
    GVQ_HIP(hipGetLastError());
    return GVQ_OK;
}

template <typename G, typename OUT>
static int launch_small(const MuonArgs& m, MuonSmallArgs a, const MuonSmallPlan& p, const MuonCoef& coef, hipStream_t st)
{
    if (p.one) {
        if (a.n <= 128) return launch_one<G, OUT, 128>(a, coef, m.x.batch, st);
        return launch_one<G, OUT, MS_ONE>(a, coef, m.x.batch, st);
    }
    char* w = m.workspace;
    int rc = gvq_launch_muon_norm(m, a.p, (double*)(w + p.sums), st);
    a.sums = (const double*)(w + p.sums);
    a.x = (_Float16*)(w + p.x);
    a.per = p.per;
    a.plane = p.m * p.ldn;
    a.ldn = p.ldn;
    a.run = (int)p.run;
    a.slab = (int)ns_padded((p.run + (p.run + MS_SLAB - 1) / MS_SLAB - 1) / ((p.run + MS_SLAB - 1) / MS_SLAB));
    a.to = (float*)(w + p.grams[0]);
    a.factors = (NsFactors*)(w + p.factors);
    if (rc == GVQ_OK) rc = launch_slab<G, float, true, false>(a, coef, p.groups, m.x.batch, st);
    for (int t = 0; t < m.steps && rc == GVQ_OK; ++t) {
        a.factors = (NsFactors*)(w + p.factors) + t;
        a.from = (float*)(w + p.grams[t & 1]);
        a.to = (float*)(w + p.grams[(t + 1) & 1]);
        rc = t + 1 < m.steps ? launch_slab<float, float, false, false>(a, {}, p.groups, m.x.batch, st)
                             : launch_slab<float, OUT, false, true>(a, {}, p.groups, m.x.batch, st);
    }
    return rc;
}

int gvq_launch_muon_small(const MuonArgs& m, hipStream_t st)
{
    MuonSmallPlan p;
    gvq_muon_small_plan(m.x, &p);
    MuonSmallArgs a{};
    a.p = gvq_muon_prep(m);
    a.p.parts = p.one ? 0 : p.parts;
    a.m = (int)p.m;
    a.n = (int)p.n;
    a.steps = m.steps;
    a.out = m.out; a.ld_out = m.ld_out; a.stride_out = m.stride_out;
    a.update = m.update; a.keep = m.keep; a.rate = m.rate;
    const MuonCoef coef = gvq_muon_coef(m);
    if (m.grad_dtype == GVQ_BF16)
        return m.out_dtype == GVQ_BF16 ? launch_small<unsigned short, unsigned short>(m, a, p, coef, st) : launch_small<unsigned short, float>(m, a, p, coef, st);
    return m.out_dtype == GVQ_BF16 ? launch_small<float, unsigned short>(m, a, p, coef, st) : launch_small<float, float>(m, a, p, coef, st);
}
