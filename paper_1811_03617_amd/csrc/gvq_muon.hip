// Muon's step: momentum, Newton-Schulz orthogonalisation, decayed weight minus the step.
//
// X_0 = U / (|U|_F + eps), then X <- a X + (b A + c A A) X with A = X X^T (for a tall matrix X (b A + c A A) with A = X^T X, the
// same polynomial of the smaller Gram matrix).  Its singular values s follow s <- a s + b s^3 + c s^5, towards 1.
//
// Precision.  The steps multiply small singular values by a = 3.4 each, 485 in all, and what rounding adds to X along such a
// direction grows with them: numbers kept in bf16 end 1 to 7 % off (2-norm, planted low rank the worst), in f16 0.1 to 0.9 %.
// So X, A and the polynomial are kept as two f16 terms, 22 bits, in units chosen by the matrix's norm and the coefficients
// (gvq_muon_plan.h; an ordinary matrix: 2^-12 for X and A, 2^-10 for the polynomial), and
// every product is hi hi + hi lo + lo hi in fp32 sums: as exact as fp32 products (0.6 to 1.4 times their error), at a third of
// the f16 matrix pipe's rate, which is three times what the fp32 pipe reaches (153 TFLOP/s of library products).
//
// A step is three products: A (half of it, mirrored), b A + c A A (half of it), and a X + P X.  Bound: the matrix pipe's power where
// matrices are large (4096 x 4096 in fp32 196 + 200 + 338 us a step), launches, half-filled rounds of tiles and the bytes of X where they
// are not (5 of 512 x 4608 36 + 6 + 11 + 67, 1000 x 4096 21 + 5 + 16 + 38).
#include "gvq_muon_device.h"

#define MUON_THREADS 256

struct PrepArgs {
    MuonPrep p;
    double* sums;        // [batch][parts]
    char* x;             // planes of the first matrix, `per` bytes further for each next one
    int64_t per, plane;  // plane: numbers
    int64_t ld;
    int tx, words;       // threads side by side, as a power of two; four neighbouring numbers are aligned words
    NsFactors* factors;  // [batch][GVQ_MAX_STEPS]
};

// Four neighbouring numbers of a row a thread, 1 << tx threads side by side and rows under each other; `at(r, c)` for every such
// four.  Runs of rows and columns are handed out one after the other; 32-bit indices (a 64-bit division for each number
// took as long as its memory).
template <typename F>
__device__ __forceinline__ void for_fours(const PrepArgs& a, int cols, F at)
{
    const int across = 1 << a.tx, down = MUON_THREADS >> a.tx, rows = (int)a.p.rows;
    const int chunks = (cols + 4 * across - 1) / (4 * across), units = (rows + down - 1) / down * chunks;
    const int x = 4 * (threadIdx.x & (across - 1)), y = threadIdx.x >> a.tx;
    for (int u = blockIdx.x; u < units; u += gridDim.x) {
        const int g = u / chunks, r = g * down + y, c = (u - g * chunks) * 4 * across + x;
        if (r < rows && c < cols) at(r, c);
    }
}

// M <- beta M + G, and the sum of squares of U, in float64 (squares of fp32 numbers are exact there and do not overflow).
template <typename G>
__global__ __launch_bounds__(MUON_THREADS) void muon_norm_kernel(PrepArgs a)
{
    __shared__ double lds[MUON_THREADS / 64];
    const G* g = (const G*)a.p.grad + blockIdx.y * a.p.stride_grad;
    double s = 0;
    const int cols = (int)a.p.cols;
    for_fours(a, cols, [&](int r, int c) {
        float u[4];
        if (a.words && c + 4 <= cols) {
            four_numbers(g + r * a.p.ld_grad + c, u);
            if (a.p.momentum) {
                f4* m = (f4*)(a.p.momentum + r * a.p.ld_momentum + c);
                const f4 v = a.p.beta * *m + f4{u[0], u[1], u[2], u[3]};
                *m = v;
#pragma unroll
                for (int i = 0; i < 4; ++i) u[i] = a.p.nesterov ? u[i] + a.p.beta * v[i] : v[i];
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) u[i] = c + i < cols ? momentum_at<G>(a.p, g, r, c + i) : 0.f;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) s += (double)u[i] * u[i];
    });
    s = group_sum<MUON_THREADS>(s, lds);
    if (threadIdx.x == 0) a.sums[blockIdx.y * a.p.parts + blockIdx.x] = s;
}

// The matrix's scale; `first`, one of its work-groups, leaves its factors.
__device__ __forceinline__ double scale_of(const PrepArgs& a, const MuonCoef& coef, int matrix, bool first, double* lds)
{
    double s = 0, r;
    for (int i = threadIdx.x; i < a.p.parts; i += MUON_THREADS) s += a.sums[matrix * a.p.parts + i];
    const double inv = scale_to_x(group_sum<MUON_THREADS>(s, lds), a.p.eps, r);
    if (first) leave_factors(coef, r, a.factors + matrix * GVQ_MAX_STEPS);
    return inv;
}

// U / (|U| + eps) into the two planes of X, with zeros behind the last column.
template <typename G>
__global__ __launch_bounds__(MUON_THREADS) void muon_planes_kernel(PrepArgs a, MuonCoef coef)
{
    __shared__ double lds[MUON_THREADS / 64];
    const double inv = scale_of(a, coef, blockIdx.y, blockIdx.x == 0, lds);
    const G* g = (const G*)a.p.grad + blockIdx.y * a.p.stride_grad;
    _Float16* X = (_Float16*)(a.x + blockIdx.y * a.per);
    const int cols = (int)a.p.cols;
    for_fours(a, (int)a.ld, [&](int r, int c) {
        float u[4];
        if (a.words && c + 4 <= cols) {
            four_numbers(g + r * a.p.ld_grad + c, u);
            if (a.p.momentum) {
                const f4 m = *(const f4*)(a.p.momentum + r * a.p.ld_momentum + c);
#pragma unroll
                for (int i = 0; i < 4; ++i) u[i] = a.p.nesterov ? u[i] + a.p.beta * m[i] : m[i];
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) u[i] = c + i < cols ? direction_at<G>(a.p, g, r, c + i) : 0.f;
        }
        h4 hi, lo;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            _Float16 h, l;
            split_f16(c + i < cols ? (float)((double)u[i] * inv) : 0.f, h, l);
            hi[i] = h; lo[i] = l;
        }
        *(h4*)(X + r * a.ld + c) = hi;
        *(h4*)(X + a.plane + r * a.ld + c) = lo;
    });
}

// The same where X is the transpose: 64 x 64 numbers a work-group, through LDS.
template <typename G>
__global__ __launch_bounds__(MUON_THREADS) void muon_turn_kernel(PrepArgs a, MuonCoef coef)
{
    __shared__ double lds[MUON_THREADS / 64];
    __shared__ float tile[64 * 65];
    const double inv = scale_of(a, coef, blockIdx.z, blockIdx.x == 0 && blockIdx.y == 0, lds);
    const G* g = (const G*)a.p.grad + blockIdx.z * a.p.stride_grad;
    _Float16* X = (_Float16*)(a.x + blockIdx.z * a.per);
    const int64_t r0 = (int64_t)blockIdx.y * 64, c0 = (int64_t)blockIdx.x * 64;
    const int x = threadIdx.x & 63, y0 = threadIdx.x >> 6;
    float v[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int64_t r = r0 + y0 + 4 * i, c = c0 + x;
        const bool in = r < a.p.rows && c < a.p.cols;
        const float u = direction_at<G>(a.p, g, r < a.p.rows ? r : a.p.rows - 1, c < a.p.cols ? c : a.p.cols - 1);
        v[i] = in ? (float)((double)u * inv) : 0.f;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) tile[(y0 + 4 * i) * 65 + x] = v[i];
    __syncthreads();
#pragma unroll 4
    for (int y = y0; y < 64; y += MUON_THREADS / 64) {
        const int64_t c = c0 + y, r = r0 + x;
        if (c < a.p.cols && r < a.ld) {
            _Float16 hi, lo;
            split_f16(tile[x * 65 + y], hi, lo);
            X[c * a.ld + r] = hi;
            X[a.plane + c * a.ld + r] = lo;
        }
    }
}

// The three products of a step.
enum { NS_GRAM = 0, NS_POLY = 1, NS_STEP = 2, NS_LAST = 3 };

struct NsArgs {
    TileOperand a, b;          // of the first matrix; `per` bytes further for each next one
    int steps, nm, nn, band;   // steps of 32 numbers of the sum; tiles, and how they are swept
    int rows, cols;            // of the result
    int64_t per;
    const NsFactors* f;        // this step's of the first matrix, GVQ_MAX_STEPS further for each next one (not GRAM)
    const _Float16* old;       // POLY: A, STEP and LAST: X
    _Float16* res;             // result (not LAST)
    int64_t plane, ld;         // of old and res, in numbers
    float* parts;              // splits > 1: [matrix][split][ldp rows][ldp_cols]
    int64_t ld_part, part;     // numbers of a row, of a split
    int splits;
    void* out;                 // LAST
    int64_t ld_out, stride_out;
    int update, words;
    float keep, rate;
};

template <typename OUT>
__device__ __forceinline__ void last_store4(OUT* p, bool words, int left, int update, float keep, float rate, f4 v);
template <>
__device__ __forceinline__ void last_store4<float>(float* p, bool words, int left, int update, float keep, float rate, f4 v)
{
    if (words && left >= 4) {
        if (update) v = keep * *(const f4*)p - rate * v;
        *(f4*)p = v;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < left) p[i] = update ? keep * p[i] - rate * v[i] : v[i];
    }
}
template <>
__device__ __forceinline__ void last_store4<unsigned short>(unsigned short* p, bool words, int left, int update, float keep, float rate, f4 v)
{
    if (words && left >= 4) {
        if (update) {
            const u2 o = *(const u2*)p;
            v = keep * f4{__uint_as_float(o[0] << 16), __uint_as_float(o[0] & 0xffff0000u), __uint_as_float(o[1] << 16), __uint_as_float(o[1] & 0xffff0000u)} - rate * v;
        }
        *(u2*)p = u2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < left) p[i] = (unsigned short)f32_to_bf16_rne(update ? keep * bf16_to_f32(p[i]) - rate * v[i] : v[i]);
    }
}

// What becomes of four neighbouring sums of row r from column c on (FLIP: of four rows from r on in column c).  a X is added here and
// not as a I to the polynomial, which would save reading X a second time: in the product it would be the largest term by far of a
// sum that is rounded every 32 numbers (1024 x 1024 of planted low rank: 2.5e-5 off instead of 1.1e-5).
template <int KIND, bool FLIP>
__device__ __forceinline__ f4 ns_value4(const NsArgs& a, const NsFactors& f, const _Float16* old, int r, int c, f4 v)
{
    if (KIND == NS_GRAM) return v * NS_GRAM_SCALE;
    f4 o;
    if (!FLIP) {
        const h4 hi = *(const h4*)(old + r * a.ld + c), lo = *(const h4*)(old + a.plane + r * a.ld + c);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = (float)hi[i] + (float)lo[i];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = r + i < a.rows ? (float)old[(r + i) * a.ld + c] + (float)old[a.plane + (r + i) * a.ld + c] : 0.f;
    }
    return KIND == NS_POLY ? f.pa * o + f.pc * v : f.sa * o + f.ss * v;
}
template <int KIND>
__device__ __forceinline__ NsFactors ns_factors_of(const NsArgs& a, int matrix)
{
    if (KIND == NS_GRAM) return NsFactors{};
    return a.f[matrix * GVQ_MAX_STEPS];
}

// Upper triangle of tiles, column by column: column tn holds the tiles (0 .. tn, tn), tn (tn + 1) / 2 of them before it.
__device__ __forceinline__ void triangle_at(int t, int& tm, int& tn)
{
    tn = (int)((sqrtf(8.f * (float)t + 1.f) - 1.f) * 0.5f);
    while (tn * (tn + 1) / 2 > t) --tn;
    while ((tn + 1) * (tn + 2) / 2 <= t) ++tn;
    tm = t - tn * (tn + 1) / 2;
}

// LDS of a wave that hands its tile out through it (one plane, rows padded by 8 numbers), and of a work-group.
template <typename T>
__host__ __device__ constexpr int ns_wave_lds()
{
    const int R = T::BM / T::WM, C = T::BN / T::WN;
    return 2 * (R * (C + 8) > C * (R + 8) ? R * (C + 8) : C * (R + 8));
}
template <typename T>
constexpr int ns_lds()
{
    static_assert(ns_wave_lds<T>() * T::WAVES <= 160 * 1024 && ns_wave_lds<T>() % 16 == 0, "LDS of a compute unit");
    return T::LDS > ns_wave_lds<T>() * T::WAVES ? T::LDS : ns_wave_lds<T>() * T::WAVES;
}

// KIND: which product; GRAM and POLY compute the tiles on and above the diagonal and mirror them.  With SPLIT a work-group
// leaves its part of the sum for ns_join_kernel.
template <typename T, int KIND, typename OUT, bool SPLIT>
__global__ __launch_bounds__(T::THREADS) void ns_tile_kernel(NsArgs a)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    constexpr bool SYM = KIND == NS_GRAM || KIND == NS_POLY;
    const int tiles = SYM ? a.nm * (a.nm + 1) / 2 : a.nm * a.nn;
    int tm, tn, split = 0, step0 = 0, steps = a.steps;
    if (SPLIT) {
        // the tiles of one part side by side on one XCD: they share its rows' bytes
        const int t = tile_of_block(blockIdx.x, tiles * a.splits);
        split = t / tiles;
        step0 = (int)((int64_t)a.steps * split / a.splits);
        steps = (int)((int64_t)a.steps * (split + 1) / a.splits) - step0;
        if (SYM) triangle_at(t - split * tiles, tm, tn);
        else tile_at(t - split * tiles, a.nm, a.nn, a.band, tm, tn);
    } else if (SYM) {
        triangle_at(tile_of_block(blockIdx.x, tiles), tm, tn);
    } else {
        tile_at(tile_of_block(blockIdx.x, tiles), a.nm, a.nn, a.band, tm, tn);
    }
    const int64_t off = blockIdx.y * a.per;
    const NsFactors f = SPLIT ? NsFactors{} : ns_factors_of<KIND>(a, blockIdx.y);   // (read here, they are there when the sums are)
    TileOperand A = a.a, B = a.b;
    A.p += off;
    B.p += off;
    f4 acc[T::MI][T::NI];
#pragma unroll
    for (int mi = 0; mi < T::MI; ++mi)
#pragma unroll
        for (int ni = 0; ni < T::NI; ++ni) acc[mi][ni] = f4{0.f, 0.f, 0.f, 0.f};
    tile_product<T>(A, B, tm * T::BM, tn * T::BN, step0, steps, lds, acc);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    constexpr int R = T::BM / T::WM, C = T::BN / T::WN;   // of a wave
    const int rw = tm * T::BM + wave / T::WN * R, cw = tn * T::BN + wave % T::WN * C;
    if (SPLIT) {
        float* p = a.parts + ((int64_t)blockIdx.y * a.splits + split) * a.part;
#pragma unroll
        for (int mi = 0; mi < T::MI; ++mi)
#pragma unroll
            for (int ni = 0; ni < T::NI; ++ni)
                *(f4*)(p + (rw + 16 * mi + (lane & 15)) * a.ld_part + cw + 16 * ni + 4 * (lane >> 4)) = acc[mi][ni];
        return;
    }
    const _Float16* old = (const _Float16*)((const char*)a.old + off);
    if constexpr (KIND == NS_LAST) {
        OUT* out = (OUT*)a.out + blockIdx.y * a.stride_out;
#pragma unroll
        for (int mi = 0; mi < T::MI; ++mi)
#pragma unroll
            for (int ni = 0; ni < T::NI; ++ni) {
                const int r = rw + 16 * mi + (T::FLIP ? 4 * (lane >> 4) : lane & 15), c = cw + 16 * ni + (T::FLIP ? lane & 15 : 4 * (lane >> 4));
                if (r >= a.rows || c >= a.cols) continue;
                const f4 v = ns_value4<KIND, T::FLIP>(a, f, old, r, c, acc[mi][ni]) * f.out;
                OUT* to = T::FLIP ? out + (int64_t)c * a.ld_out + r : out + (int64_t)r * a.ld_out + c;
                last_store4<OUT>(to, a.words != 0, T::FLIP ? a.rows - r : a.cols - c, a.update, a.keep, a.rate, v);
            }
    } else {
        // Into the planes, and for a tile above the diagonal into its mirror image: through the wave's share of LDS, so that rows
        // leave in 16-byte words side by side.  Each wave reads what it wrote itself; only the last products' reads of the
        // others have to be over first.
        _Float16* res = (_Float16*)((char*)a.res + off);
        constexpr int NP = C + 8, TP = R + 8;   // padded rows: neighbours in different banks
        _Float16* w = (_Float16*)(lds + wave * ns_wave_lds<T>());
#pragma unroll
        for (int mi = 0; mi < T::MI; ++mi)
#pragma unroll
            for (int ni = 0; ni < T::NI; ++ni) {
                const int r = rw + 16 * mi + (lane & 15), c = cw + 16 * ni + 4 * (lane >> 4);
                f4 v = {0.f, 0.f, 0.f, 0.f};
                if (r < a.rows && c < a.ld) v = ns_value4<KIND, false>(a, f, old, r, c, acc[mi][ni]);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (c + i >= a.cols) v[i] = 0.f;
                acc[mi][ni] = v;
            }
        __syncthreads();
#pragma unroll 1
        for (int pl = 0; pl < 2; ++pl) {   // the first term, then what is left of each number
#pragma unroll
            for (int mi = 0; mi < T::MI; ++mi)
#pragma unroll
                for (int ni = 0; ni < T::NI; ++ni) {
                    h4 q;
#pragma unroll
                    for (int i = 0; i < 4; ++i) q[i] = (_Float16)acc[mi][ni][i];
                    *(h4*)(w + (16 * mi + (lane & 15)) * NP + 16 * ni + 4 * (lane >> 4)) = q;
                }
            wave_lds_sync();
            for (int i = lane; i < R * (C / 8); i += 64) {
                const int r = i / (C / 8), c = i % (C / 8) * 8;
                if (rw + r < a.rows && cw + c < a.ld) *(u4*)(res + (rw + r) * a.ld + cw + c) = *(const u4*)(w + r * NP + c);
            }
            wave_lds_sync();
            if (SYM && tm != tn) {
#pragma unroll
                for (int mi = 0; mi < T::MI; ++mi)
#pragma unroll
                    for (int ni = 0; ni < T::NI; ++ni)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            w[(16 * ni + 4 * (lane >> 4) + i) * TP + 16 * mi + (lane & 15)] = (_Float16)acc[mi][ni][i];
                wave_lds_sync();
                for (int i = lane; i < C * (R / 8); i += 64) {
                    const int c = i / (R / 8), r = i % (R / 8) * 8;
                    // (a tile left of the last tile column has whole rows)
                    if (cw + c < a.cols) *(u4*)(res + (cw + c) * a.ld + rw + r) = *(const u4*)(w + c * TP + r);
                }
                wave_lds_sync();
            }
#pragma unroll
            for (int mi = 0; mi < T::MI; ++mi)
#pragma unroll
                for (int ni = 0; ni < T::NI; ++ni)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[mi][ni][i] -= (float)(_Float16)acc[mi][ni][i];
            res += a.plane;
        }
    }
}

// The parts of a sum added up in their order, and what the product's own kernel does with a sum otherwise: 32 x 32 results a
// work-group, on and above the diagonal where the result is symmetric.  TURN: LAST writes the transpose.
template <int KIND, typename OUT, bool TURN>
__global__ __launch_bounds__(256) void ns_join_kernel(NsArgs a)
{
    constexpr bool SYM = KIND == NS_GRAM || KIND == NS_POLY;
    __shared__ __attribute__((aligned(16))) float tile[32 * 36];
    int tm, tn;
    if (SYM) triangle_at(blockIdx.x, tm, tn);
    else { tm = blockIdx.x / a.nn; tn = blockIdx.x - tm * a.nn; }
    const int64_t off = blockIdx.y * a.per;
    const int y = threadIdx.x >> 3, x = 4 * (threadIdx.x & 7), r = tm * 32 + y, c = tn * 32 + x;
    const NsFactors f = ns_factors_of<KIND>(a, blockIdx.y);
    const float* p = a.parts + (int64_t)blockIdx.y * a.splits * a.part + r * a.ld_part + c;
    f4 v = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < a.splits; ++s) v += *(const f4*)(p + s * a.part);
    const _Float16* old = (const _Float16*)((const char*)a.old + off);
    const bool in = r < a.rows && c < a.ld;
    if (in) v = ns_value4<KIND, false>(a, f, old, r, c, v);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (!in || c + i >= a.cols) v[i] = 0.f;
    if (KIND == NS_LAST) v *= f.out;
    if (KIND == NS_LAST && !TURN) {
        if (in && c < a.cols)
            last_store4<OUT>((OUT*)a.out + blockIdx.y * a.stride_out + (int64_t)r * a.ld_out + c, a.words != 0, a.cols - c, a.update, a.keep, a.rate, v);
        return;
    }
    _Float16* res = (_Float16*)((char*)a.res + off);
    auto put = [&](int64_t at, f4 v) {
        h4 hi, lo;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            _Float16 h, l;
            split_f16(v[i], h, l);
            hi[i] = h; lo[i] = l;
        }
        *(h4*)(res + at) = hi;
        *(h4*)(res + a.plane + at) = lo;
    };
    if (KIND != NS_LAST && in) put(r * a.ld + c, v);
    if ((SYM && tm != tn) || KIND == NS_LAST) {
        // the other way round: row c + .. of four neighbouring r
#pragma unroll
        for (int i = 0; i < 4; ++i) tile[(x + i) * 36 + y] = v[i];
        __syncthreads();
        const int c2 = tn * 32 + y, r2 = tm * 32 + x;
        const f4 w = *(const f4*)(tile + y * 36 + x);
        if (KIND == NS_LAST) {
            if (c2 < a.cols && r2 < a.rows)
                last_store4<OUT>((OUT*)a.out + blockIdx.y * a.stride_out + (int64_t)c2 * a.ld_out + r2, a.words != 0, a.rows - r2, a.update, a.keep, a.rate, w);
        } else if (c2 < a.cols) {
            put(c2 * a.ld + r2, w);
        }
    }
}

int gvq_muon_parts(const MuonMatrix& x)
{
    const int64_t n = x.rows * x.cols, parts = (n + 16 * MUON_THREADS - 1) / (16 * MUON_THREADS);
    return (int)(parts < 1 ? 1 : parts > 1024 ? 1024 : parts);
}

MuonPrep gvq_muon_prep(const MuonArgs& m)
{
    MuonPrep p{};
    p.grad = m.grad; p.ld_grad = m.ld_grad; p.stride_grad = m.stride_grad;
    p.momentum = m.momentum; p.ld_momentum = m.ld_momentum;
    p.beta = m.beta; p.nesterov = m.nesterov;
    p.rows = m.x.rows; p.cols = m.x.cols;
    p.parts = gvq_muon_parts(m.x);
    p.eps = m.eps;
    p.turn = m.x.rows > m.x.cols;
    return p;
}

MuonCoef gvq_muon_coef(const MuonArgs& m)
{
    static const double standard[3] = {3.4445, -4.7750, 2.0315};
    MuonCoef c{};
    c.steps = m.steps;
    for (int t = 0; t < m.steps; ++t)
        for (int i = 0; i < 3; ++i) c.v[t][i] = (float)(m.coef ? m.coef[3 * t + i] : standard[i]);
    ns_factors(c.v[0], c.steps, 1.0, c.whole);
    return c;
}

static PrepArgs prep_args(const MuonArgs& m)
{
    PrepArgs q{};
    q.p = gvq_muon_prep(m);
    q.tx = 2;
    while (q.tx < 8 && (4 << q.tx) < m.x.cols) ++q.tx;
    const uintptr_t es = m.grad_dtype == GVQ_BF16 ? 2 : 4;
    q.words = ((((uintptr_t)m.grad | (uintptr_t)m.ld_grad * es | (uintptr_t)m.stride_grad * es) & (4 * es - 1)) |
               (((uintptr_t)m.momentum | (uintptr_t)m.ld_momentum * 4) & 15)) == 0;
    return q;
}

int gvq_launch_muon_norm(const MuonArgs& m, const MuonPrep& p, double* sums, hipStream_t st)
{
    PrepArgs q = prep_args(m);
    q.p = p;
    q.sums = sums;
    const dim3 grid(p.parts, (unsigned)m.x.batch);
    if (m.grad_dtype == GVQ_BF16) hipLaunchKernelGGL((muon_norm_kernel<unsigned short>), grid, dim3(MUON_THREADS), 0, st, q);
    else hipLaunchKernelGGL((muon_norm_kernel<float>), grid, dim3(MUON_THREADS), 0, st, q);
    GVQ_HIP(hipGetLastError());
    return GVQ_OK;
}

bool gvq_muon_plan(const MuonMatrix& x, MuonPlan* p)
{
    if (x.batch < 0 || x.rows < 0 || x.cols < 0 || x.batch > 65535 || x.rows > (1 << 20) || x.cols > (1 << 20)) return false;
    p->m = x.rows < x.cols ? x.rows : x.cols;
    p->n = x.rows < x.cols ? x.cols : x.rows;
    p->ldn = ns_padded(p->n);
    p->ldm = ns_padded(p->m);
    p->bytes = 0;
    // a plane stays at 2 GiB, so that both planes of a tile's rows are within 32 bits of each other
    if (p->m * p->ldn > (int64_t)1 << 30) return false;
    if (gvq_muon_small_takes(x)) {
        MuonSmallPlan small;
        p->bytes = gvq_muon_small_plan(x, &small);
        return true;
    }
    int64_t at = 0;
    auto take = [&](int64_t bytes) { const int64_t was = at; at += (bytes + 255) / 256 * 256; return was; };
    for (int i = 0; i < 2; ++i) p->x[i] = take(p->m * p->ldn * 4);
    p->gram = take(p->m * p->ldm * 4);
    p->poly = take(p->m * p->ldm * 4);
    p->per = at;
    p->parts = gvq_muon_parts(x);
    at = x.batch * p->per;
    p->sums = take(x.batch * p->parts * (int64_t)sizeof(double));
    p->factors = take(x.batch * GVQ_MAX_STEPS * (int64_t)sizeof(NsFactors));
    const NsWays ways = ns_ways(x.batch, p->m, p->n);
    p->gram_by = ways.gram; p->poly_by = ways.poly; p->step_by = ways.step;
    int64_t most = ns_part_numbers(p->gram_by, p->m, p->m);
    const int64_t b = ns_part_numbers(p->poly_by, p->m, p->m), c = ns_part_numbers(p->step_by, p->m, p->n);
    most = most > b ? most : b;
    most = most > c ? most : c;
    p->parts_at = take(x.batch * most * (int64_t)sizeof(float));
    p->bytes = at;
    return true;
}

template <typename T, int KIND, typename OUT, bool SPLIT>
static int launch_tiles(const NsArgs& a, int64_t batch, hipStream_t st)
{
    const int64_t tiles = (KIND == NS_GRAM || KIND == NS_POLY ? (int64_t)a.nm * (a.nm + 1) / 2 : (int64_t)a.nm * a.nn) * a.splits;
    if (tiles > 0x7fffffff) return GVQ_EINVAL;
    static gvq_once_per_device lds;
    int dev;
    GVQ_HIP(hipGetDevice(&dev));
    const int rc = lds.call(dev, [] {
        GVQ_HIP(hipFuncSetAttribute((const void*)ns_tile_kernel<T, KIND, OUT, SPLIT>, hipFuncAttributeMaxDynamicSharedMemorySize, ns_lds<T>()));
        return (int)GVQ_OK;
    });
    if (rc != GVQ_OK) return rc;
    hipLaunchKernelGGL((ns_tile_kernel<T, KIND, OUT, SPLIT>), dim3((unsigned)tiles, (unsigned)batch), dim3(T::THREADS), ns_lds<T>(), st, a);
    GVQ_HIP(hipGetLastError());
    return GVQ_OK;
}

// The parts of a sum, and their join.
template <typename T, int KIND, typename OUT, bool TURN>
static int launch_parts(NsArgs a, int64_t batch, hipStream_t st)
{
    a.ld_part = (int64_t)a.nn * T::BN;
    a.part = a.ld_part * a.nm * T::BM;
    // (the parts of LAST lie as those of STEP: what a transpose needs is the join's to do)
    typedef TileShape<T::BM, T::BN, T::WM, T::WN, 2, T::STAGES, T::TURNED, false> Plain;
    const int rc = launch_tiles<Plain, KIND == NS_LAST ? (int)NS_STEP : KIND, float, true>(a, batch, st);
    if (rc != GVQ_OK) return rc;
    a.nm = (a.rows + 31) / 32;
    a.nn = (int)((KIND == NS_LAST ? a.cols + 31 : a.ld) / 32);
    const int64_t tiles = KIND == NS_GRAM || KIND == NS_POLY ? (int64_t)a.nm * (a.nm + 1) / 2 : (int64_t)a.nm * a.nn;
    hipLaunchKernelGGL((ns_join_kernel<KIND, OUT, TURN>), dim3((unsigned)tiles, (unsigned)batch), dim3(256), 0, st, a);
    GVQ_HIP(hipGetLastError());
    return GVQ_OK;
}

template <typename T, int KIND, typename OUT, bool TURN>
static int launch_shape(NsArgs a, int64_t batch, hipStream_t st)
{
    a.nm = (a.rows + T::BM - 1) / T::BM;
    a.nn = (a.cols + T::BN - 1) / T::BN;
    a.band = 4;
    if (a.splits == 1) return launch_tiles<T, KIND, OUT, false>(a, batch, st);
    if constexpr (ns_in_parts(T::BM, KIND == NS_GRAM)) return launch_parts<T, KIND, OUT, TURN>(a, batch, st);
    return GVQ_EINVAL;
}

template <int KIND, typename OUT, bool TURN>
static int launch_ns(NsArgs a, const NsChoice& by, int64_t batch, hipStream_t st)
{
    constexpr bool X = KIND == NS_STEP || KIND == NS_LAST;   // the second operand is X, whose rows run across the sum
    a.splits = by.splits;
    switch (by.shape) {
    case 0: return launch_shape<TileShape<256, 256, 2, 4, 2, 2, X, TURN>, KIND, OUT, TURN>(a, batch, st);
    case 1: if constexpr (!X) return launch_shape<TileShape<192, 192, 2, 4, 2, 3, X, TURN>, KIND, OUT, TURN>(a, batch, st);
            return GVQ_EINVAL;
    case 2: return launch_shape<TileShape<128, 128, 2, 4, 2, 4, X, TURN>, KIND, OUT, TURN>(a, batch, st);
    default: return launch_shape<TileShape<64, 64, 2, 2, 2, 4, X, TURN>, KIND, OUT, TURN>(a, batch, st);
    }
}

int gvq_launch_muon(const MuonArgs& m, hipStream_t st)
{
    MuonPlan p;
    if (!gvq_muon_plan(m.x, &p)) return GVQ_EINVAL;
    if (gvq_muon_small_takes(m.x)) return gvq_launch_muon_small(m, st);
    const int64_t batch = m.x.batch;
    const bool wide = m.x.rows <= m.x.cols;
    char* w = m.workspace;
    PrepArgs q = prep_args(m);
    q.sums = (double*)(w + p.sums);
    q.x = w + p.x[0]; q.per = p.per; q.plane = p.m * p.ldn; q.ld = p.ldn;
    q.factors = (NsFactors*)(w + p.factors);
    const MuonCoef coef = gvq_muon_coef(m);
    int rc = gvq_launch_muon_norm(m, q.p, q.sums, st);
    if (rc != GVQ_OK) return rc;
    // (the padding of X's rows is written too)
    const dim3 threads(MUON_THREADS);
    if (wide) {
        const dim3 grid((unsigned)(p.parts), (unsigned)batch);
        if (m.grad_dtype == GVQ_BF16) hipLaunchKernelGGL((muon_planes_kernel<unsigned short>), grid, threads, 0, st, q, coef);
        else hipLaunchKernelGGL((muon_planes_kernel<float>), grid, threads, 0, st, q, coef);
    } else {
        const dim3 grid((unsigned)((m.x.cols + 63) / 64), (unsigned)((p.ldn + 63) / 64), (unsigned)batch);
        if (m.grad_dtype == GVQ_BF16) hipLaunchKernelGGL((muon_turn_kernel<unsigned short>), grid, threads, 0, st, q, coef);
        else hipLaunchKernelGGL((muon_turn_kernel<float>), grid, threads, 0, st, q, coef);
    }
    GVQ_HIP(hipGetLastError());
    const int mm = (int)p.m, nn = (int)p.n;
    const int64_t es = m.out_dtype == GVQ_BF16 ? 2 : 4;
    const TileOperand gram{w + p.gram, mm * p.ldm * 2, p.ldm * 2, mm, nullptr, 0};
    const TileOperand poly{w + p.poly, mm * p.ldm * 2, p.ldm * 2, mm, nullptr, 0};
    for (int s = 0; s < m.steps; ++s) {
        const TileOperand X{w + p.x[s & 1], mm * p.ldn * 2, p.ldn * 2, mm, nullptr, 0};
        NsArgs n{};
        n.per = p.per;
        n.parts = (float*)(w + p.parts_at);
        n.f = q.factors + s;
        // A = X X^T
        n.a = n.b = X;
        n.steps = (int)(p.ldn / 32);
        n.rows = n.cols = mm;
        n.res = (_Float16*)(w + p.gram);
        n.plane = mm * p.ldm;
        n.ld = p.ldm;
        rc = launch_ns<NS_GRAM, float, false>(n, p.gram_by, batch, st);
        if (rc != GVQ_OK) return rc;
        // b A + c A A
        n.a = n.b = gram;
        n.steps = (int)(p.ldm / 32);
        n.old = (const _Float16*)(w + p.gram);
        n.res = (_Float16*)(w + p.poly);
        rc = launch_ns<NS_POLY, float, false>(n, p.poly_by, batch, st);
        if (rc != GVQ_OK) return rc;
        // a X + (b A + c A A) X
        n.a = poly;
        n.b = X;
        n.b.rows = nn;
        n.b.depth = mm;
        n.cols = nn;
        n.old = (const _Float16*)(w + p.x[s & 1]);
        n.plane = mm * p.ldn;
        n.ld = p.ldn;
        if (s + 1 < m.steps) {
            n.res = (_Float16*)(w + p.x[(s + 1) & 1]);
            rc = launch_ns<NS_STEP, float, false>(n, p.step_by, batch, st);
        } else {
            n.out = m.out;
            n.ld_out = m.ld_out;
            n.stride_out = m.stride_out;
            n.update = m.update;
            n.keep = m.keep;
            n.rate = m.rate;
            n.words = (((uintptr_t)m.out | (uintptr_t)(m.ld_out * es) | (uintptr_t)(m.stride_out * es)) & (uintptr_t)(4 * es - 1)) == 0;
            if (m.out_dtype == GVQ_BF16)
                rc = wide ? launch_ns<NS_LAST, unsigned short, false>(n, p.step_by, batch, st) : launch_ns<NS_LAST, unsigned short, true>(n, p.step_by, batch, st);
            else
                rc = wide ? launch_ns<NS_LAST, float, false>(n, p.step_by, batch, st) : launch_ns<NS_LAST, float, true>(n, p.step_by, batch, st);
        }
        if (rc != GVQ_OK) return rc;
    }
    return GVQ_OK;
}
