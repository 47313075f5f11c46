// Muon's step: momentum, Newton-Schulz orthogonalisation, decayed weight minus the step.
//
// X_0 = U / (|U|_F + eps), then X <- a X + (b A + c A A) X with A = X X^T (for a tall matrix X (b A + c A A) with A = X^T X, the
// same polynomial of the smaller Gram matrix).  Its singular values s follow s <- a s + b s^3 + c s^5, towards 1.
//
// Precision.  The steps multiply small singular values by a = 3.4 each, 485 in all, and what rounding adds to X along such a
// direction grows with them: numbers kept in bf16 end 1 to 7 % off (2-norm, planted low rank the worst), in f16 0.1 to 0.9 %.
// So X, A and the polynomial are kept as two f16 terms, 22 bits, in fixed units of 2^-12 (X, A) and 2^-10 (the polynomial), and
// every product is hi hi + hi lo + lo hi in fp32 sums: as exact as fp32 products (1.0 to 1.15 times their error), at a third of
// the f16 matrix pipe's rate, which is five times the fp32 pipe's.
#include "gvq_muon.h"
#include "gvq_tile.h"

#define UNIT_X 4096.f
#define UNIT_P 1024.f
#define MUON_THREADS 256

struct PrepArgs {
    const void* grad;
    int64_t ld_grad, stride_grad;
    float* momentum;
    int64_t ld_momentum;
    float beta;
    int nesterov;
    int64_t rows, cols;
    double* sums;        // [batch][parts]
    int parts;
    double eps;
    char* ws;
    int64_t per;
    int64_t nat, tr, ldc, ldr;
};

template <typename G>
__device__ __forceinline__ float grad_at(const G* g, int64_t i);
template <>
__device__ __forceinline__ float grad_at<float>(const float* g, int64_t i) { return g[i]; }
template <>
__device__ __forceinline__ float grad_at<unsigned short>(const unsigned short* g, int64_t i) { return bf16_to_f32(g[i]); }

// Sum over a work-group of MUON_THREADS, in a fixed order; every thread gets it.
__device__ __forceinline__ double group_sum(double v, double* lds)
{
#pragma unroll
    for (int m = 32; m; m >>= 1) v += __shfl_xor(v, m);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    double s = 0;
#pragma unroll
    for (int w = 0; w < MUON_THREADS / 64; ++w) s += lds[w];
    __syncthreads();
    return s;
}

// M <- beta M + G, and the sum of squares of U, in float64 (squares of fp32 numbers are exact there and do not overflow).
template <typename G>
__global__ __launch_bounds__(MUON_THREADS) void muon_norm_kernel(PrepArgs a)
{
    __shared__ double lds[MUON_THREADS / 64];
    const G* g = (const G*)a.grad + blockIdx.y * a.stride_grad;
    double s = 0;
    const int64_t n = a.rows * a.cols, step = (int64_t)gridDim.x * MUON_THREADS;
    for (int64_t i = (int64_t)blockIdx.x * MUON_THREADS + threadIdx.x; i < n; i += step) {
        const int64_t r = i / a.cols, c = i - r * a.cols;
        float u = grad_at<G>(g, r * a.ld_grad + c);
        if (a.momentum) {
            float* m = a.momentum + r * a.ld_momentum + c;
            const float v = a.beta * *m + u;
            *m = v;
            u = a.nesterov ? u + a.beta * v : v;
        }
        s += (double)u * u;
    }
    s = group_sum(s, lds);
    if (threadIdx.x == 0) a.sums[blockIdx.y * a.parts + blockIdx.x] = s;
}

__device__ __forceinline__ void split_f16(float v, _Float16& hi, _Float16& lo)
{
    hi = (_Float16)v;
    lo = (_Float16)(v - (float)hi);
}

// U / (|U| + eps) into the planes of both orientations, with zeros behind the last column: 64 x 64 numbers a work-group.
template <typename G>
__global__ __launch_bounds__(MUON_THREADS) void muon_planes_kernel(PrepArgs a)
{
    __shared__ double lds[MUON_THREADS / 64];
    __shared__ float tile[64 * 65];
    double s = 0;
    for (int i = threadIdx.x; i < a.parts; i += MUON_THREADS) s += a.sums[blockIdx.z * a.parts + i];
    const double inv = 1.0 / (sqrt(group_sum(s, lds)) + a.eps) * UNIT_X;
    const G* g = (const G*)a.grad + blockIdx.z * a.stride_grad;
    char* ws = a.ws + blockIdx.z * a.per;
    const int64_t r0 = (int64_t)blockIdx.y * 64, c0 = (int64_t)blockIdx.x * 64;
    const int x = threadIdx.x & 63, y0 = threadIdx.x >> 6;
    _Float16* nat = (_Float16*)(ws + a.nat);
    _Float16* tr = (_Float16*)(ws + a.tr);
#pragma unroll 4
    for (int y = y0; y < 64; y += MUON_THREADS / 64) {
        const int64_t r = r0 + y, c = c0 + x;
        float v = 0.f;
        if (r < a.rows && c < a.cols) {
            float u = grad_at<G>(g, r * a.ld_grad + c);
            if (a.momentum) {
                const float m = a.momentum[r * a.ld_momentum + c];
                u = a.nesterov ? u + a.beta * m : m;
            }
            v = (float)((double)u * inv);
        }
        tile[y * 65 + x] = v;
        if (r < a.rows && c < a.ldc) {
            _Float16 hi, lo;
            split_f16(v, hi, lo);
            nat[r * a.ldc + c] = hi;
            nat[a.rows * a.ldc + r * a.ldc + c] = lo;
        }
    }
    __syncthreads();
#pragma unroll 4
    for (int y = y0; y < 64; y += MUON_THREADS / 64) {
        const int64_t c = c0 + y, r = r0 + x;
        if (c < a.cols && r < a.ldr) {
            _Float16 hi, lo;
            split_f16(tile[x * 65 + y], hi, lo);
            tr[c * a.ldr + r] = hi;
            tr[a.cols * a.ldr + c * a.ldr + r] = lo;
        }
    }
}

// The three products of a step.
enum { NS_GRAM = 0, NS_POLY = 1, NS_STEP = 2, NS_LAST = 3 };

struct NsArgs {
    TileOperand a, b;          // of the first matrix; `per` bytes further for each next one
    int steps, nm, nn, band;
    int64_t per;
    float scale;               // of the sum, in units of the result
    float ca, cb;              // POLY: result = ca old + cb sum; STEP, LAST: ca old + sum
    const _Float16* old;       // POLY: A, STEP and LAST: X, in natural layout
    int64_t old_plane;
    _Float16 *nat, *tr;        // results (POLY, GRAM: tr == nat, mirrored)
    int64_t nat_plane, tr_plane, ldn, ldt;
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

// Four neighbouring results of row r from column c on into the planes: natural, and transposed (or mirrored).
__device__ __forceinline__ void store_planes(const NsArgs& a, _Float16* nat, _Float16* tr, int r, int c, int rows, int cols, bool turn, f4 v)
{
    h4 hi, lo;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        _Float16 h, l;
        split_f16(c + i < cols && r < rows ? v[i] : 0.f, h, l);
        hi[i] = h; lo[i] = l;
    }
    if (r < rows && c < a.ldn) {
        *(h4*)(nat + (int64_t)r * a.ldn + c) = hi;
        *(h4*)(nat + a.nat_plane + (int64_t)r * a.ldn + c) = lo;
    }
    if (turn && r < a.ldt) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (c + i < cols) {
                tr[(int64_t)(c + i) * a.ldt + r] = hi[i];
                tr[a.tr_plane + (int64_t)(c + i) * a.ldt + r] = lo[i];
            }
    }
}

// KIND: which product; GRAM and POLY compute the tiles on and above the diagonal and mirror them.
template <typename T, int KIND, typename OUT>
__global__ __launch_bounds__(T::THREADS) void ns_tile_kernel(NsArgs a)
{
    extern __shared__ char lds[];
    int tm, tn;
    if (KIND == NS_GRAM || KIND == NS_POLY) {
        // column tn of the triangle holds the tiles (0 .. tn, tn), tn (tn + 1) / 2 of them before it
        const int t = tile_of_block(blockIdx.x, a.nm * (a.nm + 1) / 2);
        tn = (int)((sqrtf(8.f * (float)t + 1.f) - 1.f) * 0.5f);
        while (tn * (tn + 1) / 2 > t) --tn;
        while ((tn + 1) * (tn + 2) / 2 <= t) ++tn;
        tm = t - tn * (tn + 1) / 2;
    } else {
        tile_at(tile_of_block(blockIdx.x, a.nm * a.nn), a.nm, a.nn, a.band, tm, tn);
    }
    const int64_t off = blockIdx.y * a.per;
    TileOperand A = a.a, B = a.b;
    A.p += off;
    B.p += off;
    f4 acc[T::MI][T::NI];
#pragma unroll
    for (int mi = 0; mi < T::MI; ++mi)
#pragma unroll
        for (int ni = 0; ni < T::NI; ++ni) acc[mi][ni] = f4{0.f, 0.f, 0.f, 0.f};
    tile_product<T>(A, B, tm * T::BM, tn * T::BN, 0, a.steps, lds, acc);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int r0 = tm * T::BM + wave / T::WN * (T::BM / T::WM) + (lane & 15);
    const int c0 = tn * T::BN + wave % T::WN * (T::BN / T::WN) + 4 * (lane >> 4);
    _Float16* nat = (_Float16*)((char*)a.nat + off);
    _Float16* tr = (_Float16*)((char*)a.tr + off);
    const _Float16* old = (const _Float16*)((const char*)a.old + off);
#pragma unroll
    for (int mi = 0; mi < T::MI; ++mi) {
        const int r = r0 + 16 * mi;
#pragma unroll
        for (int ni = 0; ni < T::NI; ++ni) {
            const int c = c0 + 16 * ni;
            f4 v = acc[mi][ni] * a.scale;
            if (KIND != NS_GRAM && r < A.rows && c < a.ldn) {
                const h4 hi = *(const h4*)(old + (int64_t)r * a.ldn + c), lo = *(const h4*)(old + a.old_plane + (int64_t)r * a.ldn + c);
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = a.ca * ((float)hi[i] + (float)lo[i]) + (KIND == NS_POLY ? a.cb * v[i] : v[i]);
            }
            if (KIND == NS_LAST) {
                if (r < A.rows && c < B.rows)
                    last_store4<OUT>((OUT*)a.out + blockIdx.y * a.stride_out + (int64_t)r * a.ld_out + c, a.words != 0, B.rows - c, a.update,
                                     a.keep, a.rate, v * (1.f / UNIT_X));
            } else {
                store_planes(a, nat, tr, r, c, A.rows, B.rows, KIND == NS_STEP || tm != tn, v);
            }
        }
    }
}

static int64_t padded(int64_t n) { return (n + 31) / 32 * 32; }

bool gvq_muon_plan(const MuonMatrix& x, MuonPlan* p)
{
    const int64_t most = (int64_t)1 << 30;
    if (x.batch < 0 || x.rows < 0 || x.cols < 0 || x.batch > 65535 || x.rows > (1 << 20) || x.cols > (1 << 20)) return false;
    p->ldc = padded(x.cols);
    p->ldr = padded(x.rows);
    const int64_t m = x.rows < x.cols ? x.rows : x.cols;
    p->ldm = padded(m);
    // a plane stays below 2 GiB, so that both planes of a tile's rows are within 32 bits of each other
    if (x.rows * p->ldc > most || x.cols * p->ldr > most) return false;
    int64_t at = 0;
    auto take = [&](int64_t bytes) { const int64_t was = at; at += (bytes + 255) / 256 * 256; return was; };
    for (int i = 0; i < 2; ++i) {
        p->nat[i] = take(x.rows * p->ldc * 4);
        p->tr[i] = take(x.cols * p->ldr * 4);
    }
    p->gram = take(m * p->ldm * 4);
    p->poly = take(m * p->ldm * 4);
    p->per = at;
    const int64_t n = x.rows * x.cols;
    const int64_t parts = (n + 16 * MUON_THREADS - 1) / (16 * MUON_THREADS);
    p->parts = (int)(parts < 1 ? 1 : parts > 1024 ? 1024 : parts);
    p->sums = x.batch * p->per;
    p->bytes = p->sums + x.batch * p->parts * (int64_t)sizeof(double);
    return true;
}

template <typename T, int KIND, typename OUT>
static int launch_ns_tile(NsArgs a, int64_t batch, hipStream_t st)
{
    a.nm = (a.a.rows + T::BM - 1) / T::BM;
    a.nn = (a.b.rows + T::BN - 1) / T::BN;
    a.band = 4;
    const int64_t tiles = KIND == NS_GRAM || KIND == NS_POLY ? (int64_t)a.nm * (a.nm + 1) / 2 : (int64_t)a.nm * a.nn;
    if (tiles > 0x7fffffff) return GVQ_EINVAL;
    static gvq_once_per_device lds;
    int dev;
    GVQ_HIP(hipGetDevice(&dev));
    const int rc = lds.call(dev, [] {
        GVQ_HIP(hipFuncSetAttribute((const void*)ns_tile_kernel<T, KIND, OUT>, hipFuncAttributeMaxDynamicSharedMemorySize, T::LDS));
        return (int)GVQ_OK;
    });
    if (rc != GVQ_OK) return rc;
    hipLaunchKernelGGL((ns_tile_kernel<T, KIND, OUT>), dim3((unsigned)tiles, (unsigned)batch), dim3(T::THREADS), T::LDS, st, a);
    GVQ_HIP(hipGetLastError());
    return GVQ_OK;
}

template <int KIND, typename OUT>
static int launch_ns(const NsArgs& a, int64_t batch, hipStream_t st)
{
    const int64_t big = batch * ((a.a.rows + 255) / 256) * ((a.b.rows + 255) / 256);
    if (big >= 192) return launch_ns_tile<TileShape<256, 256, 2, 4, 2, 2>, KIND, OUT>(a, batch, st);
    return launch_ns_tile<TileShape<64, 64, 2, 2, 2, 4>, KIND, OUT>(a, batch, st);
}

int gvq_launch_muon(const MuonArgs& m, hipStream_t st)
{
    MuonPlan p;
    if (!gvq_muon_plan(m.x, &p)) return GVQ_EINVAL;
    const int64_t batch = m.x.batch, rows = m.x.rows, cols = m.x.cols;
    PrepArgs q{};
    q.grad = m.grad; q.ld_grad = m.ld_grad; q.stride_grad = m.stride_grad;
    q.momentum = m.momentum; q.ld_momentum = m.ld_momentum;
    q.beta = m.beta; q.nesterov = m.nesterov;
    q.rows = rows; q.cols = cols;
    q.sums = (double*)(m.workspace + p.sums);
    q.parts = p.parts;
    q.eps = m.eps;
    q.ws = m.workspace; q.per = p.per; q.nat = p.nat[0]; q.tr = p.tr[0]; q.ldc = p.ldc; q.ldr = p.ldr;
    const dim3 g1(p.parts, (unsigned)batch), g2((unsigned)((p.ldc + 63) / 64), (unsigned)((p.ldr + 63) / 64), (unsigned)batch);
    if (m.grad_dtype == GVQ_BF16) {
        hipLaunchKernelGGL((muon_norm_kernel<unsigned short>), g1, dim3(MUON_THREADS), 0, st, q);
        hipLaunchKernelGGL((muon_planes_kernel<unsigned short>), g2, dim3(MUON_THREADS), 0, st, q);
    } else {
        hipLaunchKernelGGL((muon_norm_kernel<float>), g1, dim3(MUON_THREADS), 0, st, q);
        hipLaunchKernelGGL((muon_planes_kernel<float>), g2, dim3(MUON_THREADS), 0, st, q);
    }
    GVQ_HIP(hipGetLastError());
    const bool wide = rows <= cols;
    const int mm = (int)(wide ? rows : cols), nn = (int)(wide ? cols : rows);
    const int64_t es = m.out_dtype == GVQ_BF16 ? 2 : 4;
    for (int s = 0; s < m.steps; ++s) {
        const float a = (float)(m.coef ? m.coef[3 * s] : 3.4445), b = (float)(m.coef ? m.coef[3 * s + 1] : -4.7750),
                    c = (float)(m.coef ? m.coef[3 * s + 2] : 2.0315);
        char* w = m.workspace;
        const int now = s & 1, next = now ^ 1;
        const TileOperand nat{w + p.nat[now], rows * p.ldc * 2, p.ldc * 2, (int)rows, nullptr};
        const TileOperand tr{w + p.tr[now], cols * p.ldr * 2, p.ldr * 2, (int)cols, nullptr};
        const TileOperand gram{w + p.gram, mm * p.ldm * 2, p.ldm * 2, mm, nullptr};
        const TileOperand poly{w + p.poly, mm * p.ldm * 2, p.ldm * 2, mm, nullptr};
        NsArgs n{};
        n.per = p.per;
        // A = X X^T, the sum along the longer side
        n.a = n.b = wide ? nat : tr;
        n.steps = (int)((padded(nn) * 2) / TILE_STEP);
        n.scale = 1.f / UNIT_X;   // (x UNIT_X)(x UNIT_X) -> A UNIT_X
        n.nat = n.tr = (_Float16*)(w + p.gram);
        n.nat_plane = n.tr_plane = mm * p.ldm;
        n.ldn = n.ldt = p.ldm;
        int rc = launch_ns<NS_GRAM, float>(n, batch, st);
        if (rc != GVQ_OK) return rc;
        // b A + c A A
        n.a = n.b = gram;
        n.steps = (int)(p.ldm * 2 / TILE_STEP);
        n.scale = UNIT_P / (UNIT_X * UNIT_X);
        n.ca = b * (UNIT_P / UNIT_X);
        n.cb = c;
        n.old = (const _Float16*)(w + p.gram);
        n.old_plane = mm * p.ldm;
        n.nat = n.tr = (_Float16*)(w + p.poly);
        rc = launch_ns<NS_POLY, float>(n, batch, st);
        if (rc != GVQ_OK) return rc;
        // a X + (b A + c A A) X, or X from the left of it
        n.a = wide ? poly : nat;
        n.b = wide ? tr : poly;
        n.scale = 1.f / UNIT_P;
        n.ca = a;
        n.old = (const _Float16*)(w + p.nat[now]);
        n.old_plane = rows * p.ldc;
        n.ldn = p.ldc;
        if (s + 1 < m.steps) {
            n.nat = (_Float16*)(w + p.nat[next]);
            n.nat_plane = rows * p.ldc;
            n.tr = (_Float16*)(w + p.tr[next]);
            n.tr_plane = cols * p.ldr;
            n.ldt = p.ldr;
            rc = launch_ns<NS_STEP, float>(n, batch, st);
        } else {
            n.out = m.out;
            n.ld_out = m.ld_out;
            n.stride_out = m.stride_out;
            n.update = m.update;
            n.keep = m.keep;
            n.rate = m.rate;
            n.words = (((uintptr_t)m.out | (uintptr_t)(m.ld_out * es) | (uintptr_t)(m.stride_out * es)) & (uintptr_t)(4 * es - 1)) == 0;
            rc = m.out_dtype == GVQ_BF16 ? launch_ns<NS_LAST, unsigned short>(n, batch, st) : launch_ns<NS_LAST, float>(n, batch, st);
        }
        if (rc != GVQ_OK) return rc;
    }
    return GVQ_OK;
}
