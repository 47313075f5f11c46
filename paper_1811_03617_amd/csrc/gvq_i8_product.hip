// Products of 8-bit integers, C = A B^T with a scale for every row of A and of B, on the int8 matrix pipe (v_mfma_i32_16x16x64_i8: exact
// products, exact 32-bit sums; (int)sum is rounded to fp32 once and multiplied by the product of both scales).  Gated: the second
// operand's rows are a gate's and another projection's, a wave has both sums of the same places, and what leaves is act(g) u, or, given the
// gradient of that, the gradients of g and u.
#include "gvq_i8.h"
#include "gvq_tile.h"

#define I8_STEP 128   // bytes of a row per step: a line

// BM rows of A by BN of B, WM x WN waves.  A step's rows lie in LDS one behind the other, row r's piece c of 16 bytes in place
// c ^ (r & 7): the 16 lanes whose reads are served together then cover all banks.
template <int BM_, int BN_, int WM_, int WN_, int STAGES_>
struct I8Shape {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, STAGES = STAGES_;
    static constexpr int WAVES = WM * WN, THREADS = 64 * WAVES, MI = BM / WM / 16, NI = BN / WN / 16;
    static constexpr int STAGE = (BM + BN) * I8_STEP, LDS = STAGE * STAGES;
    static constexpr int GROUPS = (BM + BN) / 8, COPIES = GROUPS / WAVES;   // 1 KB copies of a step: eight rows each
    static_assert(GROUPS % WAVES == 0 && BM % 16 == 0 && LDS <= 160 * 1024 && COPIES * STAGES < 64, "whole copies, LDS and vmcnt");
};

// Row of B that the tile's row j is.  Gated: groups of 16 of the gate's and of the other's in turn.
template <I8Mode MODE>
__device__ __forceinline__ int64_t i8_row_of_b(int tn, int BN, int j, int n)
{
    if (MODE == I8_PLAIN) {
        const int r = tn * BN + j;
        return r < n ? r : n - 1;
    }
    const int r = tn * (BN / 2) + (j >> 5) * 16 + (j & 15);
    return (int64_t)(r < n ? r : n - 1) + ((j >> 4) & 1 ? n : 0);
}

template <typename T, I8Mode MODE>
__device__ __forceinline__ void i8_tile(const I8ProductArgs& a, int tm, int tn, char* lds, i4v (&acc)[T::MI][T::NI])
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int wm = wave / T::WN, wn = wave % T::WN, steps = (int)(a.ldk / I8_STEP);
    const unsigned int lds0 = lds_offset(lds);
    const char* base[T::COPIES];
    unsigned int voff[T::COPIES];
#pragma unroll
    for (int i = 0; i < T::COPIES; ++i) {
        const int j0 = (wave * T::COPIES + i) * 8, j = j0 + (lane >> 3), piece = (lane & 7) ^ (lane >> 3);
        if (j0 < T::BM) {
            const int64_t first = (int64_t)tm * T::BM + j0 < a.m ? (int64_t)tm * T::BM + j0 : a.m - 1;
            const int64_t r = (int64_t)tm * T::BM + j < a.m ? (int64_t)tm * T::BM + j : a.m - 1;
            base[i] = (const char*)a.a + first * a.ldk;
            voff[i] = (unsigned int)((r - first) * a.ldk) + 16 * piece;
        } else {
            const int64_t first = i8_row_of_b<MODE>(tn, T::BN, j0 - T::BM, a.n), r = i8_row_of_b<MODE>(tn, T::BN, j - T::BM, a.n);
            base[i] = (const char*)a.b + first * a.ldk;
            voff[i] = (unsigned int)((r - first) * a.ldk) + 16 * piece;
        }
    }
    auto issue = [&](int s) {
        const unsigned int to = lds0 + (unsigned int)(s % T::STAGES) * T::STAGE + (unsigned int)(wave * T::COPIES) * 1024;
#pragma unroll
        for (int i = 0; i < T::COPIES; ++i) copy_rows_to_lds(base[i] + (int64_t)s * I8_STEP, voff[i], to + i * 1024);
    };
    const int row = lane & 15;
    for (int s = 0; s < T::STAGES - 1 && s < steps; ++s) issue(s);
    for (int s = 0; s < steps; ++s) {
        // this wave's copies of step s have arrived, and then everybody's; everybody is done with the place that is asked for next
        if (s + T::STAGES - 1 <= steps) tile_barrier<T::COPIES * (T::STAGES - 2)>();
        else tile_barrier<0>();
        if (s + T::STAGES - 1 < steps) issue(s + T::STAGES - 1);
        const char* st = lds + (s % T::STAGES) * T::STAGE;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int piece = ((4 * k + (lane >> 4)) ^ (row & 7)) * 16;
            i4v fb[T::NI];
#pragma unroll
            for (int ni = 0; ni < T::NI; ++ni) fb[ni] = *(const i4v*)(st + (T::BM + (wn * T::NI + ni) * 16 + row) * I8_STEP + piece);
#pragma unroll
            for (int mi = 0; mi < T::MI; ++mi) {
                const i4v fa = *(const i4v*)(st + ((wm * T::MI + mi) * 16 + row) * I8_STEP + piece);
#pragma unroll
                for (int ni = 0; ni < T::NI; ++ni) acc[mi][ni] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[ni], fa, acc[mi][ni], 0, 0, 0);
            }
        }
    }
}

__device__ __forceinline__ f4 i8_load4(const float* p, bool words, int left)
{
    if (words && left >= 4) return *(const f4*)p;
    f4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < left) v[i] = p[i];
    return v;
}
__device__ __forceinline__ f4 i8_load4(const unsigned short* p, bool words, int left)
{
    f4 v = {0.f, 0.f, 0.f, 0.f};
    if (words && left >= 4) {
        const u2 o = *(const u2*)p;
        return f4{__uint_as_float(o[0] << 16), __uint_as_float(o[0] & 0xffff0000u), __uint_as_float(o[1] << 16), __uint_as_float(o[1] & 0xffff0000u)};
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < left) v[i] = bf16_to_f32(p[i]);
    return v;
}

template <typename T, I8Mode MODE, typename OUT>
__global__ __launch_bounds__(T::THREADS) void i8_tile_kernel(I8ProductArgs a)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    int tm, tn;
    tile_at(tile_of_block(blockIdx.x, a.nm * a.nn), a.nm, a.nn, a.band, tm, tn);
    i4v acc[T::MI][T::NI];
#pragma unroll
    for (int mi = 0; mi < T::MI; ++mi)
#pragma unroll
        for (int ni = 0; ni < T::NI; ++ni) acc[mi][ni] = i4v{0, 0, 0, 0};
    i8_tile<T, MODE>(a, tm, tn, lds, acc);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int r0 = tm * T::BM + wave / T::WN * (T::BM / T::WM);
    constexpr int PAIR = MODE == I8_PLAIN ? 1 : 2, COLS = T::BN / T::WN / PAIR;
    const int c0 = tn * (T::BN / PAIR) + wave % T::WN * COLS + 4 * (lane >> 4);
    OUT* out = (OUT*)a.out;
#pragma unroll
    for (int ni = 0; ni < T::NI; ni += PAIR) {
        const int c = c0 + 16 * (ni / PAIR), left = a.n - c;
        f4 sg = {0.f, 0.f, 0.f, 0.f}, su = sg;
        if (a.ldk > 0) {   // (a sum over nothing has no scales)
            sg = i8_load4(a.b_scales + c, false, left);
            if constexpr (MODE != I8_PLAIN) su = i8_load4(a.b_scales + a.n + c, false, left);
        }
#pragma unroll
        for (int mi = 0; mi < T::MI; ++mi) {
            const int r = r0 + 16 * mi + (lane & 15);
            if (r >= a.m) continue;
            const float sa = a.ldk > 0 ? a.a_scales[r] : 0.f;
            f4 g, u;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                g[i] = (float)acc[mi][ni][i] * (sa * sg[i]);
                if constexpr (MODE != I8_PLAIN) u[i] = (float)acc[mi][ni + 1][i] * (sa * su[i]);
            }
            if constexpr (MODE == I8_PLAIN) {
                mx_store4(out + (int64_t)r * a.ld + c, a.words != 0, left, a.accumulate != 0, g);
            } else if constexpr (MODE == I8_GATED) {
#pragma unroll
                for (int i = 0; i < 4; ++i) g[i] = i8_activation(g[i], a.activation) * u[i];
                mx_store4(out + (int64_t)r * a.ld + c, a.words != 0, left, false, g);
            } else {
                const f4 dh = i8_load4((const OUT*)a.dh + (int64_t)r * a.ld_dh + c, a.dh_words != 0, left);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float value, slope;
                    i8_activation_slope(g[i], a.activation, value, slope);
                    g[i] = dh[i] * u[i] * slope;
                    u[i] = dh[i] * value;
                }
                mx_store4(out + (int64_t)r * a.ld + c, a.words != 0, left, false, g);
                mx_store4(out + (int64_t)r * a.ld + a.n + c, a.words != 0 && (a.n & 3) == 0, left, false, u);
            }
        }
    }
}

template <typename T, I8Mode MODE, typename OUT>
static int launch_tile(I8ProductArgs a, hipStream_t st)
{
    constexpr int COLS = MODE == I8_PLAIN ? T::BN : T::BN / 2;
    a.nm = (a.m + T::BM - 1) / T::BM;
    a.nn = (a.n + COLS - 1) / COLS;
    if ((int64_t)a.nm * a.nn > 0x7fffffff) return GVQ_EINVAL;
    a.band = 4;
    static gvq_once_per_device lds;
    int dev;
    GVQ_HIP(hipGetDevice(&dev));
    const int rc = lds.call(dev, [] {
        GVQ_HIP(hipFuncSetAttribute((const void*)i8_tile_kernel<T, MODE, OUT>, hipFuncAttributeMaxDynamicSharedMemorySize, T::LDS));
        return (int)GVQ_OK;
    });
    if (rc != GVQ_OK) return rc;
    hipLaunchKernelGGL((i8_tile_kernel<T, MODE, OUT>), dim3(a.nm * a.nn), dim3(T::THREADS), T::LDS, st, a);
    GVQ_HIP(hipGetLastError());
    return GVQ_OK;
}

template <I8Mode MODE, typename OUT>
static int launch_mode(const I8ProductArgs& a, hipStream_t st)
{
    return launch_tile<I8Shape<128, 128, 2, 2, 2>, MODE, OUT>(a, st);
}

int gvq_launch_i8_product(I8ProductArgs a, I8Mode mode, gvq_dtype_t dtype, hipStream_t st)
{
    const int64_t es = dtype == GVQ_BF16 ? 2 : 4;
    a.words = (((uintptr_t)a.out | (uintptr_t)(a.ld * es)) & (uintptr_t)(4 * es - 1)) == 0;
    a.dh_words = (((uintptr_t)a.dh | (uintptr_t)(a.ld_dh * es)) & (uintptr_t)(4 * es - 1)) == 0;
    if (dtype == GVQ_BF16)
        return mode == I8_PLAIN ? launch_mode<I8_PLAIN, unsigned short>(a, st)
                                : mode == I8_GATED ? launch_mode<I8_GATED, unsigned short>(a, st) : launch_mode<I8_INNER, unsigned short>(a, st);
    return mode == I8_PLAIN ? launch_mode<I8_PLAIN, float>(a, st)
                            : mode == I8_GATED ? launch_mode<I8_GATED, float>(a, st) : launch_mode<I8_INNER, float>(a, st);
}
