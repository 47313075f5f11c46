// Products of 4-bit microscaled matrices, C = A B^T, on the scaled 4-bit matrix pipe (v_mfma_scale_f32_16x16x128_f8f6f4: exact
// products of codes, scaled per block of 32, fp32 sums).
#include "gvq_mx.h"
#include "gvq_tile.h"

struct MxProductArgs {
    TileOperand a, b;
    int steps;         // of 128 numbers
    int nm, nn, band;  // tiles, and how they are swept
    void* out;
    int64_t ld;
    int accumulate, words;   // words: four neighbouring results are one aligned word
};

template <typename T, typename OUT>
__global__ __launch_bounds__(T::THREADS) void mx_tile_kernel(MxProductArgs a)
{
    extern __shared__ char lds[];
    int tm, tn;
    tile_at(tile_of_block(blockIdx.x, a.nm * a.nn), a.nm, a.nn, a.band, tm, tn);
    f4 acc[T::MI][T::NI];
#pragma unroll
    for (int mi = 0; mi < T::MI; ++mi)
#pragma unroll
        for (int ni = 0; ni < T::NI; ++ni) acc[mi][ni] = f4{0.f, 0.f, 0.f, 0.f};
    tile_product<T>(a.a, a.b, tm * T::BM, tn * T::BN, 0, a.steps, lds, acc);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int r0 = tm * T::BM + wave / T::WN * (T::BM / T::WM) + (lane & 15);
    const int c0 = tn * T::BN + wave % T::WN * (T::BN / T::WN) + 4 * (lane >> 4);
#pragma unroll
    for (int mi = 0; mi < T::MI; ++mi) {
        const int r = r0 + 16 * mi;
        if (r >= a.a.rows) continue;
        OUT* row = (OUT*)a.out + (int64_t)r * a.ld;
#pragma unroll
        for (int ni = 0; ni < T::NI; ++ni) mx_store4(row + c0 + 16 * ni, a.words != 0, a.b.rows - (c0 + 16 * ni), a.accumulate != 0, acc[mi][ni]);
    }
}

template <typename T, typename OUT>
static int launch_tile(MxProductArgs a, hipStream_t st)
{
    a.nm = (a.a.rows + T::BM - 1) / T::BM;
    a.nn = (a.b.rows + T::BN - 1) / T::BN;
    if ((int64_t)a.nm * a.nn > 0x7fffffff) return GVQ_EINVAL;
    a.band = 4;
    static gvq_once_per_device lds;
    int dev;
    GVQ_HIP(hipGetDevice(&dev));
    const int rc = lds.call(dev, [] {
        GVQ_HIP(hipFuncSetAttribute((const void*)mx_tile_kernel<T, OUT>, hipFuncAttributeMaxDynamicSharedMemorySize, T::LDS));
        return (int)GVQ_OK;
    });
    if (rc != GVQ_OK) return rc;
    hipLaunchKernelGGL((mx_tile_kernel<T, OUT>), dim3(a.nm * a.nn), dim3(T::THREADS), T::LDS, st, a);
    GVQ_HIP(hipGetLastError());
    return GVQ_OK;
}

template <typename OUT>
static int launch_product(const MxProductArgs& a, hipStream_t st)
{
    const int64_t big = (int64_t)((a.a.rows + 255) / 256) * ((a.b.rows + 255) / 256);
    if (big >= 192) return launch_tile<TileShape<256, 256, 2, 4, 1, 4>, OUT>(a, st);
    return launch_tile<TileShape<64, 64, 2, 2, 1, 4>, OUT>(a, st);
}

int gvq_launch_mx_matmul(const void* a_codes, const void* a_scales, const void* b_codes, const void* b_scales, int64_t m, int64_t n,
                         int64_t k, void* out, gvq_dtype_t dtype, int64_t ld, bool accumulate, hipStream_t st)
{
    MxProductArgs a;
    const int64_t row = gvq_mx_row_bytes(k), es = dtype == GVQ_BF16 ? 2 : 4;
    a.a = TileOperand{(const char*)a_codes, 0, row, (int)m, (const char*)a_scales, 0};
    a.b = TileOperand{(const char*)b_codes, 0, row, (int)n, (const char*)b_scales, 0};
    a.steps = (int)(row / TILE_STEP);
    a.out = out;
    a.ld = ld;
    a.accumulate = accumulate;
    a.words = (((uintptr_t)out | (uintptr_t)(ld * es)) & (uintptr_t)(4 * es - 1)) == 0;
    a.nm = a.nn = a.band = 0;
    return dtype == GVQ_BF16 ? launch_product<unsigned short>(a, st) : launch_product<float>(a, st);
}
