// Products of 4-bit microscaled matrices, C = A B^T, on the scaled 4-bit matrix pipe (v_mfma_scale_f32_16x16x128_f8f6f4: exact
// products of codes, scaled per block of 32, fp32 sums).  8192 x 4096 x 4096 into bf16 80 to 88 us (3.1 to 3.4 PFLOP/s), 4096 x 25088 x 4096 into bf16
// 259 to 275, into fp32 308 to 315 (411 MB of results, 80 us alone), by the box.  A round of 256 x 256 tiles costs 8 us beside its steps, most of it
// results that all compute units write at one time.
#include "gvq_mx.h"
#include "gvq_mx_plan.h"
#include "gvq_tile.h"

struct MxProductArgs {
    TileOperand a, b;
    int steps;         // of 128 numbers
    int nm, nn, band;  // tiles, and how they are swept
    void* out;
    int64_t ld;
    int accumulate, words;   // words: rows are aligned to 16 bytes
};

// A wave hands its results out through its share of LDS, so that rows leave in 16-byte words side by side: straight from the
// accumulators they would leave in pieces of 32 or 64 bytes, 16 rows at a time.  Rows are padded by one word; fp32 results go in
// two halves.
template <typename T, typename OUT>
struct MxOut {
    static constexpr int R = T::BM / T::WM / (sizeof(OUT) / 2), C = T::BN / T::WN, PAD = 16 / sizeof(OUT), LD = C + PAD;
    static constexpr int WAVE = R * LD * sizeof(OUT), ALL = T::WAVES * WAVE;
    static constexpr int LDS = T::LDS > ALL ? T::LDS : ALL;
    static_assert(LDS <= 160 * 1024 && WAVE % 16 == 0 && R % 16 == 0, "LDS of a compute unit; whole fragments");
};

__device__ __forceinline__ void mx_lds4(float* p, f4 v) { *(f4*)p = v; }
__device__ __forceinline__ void mx_lds4(unsigned short* p, f4 v) { *(u2*)p = u2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])}; }

template <typename T, typename OUT>
__global__ __launch_bounds__(T::THREADS) void mx_tile_kernel(MxProductArgs a)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    int tm, tn;
    tile_at(tile_of_block(blockIdx.x, a.nm * a.nn), a.nm, a.nn, a.band, tm, tn);
    f4 acc[T::MI][T::NI];
#pragma unroll
    for (int mi = 0; mi < T::MI; ++mi)
#pragma unroll
        for (int ni = 0; ni < T::NI; ++ni) acc[mi][ni] = f4{0.f, 0.f, 0.f, 0.f};
    tile_product<T>(a.a, a.b, tm * T::BM, tn * T::BN, 0, a.steps, lds, acc);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int r0 = tm * T::BM + wave / T::WN * (T::BM / T::WM), c0 = tn * T::BN + wave % T::WN * (T::BN / T::WN);
    OUT* out = (OUT*)a.out;
    if (a.words && !a.accumulate) {
        typedef MxOut<T, OUT> O;
        constexpr int FRAGS = O::R / 16, PER = 16 / sizeof(OUT), LANES = O::C / PER;   // lanes of a row
        OUT* w = (OUT*)(lds + wave * O::WAVE);
        __syncthreads();
        static_for<0, T::MI / FRAGS>([&](auto half) {
            constexpr int H = decltype(half)::value * FRAGS;
#pragma unroll
            for (int mi = 0; mi < FRAGS; ++mi)
#pragma unroll
                for (int ni = 0; ni < T::NI; ++ni) mx_lds4(w + (16 * mi + (lane & 15)) * O::LD + 16 * ni + 4 * (lane >> 4), acc[H + mi][ni]);
            wave_lds_sync();
#pragma unroll
            for (int i = 0; i < O::R * LANES / 64; ++i) {
                const int e = lane + 64 * i, r = e / LANES, c = e % LANES * PER, left = a.b.rows - (c0 + c);
                if (r0 + 16 * H + r >= a.a.rows) continue;
                const u4 v = *(const u4*)(w + r * O::LD + c);
                OUT* to = out + (int64_t)(r0 + 16 * H + r) * a.ld + c0 + c;
                if (left >= PER) *(u4*)to = v;
                else
#pragma unroll
                    for (int k = 0; k < PER; ++k)
                        if (k < left) to[k] = w[r * O::LD + c + k];
            }
            wave_lds_sync();
        });
        return;
    }
#pragma unroll
    for (int mi = 0; mi < T::MI; ++mi) {
        const int r = r0 + 16 * mi + (lane & 15);
        if (r >= a.a.rows) continue;
#pragma unroll
        for (int ni = 0; ni < T::NI; ++ni) {
            const int c = c0 + 16 * ni + 4 * (lane >> 4);
            mx_store4(out + (int64_t)r * a.ld + c, a.words != 0, a.b.rows - c, a.accumulate != 0, acc[mi][ni]);
        }
    }
}

template <typename T, typename OUT>
static int launch_tile(MxProductArgs a, hipStream_t st)
{
    a.nm = (a.a.rows + T::BM - 1) / T::BM;
    a.nn = (a.b.rows + T::BN - 1) / T::BN;
    if ((int64_t)a.nm * a.nn > 0x7fffffff) return GVQ_EINVAL;
    a.band = 4;
    constexpr int LDS = MxOut<T, OUT>::LDS;
    static gvq_once_per_device lds;
    int dev;
    GVQ_HIP(hipGetDevice(&dev));
    const int rc = lds.call(dev, [] {
        GVQ_HIP(hipFuncSetAttribute((const void*)mx_tile_kernel<T, OUT>, hipFuncAttributeMaxDynamicSharedMemorySize, LDS));
        return (int)GVQ_OK;
    });
    if (rc != GVQ_OK) return rc;
    hipLaunchKernelGGL((mx_tile_kernel<T, OUT>), dim3(a.nm * a.nn), dim3(T::THREADS), LDS, st, a);
    GVQ_HIP(hipGetLastError());
    return GVQ_OK;
}

template <typename OUT>
static int launch_product(const MxProductArgs& a, int shape, hipStream_t st)
{
    switch (shape) {
    case 0: return launch_tile<TileShape<256, 256, 2, 4, 1, 4>, OUT>(a, st);
    case 1: return launch_tile<TileShape<256, 128, 4, 2, 1, 4>, OUT>(a, st);
    case 2: return launch_tile<TileShape<128, 128, 2, 4, 1, 4>, OUT>(a, st);
    case 3: return launch_tile<TileShape<64, 64, 2, 2, 1, 4>, OUT>(a, st);
    default: return launch_tile<TileShape<64, 64, 2, 2, 1, 4, false, false, true>, OUT>(a, st);
    }
}

double gvq_mx_product_time(int64_t m, int64_t n, int64_t k) { return mx_way(m, n, gvq_mx_row_bytes(k) / TILE_STEP).us; }

int gvq_launch_mx_matmul(const void* a_codes, const void* a_scales, const void* b_codes, const void* b_scales, int64_t m, int64_t n,
                         int64_t k, void* out, gvq_dtype_t dtype, int64_t ld, bool accumulate, hipStream_t st)
{
    const int64_t row = gvq_mx_row_bytes(k), es = dtype == GVQ_BF16 ? 2 : 4, steps = row / TILE_STEP;
    const MxWay way = steps > 0 ? mx_way(m, n, steps) : mx_tiles(m, n, steps);
    if (way.few)
        return gvq_launch_mx_few(way.few, a_codes, a_scales, b_codes, b_scales, m, n, k, out, dtype, ld, accumulate, st);
    MxProductArgs a;
    a.a = TileOperand{(const char*)a_codes, 0, row, (int)m, (const char*)a_scales, 0};
    a.b = TileOperand{(const char*)b_codes, 0, row, (int)n, (const char*)b_scales, 0};
    a.steps = (int)steps;
    a.out = out;
    a.ld = ld;
    a.accumulate = accumulate;
    a.words = (((uintptr_t)out | (uintptr_t)(ld * es)) & 15) == 0;
    a.nm = a.nn = a.band = 0;
    return dtype == GVQ_BF16 ? launch_product<unsigned short>(a, way.shape, st) : launch_product<float>(a, way.shape, st);
}
