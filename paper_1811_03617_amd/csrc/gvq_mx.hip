// Matrices into 4-bit microscaled blocks and back.
//
// A block is 32 consecutive numbers along the axis that a product will sum over.  Its scale is 2^(floor(log2 amax) - 2), kept as
// the biased exponent in one byte, so that amax lands in [4, 8); each number is divided by it and rounded to the nearest of
// 0, 1/2, 1, 3/2, 2, 3, 4, 6 (ties to the even code, above 6 to 6) with its sign in front.  The conversion instruction does the
// division, the rounding and the saturation; it agrees with that definition on all 65536 bf16 numbers and on fp32 numbers around
// every tie, at scales from the smallest to the largest, so rounding here is exact: nothing is lost but what the format loses.
// Bound: memory.  A matrix is read once; both directions' blocks come out of the same pass, the columns' ones through LDS.
#include "gvq_mx.h"

#define MXQ_THREADS 256

// ---- rows only -------------------------------------------------------------------------------------------------

// Eight consecutive numbers a thread, four threads a block, so that a wave's loads, codes and scales are all contiguous.
// `words`: rows start at multiples of 16 bytes (32 for fp32) and so do the random bytes at multiples of 8.
template <typename T, bool NOISE>
__global__ __launch_bounds__(MXQ_THREADS) void mx_rows_kernel(MxQuantArgs a)
{
    const int64_t per = a.ldc >> 2;   // groups of eight numbers of a row, its padding among them
    const int64_t n = a.rows * per;
    for (int64_t i = (int64_t)blockIdx.x * MXQ_THREADS + threadIdx.x; i < n; i += (int64_t)gridDim.x * MXQ_THREADS) {
        const int64_t r = i / per, c = (i - r * per) * 8;
        float v[8];
        mx_load8((const T*)a.x + r * a.ld + c, a.words != 0, a.cols - c, v);
        unsigned int z[2] = {0, 0};
        if (NOISE) mx_noise8(a.noise + r * a.noise_ld + c, a.noise_words != 0, a.cols - c, z);
        // n and the stride are multiples of 4: the four threads of a block are here together
        const unsigned int top = mx_max_of_4(mx_top8(v));
        const int code = mx_scale_code(top);
        unsigned int q = mx_pack8<NOISE>(v, z, code);
        if (code == 255) q = 0;
        ((unsigned int*)a.codes)[i] = q;
        if ((threadIdx.x & 3) == 0) a.scales[i >> 2] = (unsigned char)code;
    }
}

// ---- rows and columns ---------------------------------------------------------------------------------------------

// A work-group takes 128 rows of 64 columns.  Each thread reads eight numbers of a row at a time, packs the rows' blocks as above
// and leaves the numbers (and random bytes) in LDS; then it takes one column's 32 numbers, two such blocks in all, and writes their
// 16 bytes, four threads side by side 64 bytes of a column's row of codes.
// LDS: a row is 64 words and the columns of rows [32 q, 32 q + 32) are exchanged in groups of 16 (c ^ 16 (q & 3)), so that the
// 4 x 16 (block, column) pairs that a wave reads together lie in 64 different banks.
template <typename T, bool NOISE, bool ROWS>
__global__ __launch_bounds__(MXQ_THREADS) void mx_both_kernel(MxQuantArgs a)
{
    __shared__ float tile[128 * 64];
    __shared__ unsigned char dust[NOISE ? 128 * 64 : 16];
    const int64_t r0 = (int64_t)blockIdx.y * 128, c0 = (int64_t)blockIdx.x * 64;
    const int g = threadIdx.x & 7, rr = threadIdx.x >> 3;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const int lr = 32 * p + rr;
        const int64_t r = r0 + lr, c = c0 + 8 * g;
        const bool in = r < a.rows;
        float v[8];
        mx_load8((const T*)a.x + (in ? r : a.rows - 1) * a.ld + c, a.words != 0, a.cols - c, v);
        unsigned int z[2] = {0, 0};
        if (NOISE) mx_noise8(a.noise + (in ? r : a.rows - 1) * a.noise_ld + c, a.noise_words != 0, a.cols - c, z);
        if (!in)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = 0.f;
        if (ROWS) {
            const unsigned int top = mx_max_of_4(mx_top8(v));
            const int code = mx_scale_code(top);
            unsigned int q = mx_pack8<NOISE>(v, z, code);
            if (code == 255) q = 0;
            if (in && (c >> 1) < a.ldc) {
                *(unsigned int*)(a.codes + r * a.ldc + (c >> 1)) = q;
                if ((g & 3) == 0) a.scales[r * (a.ldc >> 4) + (c >> 5)] = (unsigned char)code;
            }
        }
        const int at = lr * 64 + ((8 * g) ^ (16 * (p & 3)));
        *(f4*)(tile + at) = f4{v[0], v[1], v[2], v[3]};
        *(f4*)(tile + at + 4) = f4{v[4], v[5], v[6], v[7]};
        if (NOISE) *(u2*)(dust + at) = u2{z[0], z[1]};
    }
    __syncthreads();
    const int b = threadIdx.x & 3, cc = threadIdx.x >> 2;
    const int64_t c = c0 + cc;
    const float* from = tile + 32 * b * 64 + (cc ^ (16 * b));
    const unsigned char* zfrom = dust + (NOISE ? 32 * b * 64 + (cc ^ (16 * b)) : 0);
    float v[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = from[64 * i];
    unsigned int top = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const unsigned int t = mx_top8(v + 8 * k);
        top = t > top ? t : top;
    }
    const int code = mx_scale_code(top);
    u4 q;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        unsigned int z[2] = {0, 0};
        if (NOISE)
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i >> 2] |= (unsigned int)zfrom[64 * (8 * k + i)] << (8 * (i & 3));
        q[k] = code == 255 ? 0 : mx_pack8<NOISE>(v + 8 * k, z, code);
    }
    if (c < a.cols) {
        *(u4*)(a.codes_t + c * a.ldct + (r0 >> 1) + 16 * b) = q;
        a.scales_t[c * (a.ldct >> 4) + (r0 >> 5) + b] = (unsigned char)code;
    }
}

// ---- back -----------------------------------------------------------------------------------------------------------

template <typename T>
__global__ __launch_bounds__(MXQ_THREADS) void mx_values_kernel(const unsigned char* codes, const unsigned char* scales, int64_t ldc,
                                                               int64_t rows, int64_t cols, T* out, int64_t ld, int words)
{
    const int64_t per = (cols + 7) >> 3, n = rows * per;
    for (int64_t i = (int64_t)blockIdx.x * MXQ_THREADS + threadIdx.x; i < n; i += (int64_t)gridDim.x * MXQ_THREADS) {
        const int64_t r = i / per, g = i - r * per;
        const unsigned int q = *(const unsigned int*)(codes + r * ldc + 4 * g);
        float v[8];
        mx_unpack8(q, scales[r * (ldc >> 4) + (g >> 2)], v);
        mx_store8(out + r * ld + 8 * g, words != 0, cols - 8 * g, v);
    }
}

template <typename T>
static int launch_quantize(const MxQuantArgs& a, hipStream_t st)
{
    if (!a.codes_t) {
        const int64_t n = a.rows * (a.ldc >> 2), g = (n + MXQ_THREADS - 1) / MXQ_THREADS;
        const dim3 grid((unsigned)(g < 4096 ? g : 4096));
        if (a.noise) hipLaunchKernelGGL((mx_rows_kernel<T, true>), grid, dim3(MXQ_THREADS), 0, st, a);
        else hipLaunchKernelGGL((mx_rows_kernel<T, false>), grid, dim3(MXQ_THREADS), 0, st, a);
    } else {
        // tiles behind the last column write the padding of the rows' codes
        const dim3 grid((unsigned)(a.codes ? a.ldc >> 5 : (a.cols + 63) >> 6), (unsigned)((a.rows + 127) >> 7));
        if (a.noise && a.codes) hipLaunchKernelGGL((mx_both_kernel<T, true, true>), grid, dim3(MXQ_THREADS), 0, st, a);
        else if (a.noise) hipLaunchKernelGGL((mx_both_kernel<T, true, false>), grid, dim3(MXQ_THREADS), 0, st, a);
        else if (a.codes) hipLaunchKernelGGL((mx_both_kernel<T, false, true>), grid, dim3(MXQ_THREADS), 0, st, a);
        else hipLaunchKernelGGL((mx_both_kernel<T, false, false>), grid, dim3(MXQ_THREADS), 0, st, a);
    }
    GVQ_HIP(hipGetLastError());
    return GVQ_OK;
}

int gvq_launch_mx_quantize(MxQuantArgs a, gvq_dtype_t dtype, hipStream_t st)
{
    const int64_t es = dtype == GVQ_BF16 ? 2 : 4;
    a.ldc = gvq_mx_row_bytes(a.cols);
    a.ldct = gvq_mx_row_bytes(a.rows);
    a.words = (((uintptr_t)a.x | (uintptr_t)(a.ld * es)) & 15) == 0;
    a.noise_words = (((uintptr_t)a.noise | (uintptr_t)a.noise_ld) & 7) == 0;
    return dtype == GVQ_BF16 ? launch_quantize<unsigned short>(a, st) : launch_quantize<float>(a, st);
}

int gvq_launch_mx_dequantize(const void* codes, const void* scales, int64_t rows, int64_t cols, void* out, gvq_dtype_t dtype,
                             int64_t ld, hipStream_t st)
{
    const int64_t n = rows * ((cols + 7) >> 3), g = (n + MXQ_THREADS - 1) / MXQ_THREADS;
    const dim3 grid((unsigned)(g < 4096 ? g : 4096));
    const int64_t es = dtype == GVQ_BF16 ? 2 : 4;
    const int words = (((uintptr_t)out | (uintptr_t)(ld * es)) & 15) == 0;
    const int64_t ldc = gvq_mx_row_bytes(cols);
    if (dtype == GVQ_BF16)
        hipLaunchKernelGGL((mx_values_kernel<unsigned short>), grid, dim3(MXQ_THREADS), 0, st, (const unsigned char*)codes,
                           (const unsigned char*)scales, ldc, rows, cols, (unsigned short*)out, ld, words);
    else
        hipLaunchKernelGGL((mx_values_kernel<float>), grid, dim3(MXQ_THREADS), 0, st, (const unsigned char*)codes,
                           (const unsigned char*)scales, ldc, rows, cols, (float*)out, ld, words);
    GVQ_HIP(hipGetLastError());
    return GVQ_OK;
}
