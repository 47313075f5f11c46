// Matrices into 4-bit microscaled blocks and back.
//
// A block is 32 consecutive numbers along the axis that a product will sum over.  Its scale is 2^(floor(log2 amax) - 2), kept as
// the biased exponent in one byte, so that amax lands in [4, 8); each number is divided by it and rounded to the nearest of
// 0, 1/2, 1, 3/2, 2, 3, 4, 6 (ties to the even code, above 6 to 6) with its sign in front.  The conversion instruction does the
// division, the rounding and the saturation; it agrees with that definition on all 65536 bf16 numbers and on fp32 numbers around
// every tie, at scales from the smallest to the largest, so rounding here is exact: nothing is lost but what the format loses.
// Bound: memory, and with random bytes the 20 instructions that each of a number's two roundings takes.  A matrix is read once; both
// directions' blocks come out of the same pass, the columns' ones through LDS.  Rows of 8192 x 4096 bf16 numbers 16.6 us (5.1 TB/s),
// columns of 4096 x 25088 59 (4.4), both ways of 8191 x 4093 fp32 numbers with random bytes 83 (2.5), back into fp32 27 (5.6).
#include "gvq_mx.h"
#include "gvq_tile.h"

#define MXQ_THREADS 256

// ---- rows only -------------------------------------------------------------------------------------------------

// Eight consecutive numbers a thread, four threads a block, so that a wave's loads, codes and scales are all contiguous.
// `words`: rows start at multiples of 16 bytes and so do the random bytes at multiples of 8.  I: the index type (a 64-bit division
// is a hundred instructions, more than all the rest).
template <typename T, bool NOISE, typename I>
__global__ __launch_bounds__(MXQ_THREADS) void mx_rows_kernel(MxQuantArgs a)
{
    const I per = (I)(a.ldc >> 2);   // groups of eight numbers of a row, its padding among them
    const int64_t n = a.rows * (a.ldc >> 2);
    for (int64_t j = (int64_t)blockIdx.x * MXQ_THREADS + threadIdx.x; j < n; j += (int64_t)gridDim.x * MXQ_THREADS) {
        const I i = (I)j, r = i / per, c = (i - r * per) * 8;
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

// A work-group takes 128 rows of 64 columns.  They go into LDS, in 16-byte words where rows are aligned and otherwise one number a
// lane, so that a wave reads 64 neighbours either way (8191 x 4093 numbers, rows of no whole words: eight numbers a lane 114 us).
// Then each thread takes four blocks' quarters along the rows, and one column's 32 numbers, whose 16 bytes of codes stand
// beside those of three other threads.  Work-groups of one XCD take neighbouring tiles: their pieces of 32 bytes of a row of codes
// meet in its L2.
// LDS: a row is 64 words and the columns of rows [32 q, 32 q + 32) are exchanged in groups of 16 (c ^ 16 (q & 3)), so that the
// 4 x 16 (block, column) pairs that a wave reads together lie in 64 different banks.
__device__ __forceinline__ int mx_place(int r, int c) { return r * 64 + (c ^ (16 * (r >> 5 & 3))); }

template <typename T, bool NOISE, bool ROWS>
__global__ __launch_bounds__(MXQ_THREADS) void mx_both_kernel(MxQuantArgs a)
{
    __shared__ __attribute__((aligned(16))) float tile[128 * 64];
    __shared__ __attribute__((aligned(16))) unsigned char dust[NOISE ? 128 * 64 : 16];
    const int t = tile_of_block(blockIdx.x, gridDim.x);
    const int64_t r0 = (int64_t)(t / a.across) * 128, c0 = (int64_t)(t % a.across) * 64;
    const bool whole = r0 + 128 <= a.rows && c0 + 64 <= a.cols;
    if (whole && a.words) {
        constexpr int PER = 16 / sizeof(T), N = 128 * 64 / PER / MXQ_THREADS;
        u4 v[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int e = threadIdx.x + i * MXQ_THREADS, r = e / (64 / PER), c = e % (64 / PER) * PER;
            v[i] = stream_load((const u4*)((const T*)a.x + (r0 + r) * a.ld + c0 + c));
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int e = threadIdx.x + i * MXQ_THREADS, at = mx_place(e / (64 / PER), e % (64 / PER) * PER);
            if constexpr (sizeof(T) == 4) {
                *(u4*)(tile + at) = v[i];
            } else {
                *(u4*)(tile + at) = u4{v[i][0] << 16, v[i][0] & 0xffff0000u, v[i][1] << 16, v[i][1] & 0xffff0000u};
                *(u4*)(tile + at + 4) = u4{v[i][2] << 16, v[i][2] & 0xffff0000u, v[i][3] << 16, v[i][3] & 0xffff0000u};
            }
        }
    } else {
        const int c = threadIdx.x & 63;
        const bool in_c = c0 + c < a.cols;
#pragma unroll 1
        for (int h = 0; h < 2; ++h) {
            float v[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int64_t r = r0 + 64 * h + 4 * i + (threadIdx.x >> 6);
                const T* p = (const T*)a.x + (r < a.rows ? r : a.rows - 1) * a.ld + (in_c ? c0 + c : a.cols - 1);
                if constexpr (sizeof(T) == 4) v[i] = *p;
                else v[i] = bf16_to_f32(*p);
                if (!in_c || r >= a.rows) v[i] = 0.f;
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) tile[mx_place(64 * h + 4 * i + (threadIdx.x >> 6), c)] = v[i];
        }
    }
    if (NOISE) {
        if (whole && a.noise_words) {
            u2 v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int e = threadIdx.x + i * MXQ_THREADS;
                v[i] = *(const u2*)(a.noise + (r0 + (e >> 3)) * a.noise_ld + c0 + 8 * (e & 7));
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int e = threadIdx.x + i * MXQ_THREADS;
                *(u2*)(dust + mx_place(e >> 3, 8 * (e & 7))) = v[i];
            }
        } else {
            const int c = threadIdx.x & 63;
#pragma unroll 1
            for (int h = 0; h < 2; ++h) {
                unsigned char v[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int64_t r = r0 + 64 * h + 4 * i + (threadIdx.x >> 6);
                    v[i] = a.noise[(r < a.rows ? r : a.rows - 1) * a.noise_ld + (c0 + c < a.cols ? c0 + c : a.cols - 1)];
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) dust[mx_place(64 * h + 4 * i + (threadIdx.x >> 6), c)] = v[i];
            }
        }
    }
    __syncthreads();
    if (ROWS) {
        const int g = threadIdx.x & 7, rr = threadIdx.x >> 3;
        const int64_t c = c0 + 8 * g;
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            const int64_t r = r0 + 32 * p + rr;
            const int at = mx_place(32 * p + rr, 8 * g);
            const f4 lo = *(const f4*)(tile + at), hi = *(const f4*)(tile + at + 4);
            const float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
            unsigned int z[2] = {0, 0};
            if (NOISE) {
                const u2 d = *(const u2*)(dust + at);
                z[0] = d[0]; z[1] = d[1];
            }
            const unsigned int top = mx_max_of_4(mx_top8(v));
            const int code = mx_scale_code(top);
            unsigned int q = mx_pack8<NOISE>(v, z, code);
            if (code == 255) q = 0;
            if (r < a.rows && (c >> 1) < a.ldc) {
                *(unsigned int*)(a.codes + r * a.ldc + (c >> 1)) = q;
                if ((g & 3) == 0) a.scales[r * (a.ldc >> 4) + (c >> 5)] = (unsigned char)code;
            }
        }
    }
    const int b = threadIdx.x & 3, cc = threadIdx.x >> 2;
    const int64_t c = c0 + cc;
    const int from = mx_place(32 * b, cc);
    float v[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = tile[from + 64 * i];
    unsigned int top = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const unsigned int u = mx_top8(v + 8 * k);
        top = u > top ? u : top;
    }
    const int code = mx_scale_code(top);
    u4 q;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        unsigned int z[2] = {0, 0};
        if (NOISE)
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i >> 2] |= (unsigned int)dust[from + 64 * (8 * k + i)] << (8 * (i & 3));
        q[k] = code == 255 ? 0 : mx_pack8<NOISE>(v + 8 * k, z, code);
    }
    if (c < a.cols) {
        *(u4*)(a.codes_t + c * a.ldct + (r0 >> 1) + 16 * b) = q;
        a.scales_t[c * (a.ldct >> 4) + (r0 >> 5) + b] = (unsigned char)code;
    }
}

// ---- back -----------------------------------------------------------------------------------------------------------

// Eight numbers a thread.
template <typename T, typename I>
__global__ __launch_bounds__(MXQ_THREADS) void mx_values_kernel(const unsigned char* codes, const unsigned char* scales, int64_t ldc,
                                                               int64_t rows, int64_t cols, T* out, int64_t ld, int words)
{
    const I per = (I)((cols + 7) >> 3);
    const int64_t n = rows * ((cols + 7) >> 3);
    for (int64_t j = (int64_t)blockIdx.x * MXQ_THREADS + threadIdx.x; j < n; j += (int64_t)gridDim.x * MXQ_THREADS) {
        const I i = (I)j, r = i / per, g = i - r * per;
        const unsigned int q = *(const unsigned int*)(codes + r * ldc + 4 * g);
        float v[8];
        mx_unpack8(q, scales[r * (ldc >> 4) + (g >> 2)], v);
        mx_store8(out + r * ld + 8 * g, words != 0, cols - 8 * (int64_t)g, v);
    }
}

// Rows that are not aligned to 16 bytes: a wave takes 512 columns, eight codes a lane, and hands them round so that each store is of
// 64 neighbours (8191 x 4093 numbers in fp32: eight numbers a lane 87 us).
template <typename T>
__global__ __launch_bounds__(MXQ_THREADS) void mx_values_odd_kernel(const unsigned char* codes, const unsigned char* scales, int64_t ldc,
                                                                   int64_t rows, int64_t cols, T* out, int64_t ld)
{
    const int lane = threadIdx.x & 63;
    const int64_t c0 = (int64_t)blockIdx.x * 512, g = c0 / 8 + lane;
    const bool in = 4 * g < ldc;
    for (int64_t r = (int64_t)blockIdx.y * (MXQ_THREADS / 64) + (threadIdx.x >> 6); r < rows; r += (int64_t)gridDim.y * (MXQ_THREADS / 64)) {
        const unsigned int q = in ? *(const unsigned int*)(codes + r * ldc + 4 * g) : 0u;
        const int k = in ? scales[r * (ldc >> 4) + (g >> 2)] : 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int from = 8 * i + (lane >> 3);
            const unsigned int code = (unsigned int)__shfl((int)q, from) >> (4 * (lane & 7)) & 15u;
            const float v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, mx_scale(__shfl(k, from)), 0)[0];
            const int64_t c = c0 + 64 * i + lane;
            if (c < cols) {
                if constexpr (sizeof(T) == 2) out[r * ld + c] = (T)f32_to_bf16_rne(v);
                else out[r * ld + c] = v;
            }
        }
    }
}

template <typename T>
static int launch_quantize(MxQuantArgs a, hipStream_t st)
{
    const dim3 threads(MXQ_THREADS);
    if (!a.codes_t) {
        const int64_t n = a.rows * (a.ldc >> 2), g = (n + MXQ_THREADS - 1) / MXQ_THREADS;
        const dim3 grid((unsigned)(g < 4096 ? g : 4096));
        const bool small = n <= 0x7fffffff;
        if (a.noise && small) hipLaunchKernelGGL((mx_rows_kernel<T, true, unsigned int>), grid, threads, 0, st, a);
        else if (a.noise) hipLaunchKernelGGL((mx_rows_kernel<T, true, int64_t>), grid, threads, 0, st, a);
        else if (small) hipLaunchKernelGGL((mx_rows_kernel<T, false, unsigned int>), grid, threads, 0, st, a);
        else hipLaunchKernelGGL((mx_rows_kernel<T, false, int64_t>), grid, threads, 0, st, a);
    } else {
        // tiles behind the last column write the padding of the rows' codes
        a.across = (int)(a.codes ? a.ldc >> 5 : (a.cols + 63) >> 6);
        const int64_t tiles = a.across * ((a.rows + 127) >> 7);
        if (tiles > 0x7fffffff) return GVQ_EINVAL;
        const dim3 grid((unsigned)tiles);
        if (a.noise && a.codes) hipLaunchKernelGGL((mx_both_kernel<T, true, true>), grid, threads, 0, st, a);
        else if (a.noise) hipLaunchKernelGGL((mx_both_kernel<T, true, false>), grid, threads, 0, st, a);
        else if (a.codes) hipLaunchKernelGGL((mx_both_kernel<T, false, true>), grid, threads, 0, st, a);
        else hipLaunchKernelGGL((mx_both_kernel<T, false, false>), grid, threads, 0, st, a);
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

template <typename T>
static int launch_dequantize(const unsigned char* codes, const unsigned char* scales, int64_t rows, int64_t cols, T* out, int64_t ld,
                             hipStream_t st)
{
    const int64_t ldc = gvq_mx_row_bytes(cols), n = rows * ((cols + 7) >> 3), g = (n + MXQ_THREADS - 1) / MXQ_THREADS;
    const int words = (((uintptr_t)out | (uintptr_t)(ld * (int64_t)sizeof(T))) & 15) == 0;
    const dim3 grid((unsigned)(g < 4096 ? g : 4096)), threads(MXQ_THREADS);
    if (!words && cols >= 256) {
        const int64_t down = (rows + 3) / 4;
        hipLaunchKernelGGL((mx_values_odd_kernel<T>), dim3((unsigned)((cols + 511) / 512), (unsigned)(down < 4096 ? down : 4096)), threads, 0, st,
                           codes, scales, ldc, rows, cols, out, ld);
    } else if (n <= 0x7fffffff) {
        hipLaunchKernelGGL((mx_values_kernel<T, unsigned int>), grid, threads, 0, st, codes, scales, ldc, rows, cols, out, ld, words);
    } else {
        hipLaunchKernelGGL((mx_values_kernel<T, int64_t>), grid, threads, 0, st, codes, scales, ldc, rows, cols, out, ld, words);
    }
    GVQ_HIP(hipGetLastError());
    return GVQ_OK;
}

int gvq_launch_mx_dequantize(const void* codes, const void* scales, int64_t rows, int64_t cols, void* out, gvq_dtype_t dtype,
                             int64_t ld, hipStream_t st)
{
    const unsigned char *q = (const unsigned char*)codes, *s = (const unsigned char*)scales;
    return dtype == GVQ_BF16 ? launch_dequantize(q, s, rows, cols, (unsigned short*)out, ld, st)
                             : launch_dequantize(q, s, rows, cols, (float*)out, ld, st);
}
