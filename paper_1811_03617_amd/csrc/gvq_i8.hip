// Matrices into 8-bit integers with a scale for every row, of the matrix or of its transpose, and back.
//
// Rows: one pass, a row's numbers stay in registers between its largest magnitude and its codes.  Columns: their largest magnitudes
// first, in runs of rows that work-groups take side by side, then their codes, turned through LDS.
// Bound: memory; columns read the matrix twice.
#include "gvq_i8.h"
#include "gvq_tile.h"

#define I8Q_THREADS 256

__device__ __forceinline__ unsigned int wave_max(unsigned int v)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const unsigned int o = (unsigned int)__shfl_xor((int)v, d);
        v = o > v ? o : v;
    }
    return v;
}

// ---- rows -------------------------------------------------------------------------------------------------------

// A row to W waves, eight neighbouring numbers a thread at a time, HOLD times eight in registers; what is behind that is read again.
template <typename T, int W>
__global__ __launch_bounds__(W > 4 ? 64 * W : I8Q_THREADS) void i8_rows_kernel(I8QuantArgs a)
{
    constexpr int HOLD = 4, PER = W > 4 ? 1 : 4 / W, T_ROW = 64 * W;
    __shared__ unsigned int part[W > 4 ? W : 4];
    const int t = threadIdx.x % T_ROW;
    const int64_t r = (int64_t)blockIdx.x * PER + threadIdx.x / T_ROW;
    if (W == 1 && r >= a.rows) return;
    const T* x = (const T*)a.x + r * a.ld;
    const int chunks = (int)(a.ldc >> 3);
    float v[HOLD][8];
    unsigned int top = 0;
#pragma unroll
    for (int i = 0; i < HOLD; ++i) {
        const int c = t + i * T_ROW;
        if (c < chunks) {
            mx_load8(x + 8 * (int64_t)c, a.words != 0, a.cols - 8 * (int64_t)c, v[i]);
            const unsigned int u = mx_top8(v[i]);
            top = u > top ? u : top;
        }
    }
    for (int c = t + HOLD * T_ROW; c < chunks; c += T_ROW) {
        float f[8];
        mx_load8(x + 8 * (int64_t)c, a.words != 0, a.cols - 8 * (int64_t)c, f);
        const unsigned int u = mx_top8(f);
        top = u > top ? u : top;
    }
    top = wave_max(top);
    if constexpr (W > 1) {
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) part[wave] = top;
        __syncthreads();
        const int first = wave / W * W;
#pragma unroll
        for (int i = 0; i < W; ++i) top = part[first + i] > top ? part[first + i] : top;
    }
    const I8Scale s = i8_scale(top);
    const unsigned int keep = top >= 0x7f800000u ? 0u : ~0u;
    signed char* q = a.codes + r * a.ldc;
#pragma unroll
    for (int i = 0; i < HOLD; ++i) {
        const int c = t + i * T_ROW;
        if (c < chunks)
            *(u2*)(q + 8 * (int64_t)c) = u2{i8_pack4(v[i][0], v[i][1], v[i][2], v[i][3], s.up) & keep,
                                             i8_pack4(v[i][4], v[i][5], v[i][6], v[i][7], s.up) & keep};
    }
    for (int c = t + HOLD * T_ROW; c < chunks; c += T_ROW) {
        float f[8];
        mx_load8(x + 8 * (int64_t)c, a.words != 0, a.cols - 8 * (int64_t)c, f);
        *(u2*)(q + 8 * (int64_t)c) = u2{i8_pack4(f[0], f[1], f[2], f[3], s.up) & keep, i8_pack4(f[4], f[5], f[6], f[7], s.up) & keep};
    }
    if (t == 0) a.scales[r] = s.down;
}

// ---- columns ------------------------------------------------------------------------------------------------------

// Largest magnitudes of a run of rows: a work-group takes 64 lanes' words of columns, its waves every fourth row.
template <typename T>
__global__ __launch_bounds__(I8Q_THREADS) void i8_peaks_kernel(I8QuantArgs a)
{
    constexpr int PER = 16 / sizeof(T);
    __shared__ unsigned int part[4][64][PER + 1];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t c = ((int64_t)blockIdx.x * 64 + lane) * PER, r0 = (int64_t)blockIdx.y * a.chunk_rows;
    const int64_t r1 = r0 + a.chunk_rows < a.rows ? r0 + a.chunk_rows : a.rows;
    unsigned int top[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) top[i] = 0;
    if (c < a.cols) {
        const T* x = (const T*)a.x + c;
        if (a.words && c + PER <= a.cols) {
#pragma unroll 4
            for (int64_t r = r0 + wave; r < r1; r += 4) {
                const u4 v = *(const u4*)(x + r * a.ld);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if constexpr (sizeof(T) == 4) {
                        const unsigned int u = v[i] & 0x7fffffffu;
                        top[i] = u > top[i] ? u : top[i];
                    } else {
                        const unsigned int lo = v[i] << 16 & 0x7fffffffu, hi = v[i] & 0x7fff0000u;
                        top[2 * i] = lo > top[2 * i] ? lo : top[2 * i];
                        top[2 * i + 1] = hi > top[2 * i + 1] ? hi : top[2 * i + 1];
                    }
                }
            }
        } else {
            for (int64_t r = r0 + wave; r < r1; r += 4)
#pragma unroll
                for (int i = 0; i < PER; ++i)
                    if (c + i < a.cols) {
                        unsigned int u;
                        if constexpr (sizeof(T) == 4) u = __float_as_uint(x[r * a.ld + i]) & 0x7fffffffu;
                        else u = ((unsigned int)x[r * a.ld + i] & 0x7fffu) << 16;
                        top[i] = u > top[i] ? u : top[i];
                    }
        }
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) part[wave][lane][i] = top[i];
    __syncthreads();
    for (int e = threadIdx.x; e < 64 * PER; e += I8Q_THREADS) {
        const int64_t cc = (int64_t)blockIdx.x * 64 * PER + e;
        if (cc >= a.cols) break;
        unsigned int m = 0;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const unsigned int u = part[w][e / PER][e % PER];
            m = u > m ? u : m;
        }
        a.peaks[(int64_t)blockIdx.y * a.cols + cc] = m;
    }
}

// 128 rows of 64 columns: a thread takes four rows of one word of columns, packs each column's four codes, and the tile leaves as
// 128 bytes of each column.  In LDS a column is eight pieces of 16 bytes, exchanged by the column's group of eight.
template <typename T>
__global__ __launch_bounds__(I8Q_THREADS) void i8_columns_kernel(I8QuantArgs a)
{
    constexpr int PER = 16 / sizeof(T), WORDS = 64 / PER, QUADS = I8Q_THREADS / WORDS;   // words of a row; quads of rows at a time
    __shared__ __attribute__((aligned(16))) unsigned int turn[64 * 32];
    __shared__ float ups[64];
    __shared__ unsigned int keeps[64];
    const int64_t tile = tile_of_block(blockIdx.x, gridDim.x);
    const int64_t r0 = tile / a.across * 128, c0 = tile % a.across * 64;
    if (threadIdx.x < 64) {
        const int64_t c = c0 + threadIdx.x;
        unsigned int top = 0;
        if (c < a.cols)
            for (int k = 0; k < a.chunks; ++k) {
                const unsigned int u = a.peaks[(int64_t)k * a.cols + c];
                top = u > top ? u : top;
            }
        const I8Scale s = i8_scale(top);
        ups[threadIdx.x] = s.up;
        keeps[threadIdx.x] = top >= 0x7f800000u ? 0u : ~0u;
        if (r0 == 0 && c < a.cols) a.scales_t[c] = s.down;
    }
    __syncthreads();
    const int w = threadIdx.x % WORDS, quad0 = threadIdx.x / WORDS;
    const int64_t c = c0 + w * PER;
    float up[PER];
    unsigned int keep[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) { up[i] = ups[w * PER + i]; keep[i] = keeps[w * PER + i]; }
#pragma unroll
    for (int p = 0; p < 32 / QUADS; ++p) {
        const int quad = quad0 + p * QUADS;
        float v[4][PER];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int64_t r = r0 + 4 * quad + k;
            const T* x = (const T*)a.x + r * a.ld + c;
            if (r < a.rows && a.words && c + PER <= a.cols) {
                const u4 u = *(const u4*)x;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if constexpr (sizeof(T) == 4) v[k][i] = __uint_as_float(u[i]);
                    else { v[k][2 * i] = __uint_as_float(u[i] << 16); v[k][2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
                }
            } else {
#pragma unroll
                for (int i = 0; i < PER; ++i) {
                    v[k][i] = 0.f;
                    if (r < a.rows && c + i < a.cols) {
                        if constexpr (sizeof(T) == 4) v[k][i] = x[i];
                        else v[k][i] = bf16_to_f32(x[i]);
                    }
                }
            }
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int col = w * PER + i;
            turn[col * 32 + ((quad >> 2 ^ (col >> 3)) << 2) + (quad & 3)] = i8_pack4(v[0][i], v[1][i], v[2][i], v[3][i], up[i]) & keep[i];
        }
    }
    __syncthreads();
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        const int e = threadIdx.x + p * I8Q_THREADS, col = e >> 3, piece = e & 7;
        if (c0 + col < a.cols)
            *(u4*)(a.codes_t + (c0 + col) * a.ldct + r0 + 16 * piece) = *(const u4*)(turn + col * 32 + ((piece ^ (col >> 3)) << 2));
    }
}

// ---- back ---------------------------------------------------------------------------------------------------------

template <typename T>
__global__ __launch_bounds__(I8Q_THREADS) void i8_values_kernel(const signed char* codes, const float* scales, int64_t ldc, int64_t rows,
                                                                int64_t cols, T* out, int64_t ld, int words)
{
    const int64_t per = (cols + 7) >> 3, n = rows * per;
    for (int64_t j = (int64_t)blockIdx.x * I8Q_THREADS + threadIdx.x; j < n; j += (int64_t)gridDim.x * I8Q_THREADS) {
        const int64_t r = j / per, g = j - r * per;
        const u2 q = *(const u2*)(codes + r * ldc + 8 * g);
        const float s = scales[r];
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (float)(signed char)(q[i >> 2] >> (8 * (i & 3))) * s;
        mx_store8(out + r * ld + 8 * g, words != 0, cols - 8 * g, v);
    }
}

template <typename T>
static int launch_quantize(I8QuantArgs a, hipStream_t st)
{
    if (a.codes) {
        // the fewest waves whose registers hold a row
        if (a.ldc <= 2048)
            hipLaunchKernelGGL((i8_rows_kernel<T, 1>), dim3((unsigned)((a.rows + 3) / 4)), dim3(I8Q_THREADS), 0, st, a);
        else if (a.ldc <= 8192)
            hipLaunchKernelGGL((i8_rows_kernel<T, 4>), dim3((unsigned)a.rows), dim3(I8Q_THREADS), 0, st, a);
        else
            hipLaunchKernelGGL((i8_rows_kernel<T, 16>), dim3((unsigned)a.rows), dim3(1024), 0, st, a);
        GVQ_HIP(hipGetLastError());
    }
    if (a.codes_t) {
        constexpr int PER = 16 / sizeof(T);
        a.chunk_rows = gvq_i8_chunk_rows(a.rows);
        a.chunks = (int)((a.rows + a.chunk_rows - 1) / a.chunk_rows);
        a.across = (int)((a.cols + 63) >> 6);
        const int64_t tiles = a.across * (a.ldct >> 7);
        if (tiles > 0x7fffffff) return GVQ_EINVAL;
        hipLaunchKernelGGL((i8_peaks_kernel<T>), dim3((unsigned)((a.cols + 64 * PER - 1) / (64 * PER)), (unsigned)a.chunks), dim3(I8Q_THREADS), 0,
                           st, a);
        GVQ_HIP(hipGetLastError());
        hipLaunchKernelGGL((i8_columns_kernel<T>), dim3((unsigned)tiles), dim3(I8Q_THREADS), 0, st, a);
        GVQ_HIP(hipGetLastError());
    }
    return GVQ_OK;
}

int gvq_launch_i8_quantize(I8QuantArgs a, gvq_dtype_t dtype, hipStream_t st)
{
    const int64_t es = dtype == GVQ_BF16 ? 2 : 4;
    a.ldc = gvq_i8_row_bytes(a.cols);
    a.ldct = gvq_i8_row_bytes(a.rows);
    a.words = (((uintptr_t)a.x | (uintptr_t)(a.ld * es)) & 15) == 0;
    return dtype == GVQ_BF16 ? launch_quantize<unsigned short>(a, st) : launch_quantize<float>(a, st);
}

int gvq_launch_i8_dequantize(const void* codes, const void* scales, int64_t rows, int64_t cols, void* out, gvq_dtype_t dtype, int64_t ld,
                             hipStream_t st)
{
    const int64_t n = rows * ((cols + 7) >> 3), g = (n + I8Q_THREADS - 1) / I8Q_THREADS, es = dtype == GVQ_BF16 ? 2 : 4;
    const int words = (((uintptr_t)out | (uintptr_t)(ld * es)) & 15) == 0;
    const dim3 grid((unsigned)(g < 4096 ? g : 4096));
    if (dtype == GVQ_BF16)
        hipLaunchKernelGGL((i8_values_kernel<unsigned short>), grid, dim3(I8Q_THREADS), 0, st, (const signed char*)codes, (const float*)scales,
                           gvq_i8_row_bytes(cols), rows, cols, (unsigned short*)out, ld, words);
    else
        hipLaunchKernelGGL((i8_values_kernel<float>), grid, dim3(I8Q_THREADS), 0, st, (const signed char*)codes, (const float*)scales,
                           gvq_i8_row_bytes(cols), rows, cols, (float*)out, ld, words);
    GVQ_HIP(hipGetLastError());
    return GVQ_OK;
}
