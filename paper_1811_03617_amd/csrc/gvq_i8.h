// Matrices in 8-bit integers with a scale for every row: device helpers and the launchers' declarations.
#pragma once
#include "gvq_mx.h"

// Bytes of one row of codes: a whole number of 128 columns, zeros behind the last one.
inline int64_t gvq_i8_row_bytes(int64_t cols) { return (cols + 127) / 128 * 128; }

// What the columns' quantiser needs: the largest magnitudes of up to I8_CHUNKS runs of rows, each [cols].
constexpr int I8_CHUNKS = 32;
inline int64_t gvq_i8_chunk_rows(int64_t rows)
{
    const int64_t r = (rows + I8_CHUNKS - 1) / I8_CHUNKS;
    return r < 64 ? 64 : r;
}

struct I8QuantArgs {
    const void* x;
    int64_t rows, cols, ld;          // elements
    signed char* codes;              // of rows (may be null), rows of ldc bytes
    float* scales;
    signed char* codes_t;            // of columns (may be null), transposed, rows of ldct bytes
    float* scales_t;
    unsigned int* peaks;             // [chunks][cols], for columns
    int64_t ldc, ldct;               // filled in by the launcher, as are:
    int64_t chunk_rows;
    int words, chunks;
    int past;                        // past the caches
    int row_blocks;                  // work-groups that the rows take,
    int stripes, peak_blocks;        // that the columns' largest magnitudes take, side by side and in all,
    int across, column_blocks, band; // and the columns' codes, swept so many tiles down at a time
};

// What becomes of the sums of a product.
enum I8Mode { I8_PLAIN, I8_GATED, I8_INNER };

// C = A B^T and what is made of it: A [m][k], B [n][k] in codes of ldk bytes a row and scales.
struct I8ProductArgs {
    const signed char *a, *b;
    const float *a_scales, *b_scales;
    int64_t ldk;
    int m, n;             // rows of the result, its columns; gated: B has 2 n rows, the gate's and the other's
    void* out;
    int64_t ld;
    int accumulate;
    int activation;
    const void* dh;       // inner: the gradient of act(g) u
    int64_t ld_dh;
    int words, dh_words;  // rows are aligned to four elements
    int wide;             // all of the result's rows (inner: both halves) are aligned to 16 bytes
    int bf16;             // the result's type
    int nm, nn, band;     // tiles, and how they are swept
};

// One or two matrices of one type, in the same launches.
int gvq_launch_i8_quantize(const I8QuantArgs* matrices, int n, gvq_dtype_t dtype, hipStream_t st);
int gvq_launch_i8_dequantize(const void* codes, const void* scales, int64_t rows, int64_t cols, void* out, gvq_dtype_t dtype, int64_t ld,
                             hipStream_t st);
int gvq_launch_i8_product(I8ProductArgs a, I8Mode mode, gvq_dtype_t dtype, hipStream_t st);
// Two plain products, in one launch where that is the faster way.
int gvq_launch_i8_products(I8ProductArgs a, gvq_dtype_t a_dtype, I8ProductArgs b, gvq_dtype_t b_dtype, hipStream_t st);

typedef int i4v __attribute__((ext_vector_type(4)));

// A row's numbers are counted in units of its largest magnitude / 127.  `top`: the bits of that magnitude (infinity and NaN are above all
// numbers).  up = 127 / m and down = m / 127 are each rounded once; m is at least 2^-100, so that neither leaves fp32.  A row with
// an infinity or a NaN has codes 0 and the scale NaN.
struct I8Scale {
    float up, down;
};
__device__ __forceinline__ I8Scale i8_scale(unsigned int top)
{
    if (top >= 0x7f800000u) return {0.f, __uint_as_float(0x7fc00000u)};
    const float m = fmaxf(__uint_as_float(top), 0x1p-100f);
    return {__fdiv_rn(127.f, m), __fdiv_rn(m, 127.f)};
}
// The nearest integer to v up, halves to the even one, in the lowest byte: one fused multiply-add whose result's last place is 1, so
// that the product is rounded once, from all its bits.  (0 up for rows of no numbers: what is not finite gives any byte, masked by `keep`.)
__device__ __forceinline__ unsigned int i8_code(float v, float up) { return __float_as_uint(__builtin_fmaf(v, up, 12582912.f)); }
// The lowest bytes of four words.
__device__ __forceinline__ unsigned int i8_bytes(unsigned int a, unsigned int b, unsigned int c, unsigned int d)
{
    const unsigned int lo = __builtin_amdgcn_perm(b, a, 0x0c0c0400u), hi = __builtin_amdgcn_perm(d, c, 0x04000c0cu);
    return lo | hi;
}
__device__ __forceinline__ unsigned int i8_pack4(float a, float b, float c, float d, float up)
{
    return i8_bytes(i8_code(a, up), i8_code(b, up), i8_code(c, up), i8_code(d, up));
}

// The gate's activation and its derivative.  gelu: g Phi(g), with Phi(-y) = e^(-y^2/2) t P(t), t = 1 / (1 + y / sqrt(8)), y = |g|.  P is a
// polynomial fitted here to the least relative error of erfc(x) e^(x^2) / 2t, x = y / sqrt(2) up to 14: 8e-8, 3e-7 with fp32's rounding.
// Reciprocals and powers of 2 are the instructions', good to a step of the last place.
struct I8Gelu {
    float phi, bell;   // Phi(g), e^(-g^2/2)
};
__device__ __forceinline__ I8Gelu i8_gelu(float g)
{
    const float y = fabsf(g), t = __builtin_amdgcn_rcpf(__builtin_fmaf(y, 0.35355339f, 1.f));
    constexpr float C[9] = {-0.0297406688f, 0.143279284f, -0.245621964f, 0.141307905f, -0.0148506975f, 0.101980999f, 0.121394284f, 0.141208798f, 0.141042039f};
    float p = C[0];
#pragma unroll
    for (int i = 1; i < 9; ++i) p = __builtin_fmaf(p, t, C[i]);
    const float bell = __builtin_amdgcn_exp2f(-0.72134752f * g * g), low = bell * t * p;
    return {g > 0.f ? 1.f - low : low, bell};
}
__device__ __forceinline__ float i8_sigmoid(float g) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504f * g)); }
__device__ __forceinline__ float i8_activation(float g, int kind) { return g * (kind == 0 ? i8_sigmoid(g) : i8_gelu(g).phi); }
__device__ __forceinline__ void i8_activation_slope(float g, int kind, float& value, float& slope)
{
    if (kind == 0) {
        const float s = i8_sigmoid(g);
        value = g * s;
        slope = s * (1.f + g * (1.f - s));
    } else {
        const I8Gelu e = i8_gelu(g);
        value = g * e.phi;
        slope = e.phi + 0.39894228f * g * e.bell;
    }
}

// Four neighbouring numbers, of which `left` are in the matrix; `words`: p is aligned to all four.
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

// The scales of four neighbouring columns of the result: of the gate (or the only one) and of the other projection.  A sum over nothing
// has none.
struct I8Columns {
    f4 g, u;
};
template <I8Mode MODE>
__device__ __forceinline__ I8Columns i8_columns(const I8ProductArgs& a, int c)
{
    I8Columns s = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
    if (a.ldk > 0) {
        s.g = i8_load4(a.b_scales + c, false, a.n - c);
        if constexpr (MODE != I8_PLAIN) s.u = i8_load4(a.b_scales + a.n + c, false, a.n - c);
    }
    return s;
}

// Row r, columns c to c + 3 of the result from their sums: the gate's (or the only ones) and the other projection's.  inner: dg and du.
struct I8Results {
    f4 g, u;
};
template <I8Mode MODE>
__device__ __forceinline__ I8Results i8_results(const I8Columns& s, i4v sums_g, i4v sums_u, float scale, int activation, f4 dh)
{
    f4 g, u = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        g[i] = (float)sums_g[i] * (scale * s.g[i]);
        if constexpr (MODE != I8_PLAIN) u[i] = (float)sums_u[i] * (scale * s.u[i]);
    }
    if constexpr (MODE == I8_GATED) {
#pragma unroll
        for (int i = 0; i < 4; ++i) g[i] = i8_activation(g[i], activation) * u[i];
    } else if constexpr (MODE == I8_INNER) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float value, slope;
            i8_activation_slope(g[i], activation, value, slope);
            g[i] = dh[i] * u[i] * slope;
            u[i] = dh[i] * value;
        }
    }
    return {g, u};
}
template <I8Mode MODE, typename OUT>
__device__ __forceinline__ void i8_finish(const I8ProductArgs& a, OUT* out, int r, int c, const I8Columns& s, i4v sums_g, i4v sums_u, float scale)
{
    f4 dh = {0.f, 0.f, 0.f, 0.f};
    if constexpr (MODE == I8_INNER) dh = i8_load4((const OUT*)a.dh + (int64_t)r * a.ld_dh + c, a.dh_words != 0, a.n - c);
    const I8Results v = i8_results<MODE>(s, sums_g, sums_u, scale, a.activation, dh);
    OUT* p = out + (int64_t)r * a.ld + c;
    mx_store4(p, a.words != 0, a.n - c, MODE == I8_PLAIN && a.accumulate != 0, v.g);
    if constexpr (MODE == I8_INNER) mx_store4(p + a.n, a.words != 0 && (a.n & 3) == 0, a.n - c, false, v.u);
}

// Products of few rows without LDS tiles (gvq_i8_few.hip): of `tiles` times 16 rows of codes a work-group, or of at most four rows of numbers,
// quantised on the way.
int gvq_launch_i8_few(const I8ProductArgs& a, int tiles, I8Mode mode, gvq_dtype_t dtype, hipStream_t st);
bool gvq_i8_few_numbers_takes(const void* x, gvq_dtype_t x_dtype, int64_t rows, int64_t ld_x, int64_t k, I8Mode mode);
int gvq_launch_i8_few_numbers(I8ProductArgs a, const void* x, gvq_dtype_t x_dtype, int64_t ld_x, int64_t k, I8Mode mode, gvq_dtype_t dtype,
                              hipStream_t st);
