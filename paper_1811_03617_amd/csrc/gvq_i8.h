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
    int words, across, chunks;
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
    int nm, nn, band;     // tiles, and how they are swept
};

int gvq_launch_i8_quantize(I8QuantArgs a, gvq_dtype_t dtype, hipStream_t st);
int gvq_launch_i8_dequantize(const void* codes, const void* scales, int64_t rows, int64_t cols, void* out, gvq_dtype_t dtype, int64_t ld,
                             hipStream_t st);
int gvq_launch_i8_product(I8ProductArgs a, I8Mode mode, gvq_dtype_t dtype, hipStream_t st);

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

// The gate's activation and its derivative.
__device__ __forceinline__ float i8_activation(float g, int kind)
{
    if (kind == 0) return g / (1.f + __expf(-g));
    return 0.5f * g * erfcf(-0.70710678f * g);
}
__device__ __forceinline__ void i8_activation_slope(float g, int kind, float& value, float& slope)
{
    if (kind == 0) {
        const float s = 1.f / (1.f + __expf(-g));
        value = g * s;
        slope = s * (1.f + g * (1.f - s));
    } else {
        const float phi = 0.5f * erfcf(-0.70710678f * g);
        value = g * phi;
        slope = phi + 0.39894228f * g * __expf(-0.5f * g * g);
    }
}
