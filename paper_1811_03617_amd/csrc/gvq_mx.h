// 4-bit microscaled blocks: device helpers and the launchers' declarations.
#pragma once
#include "gvq_device.h"

struct MxQuantArgs {
    const void* x;
    int64_t rows, cols, ld;          // elements
    const unsigned char* noise;      // null: to the nearest
    int64_t noise_ld;
    unsigned char *codes, *scales;       // blocks along rows (codes may be null), rows of ldc bytes
    unsigned char *codes_t, *scales_t;   // blocks along columns (may be null), transposed, rows of ldct bytes
    int64_t ldc, ldct;               // filled in by the launcher, as are:
    int words, noise_words;          // rows are aligned for wide loads
    int across;                      // tiles of 64 columns
};

// Bytes of one row of codes: a whole number of 128 columns; the scales take a sixteenth of that.
inline int64_t gvq_mx_row_bytes(int64_t cols) { return (cols + 127) / 128 * 64; }

int gvq_launch_mx_quantize(MxQuantArgs a, gvq_dtype_t dtype, hipStream_t st);
int gvq_launch_mx_dequantize(const void* codes, const void* scales, int64_t rows, int64_t cols, void* out, gvq_dtype_t dtype,
                             int64_t ld, hipStream_t st);
// out = A B^T (+ out): A [m][k], B [n][k] in codes and scales.
int gvq_launch_mx_matmul(const void* a_codes, const void* a_scales, const void* b_codes, const void* b_scales, int64_t m, int64_t n,
                         int64_t k, void* out, gvq_dtype_t dtype, int64_t ld, bool accumulate, hipStream_t st);
// About how many us that takes.
double gvq_mx_product_time(int64_t m, int64_t n, int64_t k);
// The same without LDS, `tiles` (1 or 2) times 16 rows of A a work-group; of at most 4 rows of numbers, aligned to 16 bytes and quantised on
// the way, where that is the faster way (gvq_mx_few.hip).
int gvq_launch_mx_few(int tiles, const void* x_codes, const void* x_scales, const void* w_codes, const void* w_scales, int64_t rows, int64_t n,
                      int64_t k, void* out, gvq_dtype_t dtype, int64_t ld_out, bool accumulate, hipStream_t st);
bool gvq_mx_few_numbers_takes(const void* x, gvq_dtype_t x_dtype, int64_t rows, int64_t ld_x, int64_t n, int64_t k);
int gvq_launch_mx_few_numbers(const void* x, gvq_dtype_t x_dtype, int64_t ld_x, const void* w_codes, const void* w_scales, int64_t rows,
                              int64_t n, int64_t k, void* out, gvq_dtype_t dtype, int64_t ld_out, hipStream_t st);

// Eight numbers from p, of which `left` are in the matrix (the others are 0); `words`: p is 16-byte aligned.
__device__ __forceinline__ void mx_load8(const float* p, bool words, int64_t left, float (&v)[8])
{
    if (words && left >= 8) {
        const f4 a = stream_load((const f4*)p), b = stream_load((const f4*)p + 1);
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < left ? p[i] : 0.f;
    }
}
__device__ __forceinline__ void mx_load8(const unsigned short* p, bool words, int64_t left, float (&v)[8])
{
    if (words && left >= 8) {
        const u4 a = stream_load((const u4*)p);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(a[i] << 16);
            v[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < left ? bf16_to_f32(p[i]) : 0.f;
    }
}
__device__ __forceinline__ void mx_noise8(const unsigned char* p, bool words, int64_t left, unsigned int (&z)[2])
{
    if (words && left >= 8) {
        const u2 a = *(const u2*)p;
        z[0] = a[0]; z[1] = a[1];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) z[i >> 2] |= (unsigned int)p[i] << (8 * (i & 3));
    }
}
__device__ __forceinline__ void mx_store8(float* p, bool words, int64_t left, const float (&v)[8])
{
    if (words && left >= 8) {
        stream_store((f4*)p, f4{v[0], v[1], v[2], v[3]});
        stream_store((f4*)p + 1, f4{v[4], v[5], v[6], v[7]});
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) p[i] = v[i];
    }
}
__device__ __forceinline__ void mx_store8(unsigned short* p, bool words, int64_t left, const float (&v)[8])
{
    if (words && left >= 8) {
        stream_store((u4*)p, u4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])});
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) p[i] = (unsigned short)f32_to_bf16_rne(v[i]);
    }
}

// Largest magnitude, as bits: they order as the magnitudes do, with infinity and then NaN above every number.
__device__ __forceinline__ unsigned int mx_top8(const float* v)
{
    unsigned int m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const unsigned int u = __float_as_uint(v[i]) & 0x7fffffffu;
        m = u > m ? u : m;
    }
    return m;
}
// ... over four neighbouring lanes.
__device__ __forceinline__ unsigned int mx_max_of_4(unsigned int m)
{
    unsigned int o = (unsigned int)__builtin_amdgcn_mov_dpp((int)m, 0xB1, 0xf, 0xf, true);   // quad_perm 1 0 3 2
    m = o > m ? o : m;
    o = (unsigned int)__builtin_amdgcn_mov_dpp((int)m, 0x4E, 0xf, 0xf, true);                // quad_perm 2 3 0 1
    return o > m ? o : m;
}
// Biased exponent of the scale: two below the largest magnitude's, at least 0 (which is 2^-127); 255 marks a block that holds an
// infinity or a NaN and whose numbers are all NaN.
__device__ __forceinline__ int mx_scale_code(unsigned int top)
{
    const int e = (int)(top >> 23);
    return e == 255 ? 255 : e < 2 ? 0 : e - 2;
}
// 2^(code - 127); code 0 is a denormal, 255 becomes a NaN.
__device__ __forceinline__ float mx_scale(int code)
{
    return __uint_as_float(code == 0 ? 0x00400000u : code == 255 ? 0x7fc00000u : (unsigned int)code << 23);
}

// One number rounded stochastically: its magnitude lies u steps (1/2, 1 or 2) from 0; up if the fraction of a step is above
// (z + 1/2) / 256.  Every step here is exact: a multiplication by powers of two, floor, a difference.
__device__ __forceinline__ unsigned int mx_code_noise(float v, float inv, unsigned int z)
{
    float t = fminf(fabsf(v) * inv, 6.f);
    const float per = t < 2.f ? 2.f : t < 4.f ? 1.f : 0.5f;      // steps in 1
    const float u = t * per, f = floorf(u);
    const float up = (u - f) * 256.f > (float)z + 0.5f ? 1.f : 0.f;
    // codes: 0..3 count halves, 4 and 5 stand for 2 and 3, 6 and 7 for 4 and 6
    const float c = f + up + (t < 2.f ? 0.f : t < 4.f ? 2.f : 4.f);
    return (unsigned int)c | (__float_as_uint(v) >> 31 << 3);
}

// Eight numbers -> eight codes, the first in the lowest four bits.  z: their random bytes.
template <bool NOISE>
__device__ __forceinline__ unsigned int mx_pack8(const float* v, const unsigned int (&z)[2], int code)
{
    if constexpr (NOISE) {
        const float inv = __uint_as_float((unsigned int)(254 - code) << 23);   // 2^(127 - code), for codes of up to 252
        unsigned int q = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) q |= mx_code_noise(v[i], inv, z[i >> 2] >> (8 * (i & 3)) & 255u) << (4 * i);
        return q;
    } else {
        const float s = mx_scale(code);
        unsigned int q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, v[0], v[1], s, 0);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[2], v[3], s, 1);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[4], v[5], s, 2);
        return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[6], v[7], s, 3);
    }
}
__device__ __forceinline__ void mx_unpack8(unsigned int q, int code, float (&v)[8])
{
    const float s = mx_scale(code);
    const gvq_f2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, s, 1);
    const gvq_f2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, s, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, s, 3);
    v[0] = a[0]; v[1] = a[1]; v[2] = b[0]; v[3] = b[1];
    v[4] = c[0]; v[5] = c[1]; v[6] = d[0]; v[7] = d[1];
}

// Four neighbouring results, of which `left` are in the matrix; `words`: p is aligned to all four.
__device__ __forceinline__ void mx_store4(float* p, bool words, int left, bool add, f4 v)
{
    if (words && left >= 4) {
        if (add) v += *(const f4*)p;
        *(f4*)p = v;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < left) p[i] = add ? p[i] + v[i] : v[i];
    }
}
__device__ __forceinline__ void mx_store4(unsigned short* p, bool words, int left, bool add, f4 v)
{
    if (words && left >= 4) {
        if (add) {
            const u2 o = *(const u2*)p;
            v += f4{__uint_as_float(o[0] << 16), __uint_as_float(o[0] & 0xffff0000u), __uint_as_float(o[1] << 16), __uint_as_float(o[1] & 0xffff0000u)};
        }
        *(u2*)p = u2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < left) p[i] = (unsigned short)f32_to_bf16_rne(add ? bf16_to_f32(p[i]) + v[i] : v[i]);
    }
}
