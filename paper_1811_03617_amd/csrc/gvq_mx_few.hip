// Products of at most 16 rows with a 4-bit matrix, y = x W^T: what there is to move is W, once.
//
// A work-group has 16 rows of W, its 16 waves take the sum in turns of 256 numbers (128 bytes of every row), and each lane reads
// its operands straight into registers: row lane % 16, 16 bytes of codes and their scale.  Their loads run two turns ahead of the
// products.  Rows of x in numbers are quantised on the way: the 32 numbers that a lane needs are one block, so the lane finds its
// scale and packs its codes alone, without LDS and without a launch of its own.
// The waves' sums are added in the order of the waves.
#include "gvq_mx.h"
#include "gvq_tile.h"

#define FEW_WAVES 16

struct MxFewArgs {
    const void* x;              // numbers, or codes (rows of ld bytes)
    const char* x_scales;       // codes only
    int64_t ld;
    const char *w, *w_scales;   // rows of ldw bytes
    int64_t ldw;
    int rows, n, k, steps;
    void* out;
    int64_t ld_out;
    int accumulate, words;
};

// A block of 32 numbers as it lies in memory, or its codes and scale.
template <typename X>
struct FewBlock;

template <>
struct FewBlock<float> {
    u4 v[8];
    __device__ __forceinline__ void load(const float* p, const char*)
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = *(const u4*)(p + 4 * i);
    }
    __device__ __forceinline__ void load_some(const float* p, int left)
    {
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i >> 2][i & 3] = i < left ? __float_as_uint(p[i]) : 0u;
    }
    __device__ __forceinline__ void pack(u4& q, int& code) const
    {
        unsigned int top = 0;
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            const unsigned int t = v[i >> 2][i & 3] & 0x7fffffffu;
            top = t > top ? t : top;
        }
        code = mx_scale_code(top);
        const unsigned int none[2] = {0, 0};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float f[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) f[k] = __uint_as_float(v[2 * i + (k >> 2)][k & 3]);
            q[i] = code == 255 ? 0 : mx_pack8<false>(f, none, code);
        }
    }
};

template <>
struct FewBlock<unsigned short> {
    u4 v[4];
    __device__ __forceinline__ void load(const unsigned short* p, const char*)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = *(const u4*)(p + 8 * i);
    }
    __device__ __forceinline__ void load_some(const unsigned short* p, int left)
    {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            v[i >> 2][i & 3] = (2 * i < left ? p[2 * i] : 0u) | (2 * i + 1 < left ? (unsigned int)p[2 * i + 1] : 0u) << 16;
    }
    __device__ __forceinline__ void pack(u4& q, int& code) const
    {
        // magnitudes of bf16 numbers order as their 15 lower bits
        typedef unsigned short us2 __attribute__((ext_vector_type(2)));
        us2 top = {0, 0};
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const unsigned int w = v[i >> 2][i & 3] & 0x7fff7fffu;
            top = __builtin_elementwise_max(top, __builtin_bit_cast(us2, w));
        }
        code = mx_scale_code((unsigned int)(top[0] > top[1] ? top[0] : top[1]) << 16);
        const float s = mx_scale(code);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            // (each word as a value of its own: a bit cast of a vector's element takes the first one)
            const unsigned int w0 = v[i][0], w1 = v[i][1], w2 = v[i][2], w3 = v[i][3];
            unsigned int r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(0u, __builtin_bit_cast(gvq_bf2, w0), s, 0);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(gvq_bf2, w1), s, 1);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(gvq_bf2, w2), s, 2);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(gvq_bf2, w3), s, 3);
            q[i] = code == 255 ? 0 : r;
        }
    }
};

template <>
struct FewBlock<unsigned char> {
    u4 v;
    int k;
    __device__ __forceinline__ void load(const unsigned char* p, const char* s)
    {
        v = *(const u4*)p;
        k = *(const unsigned char*)s;
    }
    __device__ __forceinline__ void pack(u4& q, int& code) const { q = v; code = k; }
};
__device__ __forceinline__ i8v few_operand(const u4& q) { return i8v{(int)q[0], (int)q[1], (int)q[2], (int)q[3], 0, 0, 0, 0}; }

// X: float or unsigned short (bf16): numbers; unsigned char: codes.  16 rows at most.
template <typename X, typename OUT>
__global__ __launch_bounds__(64 * FEW_WAVES) void mx_few_kernel(MxFewArgs a)
{
    constexpr bool CODES = sizeof(X) == 1;
    constexpr int TURN = sizeof(X) == 4 ? 1 : 2;   // steps of 128 numbers a wave takes at a time: 32 registers of numbers at most
    __shared__ f4 sums[FEW_WAVES][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int n0 = blockIdx.x * 16, b = lane >> 4, wr = n0 + (lane & 15) < a.n ? n0 + (lane & 15) : a.n - 1;
    const char* w = a.w + wr * a.ldw + 16 * b;
    const char* ws = a.w_scales + wr * (a.ldw >> 4) + b;
    const int64_t xr = (lane & 15) < a.rows ? lane & 15 : a.rows - 1;
    const X* x = (const X*)a.x + xr * a.ld + (CODES ? 16 * b : 32 * b);
    const char* xs = CODES ? a.x_scales + xr * (a.ld >> 4) + b : nullptr;
    f4 acc = {0.f, 0.f, 0.f, 0.f};
    // Turn t of this wave: TURN steps from s0 + t FEW_WAVES TURN on; what is asked for behind the last one is the last one once
    // more, and not multiplied.  Only whole steps of numbers: a branch around a load would have every load waited for.
    const int steps = CODES ? a.steps : a.k / 128, s0 = wave * TURN;
    const int turns = steps > s0 ? (steps - s0 + FEW_WAVES * TURN - 1) / (FEW_WAVES * TURN) : 0;
    u4 q[2][TURN];
    int k[2][TURN];
    FewBlock<X> blocks[2][TURN];
    auto ask = [&](int t, int set) {
#pragma unroll
        for (int i = 0; i < TURN; ++i) {
            const int next = s0 + t * (FEW_WAVES * TURN) + i, s = next < steps ? next : steps - 1;
            q[set][i] = stream_load((const u4*)(w + (int64_t)s * TILE_STEP));
            k[set][i] = *(const unsigned char*)(ws + (int64_t)s * 4);
            blocks[set][i].load(x + (int64_t)s * (CODES ? TILE_STEP : 128), CODES ? xs + (int64_t)s * 4 : nullptr);
        }
    };
    auto multiply = [&](const u4& wq, int wk, const FewBlock<X>& block) {
        u4 xq;
        int xk;
        block.pack(xq, xk);
        acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(few_operand(wq), few_operand(xq), acc, 4, 4, 0, wk, 0, xk);
    };
    auto take = [&](int t, int set) {
#pragma unroll
        for (int i = 0; i < TURN; ++i)
            if (s0 + t * (FEW_WAVES * TURN) + i < steps) multiply(q[set][i], k[set][i], blocks[set][i]);
    };
    if (turns > 0) ask(0, 0);
    for (int t = 0; t < turns; t += 2) {
        ask(t + 1, 1);
        take(t, 0);
        if (t + 1 >= turns) break;
        ask(t + 2, 0);
        take(t + 1, 1);
    }
    if constexpr (!CODES)
        if (steps < a.steps && wave == FEW_WAVES - 1) {   // what is left of the last step
            FewBlock<X> block;
            block.load_some(x + (int64_t)steps * 128, a.k - steps * 128 - 32 * b);
            multiply(*(const u4*)(w + (int64_t)steps * TILE_STEP), *(const unsigned char*)(ws + (int64_t)steps * 4), block);
        }
    sums[wave][lane] = acc;
    __syncthreads();
    if (wave == 0) {
        f4 v = acc;
#pragma unroll
        for (int i = 1; i < FEW_WAVES; ++i) v += sums[i][lane];
        const int r = lane & 15, c = n0 + 4 * b;
        if (r < a.rows && c < a.n) mx_store4((OUT*)a.out + (int64_t)r * a.ld_out + c, a.words != 0, a.n - c, a.accumulate != 0, v);
    }
}

template <typename X, typename OUT>
static int launch_few(const MxFewArgs& a, hipStream_t st)
{
    const dim3 grid((a.n + 15) / 16), threads(64 * FEW_WAVES);
    hipLaunchKernelGGL((mx_few_kernel<X, OUT>), grid, threads, 0, st, a);
    GVQ_HIP(hipGetLastError());
    return GVQ_OK;
}

static MxFewArgs few_args(const void* w_codes, const void* w_scales, int64_t rows, int64_t n, int64_t k, void* out, gvq_dtype_t dtype,
                          int64_t ld_out, bool accumulate)
{
    MxFewArgs a{};
    const int64_t es = dtype == GVQ_BF16 ? 2 : 4;
    a.w = (const char*)w_codes; a.w_scales = (const char*)w_scales;
    a.ldw = gvq_mx_row_bytes(k);
    a.rows = (int)rows; a.n = (int)n; a.k = (int)k;
    a.steps = (int)(a.ldw / TILE_STEP);
    a.out = out; a.ld_out = ld_out; a.accumulate = accumulate;
    a.words = (((uintptr_t)out | (uintptr_t)(ld_out * es)) & (uintptr_t)(4 * es - 1)) == 0;
    return a;
}

int gvq_launch_mx_few(const void* x_codes, const void* x_scales, const void* w_codes, const void* w_scales, int64_t rows, int64_t n,
                      int64_t k, void* out, gvq_dtype_t dtype, int64_t ld_out, bool accumulate, hipStream_t st)
{
    MxFewArgs a = few_args(w_codes, w_scales, rows, n, k, out, dtype, ld_out, accumulate);
    a.x = x_codes; a.x_scales = (const char*)x_scales; a.ld = a.ldw;
    return dtype == GVQ_BF16 ? launch_few<unsigned char, unsigned short>(a, st) : launch_few<unsigned char, float>(a, st);
}

bool gvq_mx_few_numbers_takes(const void* x, gvq_dtype_t x_dtype, int64_t rows, int64_t ld_x)
{
    return rows <= 16 && (((uintptr_t)x | (uintptr_t)(ld_x * (x_dtype == GVQ_BF16 ? 2 : 4))) & 15) == 0;
}

int gvq_launch_mx_few_numbers(const void* x, gvq_dtype_t x_dtype, int64_t ld_x, const void* w_codes, const void* w_scales, int64_t rows,
                              int64_t n, int64_t k, void* out, gvq_dtype_t dtype, int64_t ld_out, hipStream_t st)
{
    MxFewArgs a = few_args(w_codes, w_scales, rows, n, k, out, dtype, ld_out, false);
    a.x = x; a.ld = ld_x;
    if (x_dtype == GVQ_BF16)
        return dtype == GVQ_BF16 ? launch_few<unsigned short, unsigned short>(a, st) : launch_few<unsigned short, float>(a, st);
    return dtype == GVQ_BF16 ? launch_few<float, unsigned short>(a, st) : launch_few<float, float>(a, st);
}
