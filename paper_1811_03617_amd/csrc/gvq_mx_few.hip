// Products of at most 16 rows with a 4-bit matrix, y = x W^T: what there is to move is W, once.
//
// A work-group has 16 rows of W, its 16 waves take the sum in turns of 512 numbers (256 bytes of every row), and each lane reads
// its operands straight into registers: row lane % 16, 16 bytes of codes a step, and four steps' scales in one word.  The loads run
// a turn ahead of the products, with no branch around any of them (or every load would be waited for).  Up to four rows of x are
// quantised on the way: the 32 numbers that a lane needs are one block, so the lane finds its scale and packs its codes alone, without
// LDS and without a launch of its own.  More rows come in codes.
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

// A block of 32 numbers as it lies in memory.
template <typename X>
struct FewBlock;

template <>
struct FewBlock<float> {
    u4 v[8];
    __device__ __forceinline__ void load(const float* p)
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
    __device__ __forceinline__ void load(const unsigned short* p)
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

__device__ __forceinline__ i8v few_operand(const u4& q) { return i8v{(int)q[0], (int)q[1], (int)q[2], (int)q[3], 0, 0, 0, 0}; }

struct MxScales4 {
    unsigned int v[4];
} __attribute__((aligned(4)));

// The waves' sums of 16 rows of W, a lane four neighbouring results of one row of x, added in the order of the waves.
template <typename OUT>
__device__ __forceinline__ void few_out(const MxFewArgs& a, int n0, int wave, int lane, const f4& acc, f4 (*sums)[64])
{
    sums[wave][lane] = acc;
    __syncthreads();
    if (wave != 0) return;
    f4 v = acc;
#pragma unroll
    for (int i = 1; i < FEW_WAVES; ++i) v += sums[i][lane];
    const int r = lane & 15, c = n0 + 4 * (lane >> 4);
    if (r < a.rows && c < a.n) mx_store4((OUT*)a.out + (int64_t)r * a.ld_out + c, a.words != 0, a.n - c, a.accumulate != 0, v);
}

// At most four rows of numbers.  A wave packs the blocks of four steps at once, lane 16 b + 4 k + r that of row r, step k and block b
// (alone they would fill a quarter of the lanes or less), and turns the lanes by 4 k for step k's product, where only the first
// four of sixteen matter.  One row of 25088 numbers in bf16 to 4096: with the blocks of each step packed on their own 22 us, so
// 15, of which W's bytes would take 9 to 11 alone.
// Lane i of 16 gets what lane (i + N) % 16 has.
template <int N>
__device__ __forceinline__ unsigned int turn_lanes(unsigned int v)
{
    if constexpr (N == 0) return v;
    else return (unsigned int)__builtin_amdgcn_mov_dpp((int)v, 0x120 + 16 - N, 0xf, 0xf, true);   // row_ror
}

template <typename X, typename OUT>
__global__ __launch_bounds__(64 * FEW_WAVES) void mx_four_kernel(MxFewArgs a)
{
    __shared__ f4 sums[FEW_WAVES][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int n0 = blockIdx.x * 16, b = lane >> 4, wr = n0 + (lane & 15) < a.n ? n0 + (lane & 15) : a.n - 1;
    const int64_t lds = a.ldw >> 4;
    const char* w = a.w + wr * a.ldw + 16 * b;
    const char* ws = a.w_scales + wr * lds;
    const int xr = lane & 3, kk = lane >> 2 & 3;
    const X* x = (const X*)a.x + (int64_t)(xr < a.rows ? xr : a.rows - 1) * a.ld + 32 * b;
    f4 acc = {0.f, 0.f, 0.f, 0.f};
    // A turn is four whole steps of numbers; this wave has the turns wave, wave + FEW_WAVES, ..  What is asked for behind the last
    // one is the last one once more.
    const int whole = a.k / 128, turns_all = whole / 4;
    const int turns = turns_all > wave ? (turns_all - wave + FEW_WAVES - 1) / FEW_WAVES : 0;
    u4 q[2][4];
    MxScales4 k[2];
    FewBlock<X> block[2];
    auto ask = [&](int t, int set) {
        const int turn = t < turns ? wave + t * FEW_WAVES : wave + (turns - 1) * FEW_WAVES;
        const int64_t s = 4 * (int64_t)turn;
        block[set].load(x + (s + kk) * 128);
#pragma unroll
        for (int i = 0; i < 4; ++i) q[set][i] = stream_load((const u4*)(w + (s + i) * TILE_STEP));
        k[set] = *(const MxScales4*)(ws + s * 4);
    };
    auto take = [&](int set) {
        u4 xq;
        int xk;
        block[set].pack(xq, xk);
        static_for<0, 4>([&](auto c) {
            constexpr int i = decltype(c)::value;
            const u4 y = {turn_lanes<4 * i>(xq[0]), turn_lanes<4 * i>(xq[1]), turn_lanes<4 * i>(xq[2]), turn_lanes<4 * i>(xq[3])};
            const int yk = (int)turn_lanes<4 * i>((unsigned int)xk);
            acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(few_operand(q[set][i]), few_operand(y), acc, 4, 4, 0,
                                                                   (int)(k[set].v[i] >> (8 * b)), 0, yk);
        });
    };
    if (turns > 0) ask(0, 0);
    for (int t = 0; t < turns; t += 2) {
        ask(t + 1, 1);
        take(0);
        if (t + 1 >= turns) break;
        ask(t + 2, 0);
        take(1);
    }
    // what is left: up to three whole steps and a part of one, a wave each
    const int rest = 4 * turns_all + (FEW_WAVES - 1 - wave);
    if (rest < a.steps) {
        FewBlock<X> last;
        last.load_some(x + (int64_t)rest * 128, a.k - rest * 128 - 32 * b);
        u4 xq;
        int xk;
        last.pack(xq, xk);
        acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(few_operand(*(const u4*)(w + (int64_t)rest * TILE_STEP)), few_operand(xq), acc, 4, 4, 0,
                                                               *(const unsigned char*)(ws + (int64_t)rest * 4 + b), 0, xk);
    }
    few_out<OUT>(a, n0, wave, lane, acc, sums);
}

// Rows of codes, up to 16: a turn is four steps here too, both operands' scales a word.
template <typename OUT>
__global__ __launch_bounds__(64 * FEW_WAVES) void mx_few_kernel(MxFewArgs a)
{
    __shared__ f4 sums[FEW_WAVES][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int n0 = blockIdx.x * 16, b = lane >> 4, wr = n0 + (lane & 15) < a.n ? n0 + (lane & 15) : a.n - 1;
    const int64_t lds = a.ldw >> 4, xr = (lane & 15) < a.rows ? lane & 15 : a.rows - 1;
    const char *w = a.w + wr * a.ldw + 16 * b, *x = (const char*)a.x + xr * a.ldw + 16 * b;
    const char *ws = a.w_scales + wr * lds, *xs = a.x_scales + xr * lds;
    f4 acc = {0.f, 0.f, 0.f, 0.f};
    const int turns_all = a.steps / 4, turns = turns_all > wave ? (turns_all - wave + FEW_WAVES - 1) / FEW_WAVES : 0;
    u4 q[2][4], y[2][4];
    MxScales4 k[2], yk[2];
    auto ask = [&](int t, int set) {
        const int turn = t < turns ? wave + t * FEW_WAVES : wave + (turns - 1) * FEW_WAVES;
        const int64_t s = 4 * (int64_t)turn;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            q[set][i] = stream_load((const u4*)(w + (s + i) * TILE_STEP));
            y[set][i] = *(const u4*)(x + (s + i) * TILE_STEP);
        }
        k[set] = *(const MxScales4*)(ws + s * 4);
        yk[set] = *(const MxScales4*)(xs + s * 4);
    };
    auto take = [&](int set) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(few_operand(q[set][i]), few_operand(y[set][i]), acc, 4, 4, 0,
                                                                   (int)(k[set].v[i] >> (8 * b)), 0, (int)(yk[set].v[i] >> (8 * b)));
    };
    if (turns > 0) ask(0, 0);
    for (int t = 0; t < turns; t += 2) {
        ask(t + 1, 1);
        take(0);
        if (t + 1 >= turns) break;
        ask(t + 2, 0);
        take(1);
    }
    const int rest = 4 * turns_all + (FEW_WAVES - 1 - wave);   // up to three more steps, a wave each
    if (rest < a.steps)
        acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
            few_operand(*(const u4*)(w + (int64_t)rest * TILE_STEP)), few_operand(*(const u4*)(x + (int64_t)rest * TILE_STEP)), acc, 4, 4, 0,
            *(const unsigned char*)(ws + (int64_t)rest * 4 + b), 0, *(const unsigned char*)(xs + (int64_t)rest * 4 + b));
    few_out<OUT>(a, n0, wave, lane, acc, sums);
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

template <typename K>
static int launch_few(K kernel, const MxFewArgs& a, hipStream_t st)
{
    hipLaunchKernelGGL(kernel, dim3((a.n + 15) / 16), dim3(64 * FEW_WAVES), 0, st, a);
    GVQ_HIP(hipGetLastError());
    return GVQ_OK;
}

int gvq_launch_mx_few(const void* x_codes, const void* x_scales, const void* w_codes, const void* w_scales, int64_t rows, int64_t n,
                      int64_t k, void* out, gvq_dtype_t dtype, int64_t ld_out, bool accumulate, hipStream_t st)
{
    MxFewArgs a = few_args(w_codes, w_scales, rows, n, k, out, dtype, ld_out, accumulate);
    a.x = x_codes; a.x_scales = (const char*)x_scales; a.ld = a.ldw;
    return dtype == GVQ_BF16 ? launch_few(mx_few_kernel<unsigned short>, a, st) : launch_few(mx_few_kernel<float>, a, st);
}

bool gvq_mx_few_numbers_takes(const void* x, gvq_dtype_t x_dtype, int64_t rows, int64_t ld_x)
{
    return rows <= 4 && (((uintptr_t)x | (uintptr_t)(ld_x * (x_dtype == GVQ_BF16 ? 2 : 4))) & 15) == 0;
}

int gvq_launch_mx_few_numbers(const void* x, gvq_dtype_t x_dtype, int64_t ld_x, const void* w_codes, const void* w_scales, int64_t rows,
                              int64_t n, int64_t k, void* out, gvq_dtype_t dtype, int64_t ld_out, hipStream_t st)
{
    MxFewArgs a = few_args(w_codes, w_scales, rows, n, k, out, dtype, ld_out, false);
    a.x = x; a.ld = ld_x;
    if (x_dtype == GVQ_BF16)
        return dtype == GVQ_BF16 ? launch_few(mx_four_kernel<unsigned short, unsigned short>, a, st) : launch_few(mx_four_kernel<unsigned short, float>, a, st);
    return dtype == GVQ_BF16 ? launch_few(mx_four_kernel<float, unsigned short>, a, st) : launch_few(mx_four_kernel<float, float>, a, st);
}
