// Products of few rows with a 4-bit matrix, y = x W^T, where what there is to move is W, once, and a tile's work-groups would be too few
// to move it.
//
// A work-group has 16 rows of W, its 16 waves take the sum in turns of 512 numbers (256 bytes of every row), and each lane reads
// its operands straight into registers: row lane % 16, 16 bytes of codes a step, and four steps' scales in one word.  A turn's loads are
// asked for before the products of the turn before, with no branch around any of them (or every load would be waited for); where that
// would take more registers than two work-groups of a unit have (64 a lane), the compiler moves them back to their own turn and a wave waits for them
// there: all but the fp32 kernel of one to four rows (127 registers) are built so, and rely on the unit's other waves.  Loads go through the caches: an
// instruction takes half a line of each of 16 rows, the next one the other half (with loads past the caches 16 x 512 x 25088 17.8 us, so
// 13.6).  Up to four rows of x are quantised on the way: the 32 numbers that a lane needs are one block, so the lane finds its scale and
// packs its codes alone, without LDS and without a launch of its own.  More rows come in codes, 16 or 32 to a work-group.
// Bound: a compute unit's loads, 33 bytes a ns of codes each, and a turn's latency at the beginning and the end, in the products of codes also between.
// 77 x 1000 x 4096 6 us, 1 x 4096 x 25088 (54.6 MB) 10.9.
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
    int down;                   // work-groups of the same rows of W (codes)
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

// The waves' sums of 16 rows of W and R times 16 of x, a lane four neighbouring results of one row of x, added in the order of the waves.
template <typename OUT, int R>
__device__ __forceinline__ void few_out(const MxFewArgs& a, int r0, int n0, int wave, int lane, const f4 (&acc)[R], f4 (*sums)[FEW_WAVES][64])
{
#pragma unroll
    for (int t = 0; t < R; ++t) sums[t][wave][lane] = acc[t];
    __syncthreads();
    if (wave >= R) return;
    f4 v = sums[wave][0][lane];
#pragma unroll
    for (int i = 1; i < FEW_WAVES; ++i) v += sums[wave][i][lane];
    const int r = r0 + 16 * wave + (lane & 15), c = n0 + 4 * (lane >> 4);
    if (r < a.rows && c < a.n) mx_store4((OUT*)a.out + (int64_t)r * a.ld_out + c, a.words != 0, a.n - c, a.accumulate != 0, v);
}

// At most four rows of numbers.  A wave packs the blocks of four steps at once, lane 16 b + 4 k + r that of row r, step k and block b
// (alone they would fill a quarter of the lanes or less), and turns the lanes by 4 k for step k's product, where only the first
// four of sixteen matter.  One row of 25088 numbers in bf16 to 4096: with the blocks of each step packed on their own 22 us, so
// 11, which is what W's bytes take alone.
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
    __shared__ f4 sums[1][FEW_WAVES][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int n0 = blockIdx.x * 16, b = lane >> 4, wr = n0 + (lane & 15) < a.n ? n0 + (lane & 15) : a.n - 1;
    const int64_t lds = a.ldw >> 4;
    const char* w = a.w + wr * a.ldw + 16 * b;
    const char* ws = a.w_scales + wr * lds;
    const int xr = lane & 3, kk = lane >> 2 & 3;
    const X* x = (const X*)a.x + (int64_t)(xr < a.rows ? xr : a.rows - 1) * a.ld + 32 * b;
    f4 acc[1] = {f4{0.f, 0.f, 0.f, 0.f}};
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
        for (int i = 0; i < 4; ++i) q[set][i] = *(const u4*)(w + (s + i) * TILE_STEP);
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
            acc[0] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(few_operand(q[set][i]), few_operand(y), acc[0], 4, 4, 0,
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
        acc[0] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(few_operand(*(const u4*)(w + (int64_t)rest * TILE_STEP)), few_operand(xq), acc[0], 4, 4, 0,
                                                               *(const unsigned char*)(ws + (int64_t)rest * 4 + b), 0, xk);
    }
    few_out<OUT, 1>(a, 0, n0, wave, lane, acc, sums);
}

// Rows of codes, R times 16 a work-group: a turn is four steps here too, both operands' scales a word.  Work-groups of the same rows of W
// go side by side on one XCD.
template <typename OUT, int R>
__global__ __launch_bounds__(64 * FEW_WAVES) void mx_few_kernel(MxFewArgs a)
{
    __shared__ f4 sums[R][FEW_WAVES][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int t = tile_of_block(blockIdx.x, gridDim.x), r0 = t % a.down * (16 * R), n0 = t / a.down * 16;
    const int b = lane >> 4, wr = n0 + (lane & 15) < a.n ? n0 + (lane & 15) : a.n - 1;
    const int64_t lds = a.ldw >> 4;
    const char *w = a.w + wr * a.ldw + 16 * b, *ws = a.w_scales + wr * lds, *x[R], *xs[R];
#pragma unroll
    for (int j = 0; j < R; ++j) {
        const int64_t r = r0 + 16 * j + (lane & 15), xr = r < a.rows ? r : a.rows - 1;
        x[j] = (const char*)a.x + xr * a.ldw + 16 * b;
        xs[j] = a.x_scales + xr * lds;
    }
    f4 acc[R];
#pragma unroll
    for (int j = 0; j < R; ++j) acc[j] = f4{0.f, 0.f, 0.f, 0.f};
    const int turns_all = a.steps / 4, turns = turns_all > wave ? (turns_all - wave + FEW_WAVES - 1) / FEW_WAVES : 0;
    u4 q[2][4], y[2][R][4];
    MxScales4 k[2], yk[2][R];
    auto ask = [&](int t, int set) {
        const int turn = t < turns ? wave + t * FEW_WAVES : wave + (turns - 1) * FEW_WAVES;
        const int64_t s = 4 * (int64_t)turn;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            q[set][i] = *(const u4*)(w + (s + i) * TILE_STEP);
#pragma unroll
            for (int j = 0; j < R; ++j) y[set][j][i] = *(const u4*)(x[j] + (s + i) * TILE_STEP);
        }
        k[set] = *(const MxScales4*)(ws + s * 4);
#pragma unroll
        for (int j = 0; j < R; ++j) yk[set][j] = *(const MxScales4*)(xs[j] + s * 4);
    };
    auto take = [&](int set) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < R; ++j)
                acc[j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(few_operand(q[set][i]), few_operand(y[set][j][i]), acc[j], 4, 4, 0,
                                                                         (int)(k[set].v[i] >> (8 * b)), 0, (int)(yk[set][j].v[i] >> (8 * b)));
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
#pragma unroll
        for (int j = 0; j < R; ++j)
            acc[j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
                few_operand(*(const u4*)(w + (int64_t)rest * TILE_STEP)), few_operand(*(const u4*)(x[j] + (int64_t)rest * TILE_STEP)), acc[j], 4, 4, 0,
                *(const unsigned char*)(ws + (int64_t)rest * 4 + b), 0, *(const unsigned char*)(xs[j] + (int64_t)rest * 4 + b));
    few_out<OUT, R>(a, r0, n0, wave, lane, acc, sums);
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
    a.down = 1;
    a.out = out; a.ld_out = ld_out; a.accumulate = accumulate;
    a.words = (((uintptr_t)out | (uintptr_t)(ld_out * es)) & (uintptr_t)(4 * es - 1)) == 0;
    return a;
}

template <typename K>
static int launch_few(K kernel, const MxFewArgs& a, hipStream_t st)
{
    hipLaunchKernelGGL(kernel, dim3((unsigned)((a.n + 15) / 16 * a.down)), dim3(64 * FEW_WAVES), 0, st, a);
    GVQ_HIP(hipGetLastError());
    return GVQ_OK;
}

int gvq_launch_mx_few(int tiles, const void* x_codes, const void* x_scales, const void* w_codes, const void* w_scales, int64_t rows, int64_t n,
                      int64_t k, void* out, gvq_dtype_t dtype, int64_t ld_out, bool accumulate, hipStream_t st)
{
    MxFewArgs a = few_args(w_codes, w_scales, rows, n, k, out, dtype, ld_out, accumulate);
    a.x = x_codes; a.x_scales = (const char*)x_scales; a.ld = a.ldw;
    a.down = (int)((rows + 16 * tiles - 1) / (16 * tiles));
    if ((int64_t)(a.n + 15) / 16 * a.down > 0x7fffffff) return GVQ_EINVAL;
    if (tiles == 1) return dtype == GVQ_BF16 ? launch_few(mx_few_kernel<unsigned short, 1>, a, st) : launch_few(mx_few_kernel<float, 1>, a, st);
    return dtype == GVQ_BF16 ? launch_few(mx_few_kernel<unsigned short, 2>, a, st) : launch_few(mx_few_kernel<float, 2>, a, st);
}

// Numbers are packed by every work-group again, which costs little with one row of bf16 and most with four of fp32: rounds as for codes
// (gvq_mx_plan.h), fitted to 20 layers of 1 and 4 rows.  The other way is a launch that packs them once, 4 us, and the
// product of codes (4 rows of 4096 fp32 numbers to 25088 here 47 us, there 17; one row of 25088 bf16 numbers to 4096 here 11.2, there 13.6).  Of 32 layers measured
// both ways 28 take the faster one or lose less than 6 %; the others lose up to a quarter (4 fp32 rows of 4096 to 4096 8.1 us for 6.5).
bool gvq_mx_few_numbers_takes(const void* x, gvq_dtype_t x_dtype, int64_t rows, int64_t ld_x, int64_t n, int64_t k)
{
    const bool bf16 = x_dtype == GVQ_BF16;
    if (rows > 4 || (((uintptr_t)x | (uintptr_t)(ld_x * (bf16 ? 2 : 4))) & 15) != 0) return false;
    const int64_t steps = gvq_mx_row_bytes(k) / TILE_STEP, rounds = ((n + 15) / 16 + 255) / 256;
    const double round = bf16 ? (rows == 1 ? 0.45 + 0.06 * steps : 0.45 + 0.08 * steps) : (rows == 1 ? 1.3 + 0.074 * steps : 2.2 + 0.12 * steps);
    return 1.5 + rounds * round < 4.0 + gvq_mx_product_time(rows, n, k);
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
