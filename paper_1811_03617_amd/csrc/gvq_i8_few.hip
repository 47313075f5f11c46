// Products of few rows with a matrix of 8-bit integers, where what there is to move is that matrix, once, and a tile's work-groups would be
// too few to move it.
//
// A work-group has 16 rows of W (gated: 16 of each projection), its 16 waves take the sum in turns of 256 numbers, and each lane reads its operands
// straight into registers: row lane % 16, 16 bytes of 64.  The waves' sums are whole numbers and are added exactly.  Up to four rows of x
// are quantised by every work-group for itself, into LDS, while the first turns of W are on their way: that costs it one read of x from the
// caches and saves a launch.  More rows come in codes, 16 or 32 to a work-group.
// Bound: memory, W once; what a compute unit can have on its way (about 29 bytes a ns) and the latency at both ends for small ones.  One bf16 row of
// 25088 numbers into 4096 20.1 us (5.1 TB/s of W), of 4096 into 25088 22.6, of 4096 into 4096 5.0; gated, of 4096 into 2 x 8192, 15.8; codes of 16 rows of 4096 numbers into
// 4096 6.3.
#include "gvq_i8.h"
#include "gvq_tile.h"

#define I8_FEW_WAVES 16

// The waves' sums of 16 rows of W and R times 16 of x, joined; a lane has four neighbouring results of one row of x.
template <I8Mode MODE, typename OUT, int R>
__device__ __forceinline__ void i8_few_out(const I8ProductArgs& a, int r0, int n0, int wave, int lane, const i4v (&acc)[R][MODE == I8_PLAIN ? 1 : 2],
                                           const float* scales, i4v (*sums)[I8_FEW_WAVES][64])
{
    constexpr int PAIR = MODE == I8_PLAIN ? 1 : 2;
#pragma unroll
    for (int t = 0; t < R; ++t)
#pragma unroll
        for (int p = 0; p < PAIR; ++p) sums[t * PAIR + p][wave][lane] = acc[t][p];
    __syncthreads();
    if (wave >= R) return;
    i4v v[2] = {sums[wave * PAIR][0][lane], sums[wave * PAIR + PAIR - 1][0][lane]};
#pragma unroll 5   // (all of a pair's sums at one time would take 128 registers)
    for (int i = 1; i < I8_FEW_WAVES; ++i) {
        v[0] += sums[wave * PAIR][i][lane];
        if constexpr (PAIR == 2) v[1] += sums[wave * PAIR + 1][i][lane];
    }
    const int r = r0 + 16 * wave + (lane & 15), c = n0 + 4 * (lane >> 4);
    if (r < a.m && c < a.n) i8_finish<MODE>(a, (OUT*)a.out, r, c, i8_columns<MODE>(a, c), v[0], v[1], scales[r - r0]);
}

// Where a lane's row of W begins.
__device__ __forceinline__ const signed char* i8_few_row(const I8ProductArgs& a, int n0, int lane, int which)
{
    const int r = n0 + (lane & 15) < a.n ? n0 + (lane & 15) : a.n - 1;
    return a.b + (int64_t)(which ? a.n + r : r) * a.ldk + 16 * (lane >> 4);
}

// ---- codes --------------------------------------------------------------------------------------------------------

template <I8Mode MODE, typename OUT, int R>
__global__ __launch_bounds__(64 * I8_FEW_WAVES) void i8_few_kernel(I8ProductArgs a)
{
    constexpr int PAIR = MODE == I8_PLAIN ? 1 : 2;
    __shared__ __attribute__((aligned(16))) i4v sums[R * PAIR][I8_FEW_WAVES][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int t = tile_of_block(blockIdx.x, gridDim.x), r0 = t % a.nm * (16 * R), n0 = t / a.nm * 16;
    const signed char *w[PAIR], *x[R];
#pragma unroll
    for (int p = 0; p < PAIR; ++p) w[p] = i8_few_row(a, n0, lane, p);
#pragma unroll
    for (int j = 0; j < R; ++j) {
        const int r = r0 + 16 * j + (lane & 15);
        x[j] = a.a + (int64_t)(r < a.m ? r : a.m - 1) * a.ldk + 16 * (lane >> 4);
    }
    i4v acc[R][PAIR];
#pragma unroll
    for (int j = 0; j < R; ++j)
#pragma unroll
        for (int p = 0; p < PAIR; ++p) acc[j][p] = i4v{0, 0, 0, 0};
    // this wave has the turns wave, wave + 16, ..; what is asked for behind the last one is the last one once more
    const int turns_all = (int)(a.ldk / 256), turns = turns_all > wave ? (turns_all - wave + I8_FEW_WAVES - 1) / I8_FEW_WAVES : 0;
    i4v q[2][PAIR][4], y[2][R][4];
    auto ask = [&](int t, int set) {
        const int64_t at = 256 * (int64_t)(t < turns ? wave + t * I8_FEW_WAVES : wave + (turns - 1) * I8_FEW_WAVES);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int p = 0; p < PAIR; ++p) q[set][p][i] = *(const i4v*)(w[p] + at + 64 * i);
#pragma unroll
            for (int j = 0; j < R; ++j) y[set][j][i] = *(const i4v*)(x[j] + at + 64 * i);
        }
    };
    auto take = [&](int set) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < R; ++j)
#pragma unroll
                for (int p = 0; p < PAIR; ++p) acc[j][p] = __builtin_amdgcn_mfma_i32_16x16x64_i8(q[set][p][i], y[set][j][i], acc[j][p], 0, 0, 0);
    };
    if (turns > 0) ask(0, 0);
    for (int t = 0; t < turns; t += 2) {
        ask(t + 1, 1);
        take(0);
        if (t + 1 >= turns) break;
        ask(t + 2, 0);
        take(1);
    }
    if ((a.ldk & 128) && wave == I8_FEW_WAVES - 1)   // half a turn is left
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < R; ++j)
#pragma unroll
                for (int p = 0; p < PAIR; ++p)
                    acc[j][p] = __builtin_amdgcn_mfma_i32_16x16x64_i8(*(const i4v*)(w[p] + a.ldk - 128 + 64 * i), *(const i4v*)(x[j] + a.ldk - 128 + 64 * i),
                                                                    acc[j][p], 0, 0, 0);
    i8_few_out<MODE, OUT, R>(a, r0, n0, wave, lane, acc, a.a_scales + r0, sums);
}

// Every wave's LDS writes are done; what it asked of memory may still be on its way.
__device__ __forceinline__ void i8_join_barrier()
{
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// ---- numbers --------------------------------------------------------------------------------------------------------

// Eight neighbouring numbers as they lie in memory, of which `left` are in the matrix (the others are 0).
template <typename T>
struct I8Word {
    u4 v[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T* p, int left)
    {
        if (left >= 8) {
#pragma unroll
            for (int i = 0; i < (int)sizeof(T) / 2; ++i) v[i] = *((const u4*)p + i);
        } else {
#pragma unroll
            for (int i = 0; i < (int)sizeof(T) / 2; ++i) v[i] = u4{0u, 0u, 0u, 0u};
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < left) {
                    if constexpr (sizeof(T) == 4) v[i >> 2][i & 3] = __float_as_uint(p[i]);
                    else v[0][i >> 1] |= (unsigned int)p[i] << (16 * (i & 1));
                }
        }
    }
    __device__ __forceinline__ void numbers(float (&f)[8]) const
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (sizeof(T) == 4) f[i] = __uint_as_float(v[i >> 2][i & 3]);
            else f[i] = __uint_as_float(i & 1 ? v[0][i >> 1] & 0xffff0000u : v[0][i >> 1] << 16);
        }
    }
    __device__ __forceinline__ unsigned int top() const
    {
        float f[8];
        numbers(f);
        return mx_top8(f);
    }
    __device__ __forceinline__ u2 codes(float up, unsigned int keep) const
    {
        float f[8];
        numbers(f);
        return u2{i8_pack4(f[0], f[1], f[2], f[3], up) & keep, i8_pack4(f[4], f[5], f[6], f[7], up) & keep};
    }
};

// ROWS (1, 2 or 4, some of which may lie behind the last) of x; each has its share of the work-group's threads, that take eight numbers
// at a time and keep their first HOLD words between the largest magnitude and the codes.  A work-group packs x once and goes through
// every gridDim-th group of 16 rows of W: a wave's turns of all its groups are one stream, asked for two turns ahead, and while one wave joins
// the sums of a group the others are at the next.
template <typename X, I8Mode MODE, typename OUT, int ROWS>
__global__ __launch_bounds__(64 * I8_FEW_WAVES) void i8_four_kernel(I8ProductArgs a, const X* x, int64_t ld_x, int k)
{
    constexpr int PAIR = MODE == I8_PLAIN ? 1 : 2, HOLD = 8 / sizeof(X), T_ROW = 1024 / ROWS;
    extern __shared__ __attribute__((aligned(16))) char lds[];   // [ROWS][ldk] codes
    __shared__ __attribute__((aligned(16))) i4v sums[2][PAIR][I8_FEW_WAVES][64];
    __shared__ unsigned int part[I8_FEW_WAVES];
    __shared__ float scales[16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int row = threadIdx.x / T_ROW, t = threadIdx.x % T_ROW, chunks = (int)(a.ldk >> 3);
    const X* from = x + (int64_t)(row < a.m ? row : a.m - 1) * ld_x;
    I8Word<X> held[HOLD];
    unsigned int top = 0;
#pragma unroll
    for (int i = 0; i < HOLD; ++i) {
        const int c = t + i * T_ROW;
        if (c < chunks) held[i].load(from + 8 * c, k - 8 * c);
    }
#pragma unroll
    for (int i = 0; i < HOLD; ++i)
        if (t + i * T_ROW < chunks) {
            const unsigned int u = held[i].top();
            top = u > top ? u : top;
        }
    // W's first turns are on their way while x is packed
    const int turns_all = (int)(a.ldk / 256), turns = turns_all > wave ? (turns_all - wave + I8_FEW_WAVES - 1) / I8_FEW_WAVES : 0;
    const int groups = ((a.n + 15) / 16 - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x;
    i4v q[2][PAIR][4];
    int ask_turn = 0, ask_group = 0;   // what is asked for next; behind the last turn nothing is
    auto ask = [&](int set) {
        if (ask_group >= groups) return;
        const int n0 = ((int)blockIdx.x + ask_group * (int)gridDim.x) * 16;
        const int64_t at = 256 * (int64_t)(wave + ask_turn * I8_FEW_WAVES);
#pragma unroll
        for (int p = 0; p < PAIR; ++p) {
            const signed char* w = i8_few_row(a, n0, lane, p) + at;
#pragma unroll
            for (int i = 0; i < 4; ++i) q[set][p][i] = *(const i4v*)(w + 64 * i);
        }
        if (++ask_turn == turns) { ask_turn = 0; ++ask_group; }
    };
    if (turns > 0) {
        ask(0);
        ask(1);
    }
    for (int c = t + HOLD * T_ROW; c < chunks; c += T_ROW) {
        I8Word<X> more;
        more.load(from + 8 * c, k - 8 * c);
        const unsigned int u = more.top();
        top = u > top ? u : top;
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const unsigned int o = (unsigned int)__shfl_xor((int)top, d);
        top = o > top ? o : top;
    }
    if (lane == 0) part[wave] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < I8_FEW_WAVES / ROWS; ++i) {
        const unsigned int o = part[row * (I8_FEW_WAVES / ROWS) + i];
        top = o > top ? o : top;
    }
    const I8Scale s = i8_scale(top);
    const unsigned int keep = top >= 0x7f800000u ? 0u : ~0u;
    if (t == 0) scales[row] = s.down;
    char* codes = lds + row * a.ldk;
#pragma unroll
    for (int i = 0; i < HOLD; ++i) {
        const int c = t + i * T_ROW;
        if (c < chunks) *(u2*)(codes + 8 * c) = held[i].codes(s.up, keep);
    }
    for (int c = t + HOLD * T_ROW; c < chunks; c += T_ROW) {
        I8Word<X> more;
        more.load(from + 8 * c, k - 8 * c);
        *(u2*)(codes + 8 * c) = more.codes(s.up, keep);
    }
    __syncthreads();
    // lanes of rows that there are not multiply row 0, and nobody looks at what they get
    const char* y = lds + ((lane & 15) < ROWS ? (lane & 15) : 0) * a.ldk + 16 * (lane >> 4);
    i4v acc[PAIR];
    int turn = 0, group = 0;   // what is multiplied next
    auto clear = [&]() {
#pragma unroll
        for (int p = 0; p < PAIR; ++p) acc[p] = i4v{0, 0, 0, 0};
    };
    // A group's sums meet: all waves' in one of two places, which a wave in turn adds up.  That wave is here again, past the next group's
    // barrier, before anybody writes the same place.
    auto join = [&]() {
        const int n0 = ((int)blockIdx.x + group * (int)gridDim.x) * 16;
        if ((a.ldk & 128) && wave == I8_FEW_WAVES - 1)   // half a turn is left
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const i4v b = *(const i4v*)(y + a.ldk - 128 + 64 * i);
#pragma unroll
                for (int p = 0; p < PAIR; ++p)
                    acc[p] = __builtin_amdgcn_mfma_i32_16x16x64_i8(*(const i4v*)(i8_few_row(a, n0, lane, p) + a.ldk - 128 + 64 * i), b, acc[p], 0, 0, 0);
            }
        i4v(*place)[I8_FEW_WAVES][64] = sums[group & 1];
#pragma unroll
        for (int p = 0; p < PAIR; ++p) place[p][wave][lane] = acc[p];
        i8_join_barrier();
        if (wave == (group & (I8_FEW_WAVES - 1))) {
            i4v v[2] = {place[0][0][lane], place[PAIR - 1][0][lane]};
#pragma unroll 5   // (all of a pair's sums at one time would take 128 registers)
            for (int i = 1; i < I8_FEW_WAVES; ++i) {
                v[0] += place[0][i][lane];
                if constexpr (PAIR == 2) v[1] += place[1][i][lane];
            }
            const int r = lane & 15, c = n0 + 4 * (lane >> 4);
            if (r < a.m && c < a.n) i8_finish<MODE>(a, (OUT*)a.out, r, c, i8_columns<MODE>(a, c), v[0], v[1], scales[r]);
        }
        clear();
        ++group;
        turn = 0;
    };
    auto take = [&](int set) {
        const int at = 256 * (wave + turn * I8_FEW_WAVES);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const i4v b = *(const i4v*)(y + at + 64 * i);
#pragma unroll
            for (int p = 0; p < PAIR; ++p) acc[p] = __builtin_amdgcn_mfma_i32_16x16x64_i8(q[set][p][i], b, acc[p], 0, 0, 0);
        }
        ask(set);
        if (++turn == turns) join();
    };
    clear();
    if (turns == 0) {
        while (group < groups) join();
        return;
    }
    while (group < groups) {
        take(0);
        if (group >= groups) break;
        take(1);
    }
}

template <I8Mode MODE, typename OUT>
static int launch_codes(I8ProductArgs a, int tiles, hipStream_t st)
{
    a.nm = (a.m + 16 * tiles - 1) / (16 * tiles);
    const int64_t groups = (int64_t)((a.n + 15) / 16) * a.nm;
    if (groups > 0x7fffffff) return GVQ_EINVAL;
    if (tiles == 1) hipLaunchKernelGGL((i8_few_kernel<MODE, OUT, 1>), dim3((unsigned)groups), dim3(64 * I8_FEW_WAVES), 0, st, a);
    else hipLaunchKernelGGL((i8_few_kernel<MODE, OUT, 2>), dim3((unsigned)groups), dim3(64 * I8_FEW_WAVES), 0, st, a);
    GVQ_HIP(hipGetLastError());
    return GVQ_OK;
}

int gvq_launch_i8_few(const I8ProductArgs& a, int tiles, I8Mode mode, gvq_dtype_t dtype, hipStream_t st)
{
    if (dtype == GVQ_BF16)
        return mode == I8_PLAIN ? launch_codes<I8_PLAIN, unsigned short>(a, tiles, st)
                                : mode == I8_GATED ? launch_codes<I8_GATED, unsigned short>(a, tiles, st) : launch_codes<I8_INNER, unsigned short>(a, tiles, st);
    return mode == I8_PLAIN ? launch_codes<I8_PLAIN, float>(a, tiles, st)
                            : mode == I8_GATED ? launch_codes<I8_GATED, float>(a, tiles, st) : launch_codes<I8_INNER, float>(a, tiles, st);
}

#define I8_FOUR_LDS (64 * 1024)   // of codes, beside 64 KB of sums

template <typename X, I8Mode MODE, typename OUT, int ROWS>
static int launch_numbers(const I8ProductArgs& a, const void* x, int64_t ld_x, int k, hipStream_t st)
{
    static gvq_once_per_device lds;
    int dev;
    GVQ_HIP(hipGetDevice(&dev));
    const int rc = lds.call(dev, [] {
        GVQ_HIP(hipFuncSetAttribute((const void*)i8_four_kernel<X, MODE, OUT, ROWS>, hipFuncAttributeMaxDynamicSharedMemorySize, I8_FOUR_LDS));
        return (int)GVQ_OK;
    });
    if (rc != GVQ_OK) return rc;
    const int groups = (a.n + 15) / 16;
    hipLaunchKernelGGL((i8_four_kernel<X, MODE, OUT, ROWS>), dim3((unsigned)(groups < 256 ? groups : 256)), dim3(64 * I8_FEW_WAVES), (unsigned)(ROWS * a.ldk), st, a,
                       (const X*)x, ld_x, k);
    GVQ_HIP(hipGetLastError());
    return GVQ_OK;
}
template <typename X, I8Mode MODE, typename OUT>
static int launch_rows(const I8ProductArgs& a, const void* x, int64_t ld_x, int k, hipStream_t st)
{
    return a.m == 1 ? launch_numbers<X, MODE, OUT, 1>(a, x, ld_x, k, st)
                    : a.m == 2 ? launch_numbers<X, MODE, OUT, 2>(a, x, ld_x, k, st) : launch_numbers<X, MODE, OUT, 4>(a, x, ld_x, k, st);
}
template <typename X, typename OUT>
static int launch_numbers_mode(const I8ProductArgs& a, const void* x, int64_t ld_x, int k, I8Mode mode, hipStream_t st)
{
    return mode == I8_PLAIN ? launch_rows<X, I8_PLAIN, OUT>(a, x, ld_x, k, st) : launch_rows<X, I8_GATED, OUT>(a, x, ld_x, k, st);
}

// Against a launch that quantises and another that multiplies (us, one and four bf16 rows, numbers in and out): 1000, 1000 4.0 and 6.1, 4.4 and 6.4; 4096, 4096 5.0
// and 7.9, 5.6 and 8.4; 25088, 4096 20 and 29, 30.5 and 30.4; gated 4096, 8192 15.8 and 19.8, 16.8 and 20.2; at worst 4096, 25088 22.7 and 21.7, 24.0 and 22.1, where
// each unit goes through many groups.  At most 64 KB of codes: LDS has to hold them beside as much of sums.
bool gvq_i8_few_numbers_takes(const void* x, gvq_dtype_t x_dtype, int64_t rows, int64_t ld_x, int64_t k, I8Mode mode)
{
    const int64_t row = rows > 1 ? ld_x * (x_dtype == GVQ_BF16 ? 2 : 4) : 0;   // a single row is aligned where it begins
    if (rows > 4 || mode == I8_INNER || (((uintptr_t)x | (uintptr_t)row) & 15) != 0) return false;
    return (rows > 2 ? 4 : rows) * gvq_i8_row_bytes(k) <= I8_FOUR_LDS;
}

int gvq_launch_i8_few_numbers(I8ProductArgs a, const void* x, gvq_dtype_t x_dtype, int64_t ld_x, int64_t k, I8Mode mode, gvq_dtype_t dtype,
                              hipStream_t st)
{
    const int64_t es = dtype == GVQ_BF16 ? 2 : 4;
    a.words = (((uintptr_t)a.out | (uintptr_t)(a.ld * es)) & (uintptr_t)(4 * es - 1)) == 0;
    if (x_dtype == GVQ_BF16)
        return dtype == GVQ_BF16 ? launch_numbers_mode<unsigned short, unsigned short>(a, x, ld_x, (int)k, mode, st)
                                 : launch_numbers_mode<unsigned short, float>(a, x, ld_x, (int)k, mode, st);
    return dtype == GVQ_BF16 ? launch_numbers_mode<float, unsigned short>(a, x, ld_x, (int)k, mode, st)
                             : launch_numbers_mode<float, float>(a, x, ld_x, (int)k, mode, st);
}
