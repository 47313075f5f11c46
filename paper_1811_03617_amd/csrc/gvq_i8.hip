// Matrices into 8-bit integers with a scale for every row, of the matrix or of its transpose, and back.
//
// A row's scale is its largest magnitude / 127, so that a row has to be seen whole before its first code.  Rows: one pass, a row's numbers stay in
// registers between the two.  Columns of few rows too: a work-group holds a few columns whole.  Of more rows it would hold pieces of lines, so their
// largest magnitudes come first, of runs of rows that work-groups take side by side, and then the codes, turned through LDS so that each column's leave in
// whole lines.
// Bound: memory; columns of many rows read the matrix twice; below that a launch (500 x 4096 and 500 x 1000 fp32, the first by columns, the second both ways,
// 8.8 us in one launch).  8192 x 4096 bf16 rows 20 us (5.0 TB/s read and written, a plain copy's 5.1), fp32 30; 4096 x 25088 bf16
// columns 35 + 72 (5.9 and 4.3 TB/s: lines of codes that lie a column apart).
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

// The `block`-th work-group's rows, TEAMS times four of them, a wave each, or TEAMS, four waves each.  Eight neighbouring numbers a thread at a time,
// HOLD times eight in registers; what is behind that is read again.
template <typename T, int W, int HOLD, int TEAMS = 1>
__device__ __forceinline__ void i8_rows(const I8QuantArgs& a, int block, unsigned int* part)
{
    constexpr int PER = 4 * TEAMS / W, T_ROW = 64 * W;
    const int t = threadIdx.x % T_ROW;
    const int64_t r = (int64_t)block * PER + threadIdx.x / T_ROW;
    const bool there = (W > 1 && TEAMS == 1) || r < a.rows;
    if (W == 1 && !there) return;
    const T* x = (const T*)a.x + r * a.ld;
    const int chunks = there ? (int)(a.ldc >> 3) : 0;
    float v[HOLD][8];
    unsigned int top = 0;
#pragma unroll
    for (int i = 0; i < HOLD; ++i) {
        const int c = t + i * T_ROW;
        if (c < chunks) mx_load8(x + 8 * (int64_t)c, a.words != 0, a.cols - 8 * (int64_t)c, v[i]);
    }
#pragma unroll
    for (int i = 0; i < HOLD; ++i)
        if (t + i * T_ROW < chunks) {
            const unsigned int u = mx_top8(v[i]);
            top = u > top ? u : top;
        }
    for (int c = t + HOLD * T_ROW; c < chunks; c += T_ROW) {
        float f[8];
        mx_load8(x + 8 * (int64_t)c, a.words != 0, a.cols - 8 * (int64_t)c, f);
        const unsigned int u = mx_top8(f);
        top = u > top ? u : top;
    }
    top = wave_max(top);
    if constexpr (W > 1) {
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = top;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const unsigned int o = part[threadIdx.x / T_ROW * W + i];
            top = o > top ? o : top;
        }
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
    if (there && t == 0) a.scales[r] = s.down;
}

// ---- columns ------------------------------------------------------------------------------------------------------

// A number's bits as fp32 has them.
__device__ __forceinline__ unsigned int i8_bits(float v) { return __float_as_uint(v); }
__device__ __forceinline__ unsigned int i8_bits(unsigned short v) { return (unsigned int)v << 16; }
// 16 bytes, past the caches or through them.
template <bool PAST>
__device__ __forceinline__ u4 i8_word(const void* p)
{
    if constexpr (PAST) return stream_load((const u4*)p);
    else return *(const u4*)p;
}
__device__ __forceinline__ void i8_raise(unsigned int& top, unsigned int u) { top = u > top ? u : top; }
template <typename T>
__device__ __forceinline__ void i8_raise_word(unsigned int (&top)[16 / sizeof(T)], const u4& v)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
            i8_raise(top[i], v[i] & 0x7fffffffu);
        } else {
            i8_raise(top[2 * i], v[i] << 16 & 0x7fffffffu);
            i8_raise(top[2 * i + 1], v[i] & 0x7fff0000u);
        }
    }
}

// Row r's word of columns from c on; what is not in the matrix is 0.
template <typename T, bool PAST>
__device__ __forceinline__ u4 i8_word_at(const I8QuantArgs& a, int64_t r, int64_t c)
{
    constexpr int PER = 16 / sizeof(T);
    u4 v = {0u, 0u, 0u, 0u};
    if (a.words && c + PER <= a.cols) {
        if (r < a.rows) v = i8_word<PAST>((const T*)a.x + r * a.ld + c);
    } else if (c < a.cols) {
        // (from addresses that are always there, so that none of these loads waits for another)
        const T* p = (const T*)a.x + (r < a.rows ? r : a.rows - 1) * a.ld;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const unsigned int u = i8_bits(p[c + i < a.cols ? c + i : a.cols - 1]), in = r < a.rows && c + i < a.cols ? u : 0u;
            if constexpr (sizeof(T) == 4) v[i] = in;
            else v[i >> 1] |= i & 1 ? in : in >> 16;
        }
    }
    return v;
}
// The four codes of column i of four rows' words.
template <typename T>
__device__ __forceinline__ unsigned int i8_pack_column(const u4 (&word)[4], int i, float up)
{
    float v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if constexpr (sizeof(T) == 4) v[k] = __uint_as_float(word[k][i]);
        else v[k] = __uint_as_float(i & 1 ? word[k][i >> 1] & 0xffff0000u : word[k][i >> 1] << 16);
    }
    return i8_pack4(v[0], v[1], v[2], v[3], up);
}

// Largest magnitudes of a run of rows: a work-group takes 64 lanes' words of columns, its waves every fourth row, eight at a time.
// part: [4][64][PER + 1].
template <typename T>
__device__ __forceinline__ void i8_peaks(const I8QuantArgs& a, int block, unsigned int* part)
{
    constexpr int PER = 16 / sizeof(T);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int stripe = block % a.stripes, chunk = block / a.stripes;
    const int64_t c = ((int64_t)stripe * 64 + lane) * PER, r0 = (int64_t)chunk * a.chunk_rows;
    const int64_t r1 = r0 + a.chunk_rows < a.rows ? r0 + a.chunk_rows : a.rows;
    unsigned int top[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) top[i] = 0;
    if (a.words) {
        const T* x = (const T*)a.x + c;
        int64_t r = r0 + wave;
        if (c + PER <= a.cols) {
            auto eight = [&](auto past) {
                for (; r + 28 < r1; r += 32) {
                    u4 v[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] = i8_word<decltype(past)::value>(x + (r + 4 * i) * a.ld);
#pragma unroll
                    for (int i = 0; i < 8; ++i) i8_raise_word<T>(top, v[i]);
                }
            };
            if (a.past) eight(std::true_type{});
            else eight(std::false_type{});
            for (; r < r1; r += 4) i8_raise_word<T>(top, *(const u4*)(x + r * a.ld));
        } else if (c < a.cols) {
            for (; r < r1; r += 4)
#pragma unroll
                for (int i = 0; i < PER; ++i)
                    if (c + i < a.cols) i8_raise(top[i], i8_bits(x[r * a.ld + i]) & 0x7fffffffu);
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) part[(wave * 64 + lane) * (PER + 1) + i] = top[i];
    } else {
        // rows that start anywhere: a lane has one number of each 64, next to its neighbours'
        const int first = stripe * 64 * PER + lane, last = (int)a.cols - 1;
#pragma unroll 2
        for (int64_t r = r0 + wave; r < r1; r += 4) {
            const T* x = (const T*)a.x + r * a.ld;
#pragma unroll
            for (int i = 0; i < PER; ++i) i8_raise(top[i], i8_bits(x[first + 64 * i < last ? first + 64 * i : last]) & 0x7fffffffu);
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int e = 64 * i + lane;
            part[(wave * 64 + e / PER) * (PER + 1) + e % PER] = top[i];
        }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < 64 * PER; e += I8Q_THREADS) {
        const int64_t cc = (int64_t)stripe * 64 * PER + e;
        if (cc >= a.cols) break;
        unsigned int m = 0;
#pragma unroll
        for (int w = 0; w < 4; ++w) i8_raise(m, part[(w * 64 + e / PER) * (PER + 1) + e % PER]);
        a.peaks[(int64_t)chunk * a.cols + cc] = m;
    }
}

template <typename T>
constexpr int I8_COLUMNS = 256 / sizeof(T);   // of a tile
// 128 rows of 256 bytes: a thread takes four rows of one word of columns, packs each column's four codes, and the tile leaves as
// 128 bytes of each column.  In LDS a column is eight pieces of 16 bytes, exchanged by the column's group of eight.
template <typename T, bool PAST>
__device__ __forceinline__ void i8_columns_of(const I8QuantArgs& a, int block, unsigned int* turn, unsigned int* tops)
{
    constexpr int PER = 16 / sizeof(T), COLS = I8_COLUMNS<T>, QUADS = I8Q_THREADS / 16, TURNS = 32 / QUADS;   // quads of rows at a time
    constexpr int PARTS = I8Q_THREADS / COLS;   // threads that look for one column's largest magnitude
    int down, over;
    tile_at(block, (int)(a.ldct >> 7), a.across, a.band, down, over);
    const int64_t r0 = (int64_t)down * 128, c0 = (int64_t)over * COLS;
    const int w = threadIdx.x & 15, quad0 = threadIdx.x >> 4;
    const int64_t c = c0 + w * PER;
    // the numbers first, then what they are divided by
    u4 word[TURNS][4];
#pragma unroll
    for (int p = 0; p < TURNS; ++p)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int64_t r = r0 + 4 * (quad0 + p * QUADS) + k;
            word[p][k] = i8_word_at<T, PAST>(a, r, c);
        }
    {
        const int col = threadIdx.x % COLS, first = threadIdx.x / COLS;
        unsigned int top = 0;
        if (c0 + col < a.cols) {
#pragma unroll
            for (int k = 0; k < I8_CHUNKS / PARTS; ++k)
                if (first + PARTS * k < a.chunks) i8_raise(top, a.peaks[(int64_t)(first + PARTS * k) * a.cols + c0 + col]);
        }
        tops[first * COLS + col] = top;
    }
    __syncthreads();
    float up[PER];
    unsigned int keep[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int col = w * PER + i;
        unsigned int top = tops[col];
#pragma unroll
        for (int k = 1; k < PARTS; ++k) i8_raise(top, tops[k * COLS + col]);
        const I8Scale s = i8_scale(top);
        up[i] = s.up;
        keep[i] = top >= 0x7f800000u ? 0u : ~0u;
        if (r0 == 0 && quad0 == 0 && c + i < a.cols) a.scales_t[c + i] = s.down;
    }
#pragma unroll
    for (int p = 0; p < TURNS; ++p) {
        const int quad = quad0 + p * QUADS;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int col = w * PER + i;
            turn[col * 32 + ((quad >> 2 ^ (col >> 3 & 7)) << 2) + (quad & 3)] = i8_pack_column<T>(word[p], i, up[i]) & keep[i];
        }
    }
    __syncthreads();
#pragma unroll
    for (int p = 0; p < COLS / 32; ++p) {
        const int e = threadIdx.x + p * I8Q_THREADS, col = e >> 3, piece = e & 7;
        u4* to = (u4*)(a.codes_t + (c0 + col) * a.ldct + r0 + 16 * piece);
        const u4 v = *(const u4*)(turn + col * 32 + ((piece ^ (col >> 3 & 7)) << 2));
        if (c0 + col < a.cols) {
            if constexpr (PAST) stream_store(to, v);
            else *to = v;
        }
    }
}

constexpr int I8_ACROSS = 4;              // words of columns,
constexpr int I8_DOWN = 1024 / I8_ACROSS; // and rows of 256 threads
// At most I8_DOWN TEAMS rows: a work-group holds I8_ACROSS words' columns whole, four rows of one word to a thread.  In LDS a column has a byte for each
// of the rows that there could be, in pieces of 16 that are exchanged by the word that the column is in.
template <typename T, int TEAMS>
__device__ __forceinline__ void i8_columns_once(const I8QuantArgs& a, int block, unsigned int* turn, unsigned int* tops)
{
    constexpr int PER = 16 / sizeof(T), COLS = I8_ACROSS * PER, COLUMN = I8_DOWN / 4 * TEAMS, PIECES = COLUMN / 4;   // words and pieces of a column
    constexpr int TURN = 16 / I8_ACROSS;   // (a wave's 64 words go to all banks)
    const int w = threadIdx.x % I8_ACROSS, quad = threadIdx.x / I8_ACROSS, wave = threadIdx.x >> 6;
    const int64_t c0 = (int64_t)block * COLS, c = c0 + w * PER;
    const bool inside = a.words && c0 + COLS <= a.cols;   // (the same for all threads)
    u4 word[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int64_t r = 4 * quad + k;
        if (inside) {
            word[k] = i8_word<false>((const T*)a.x + (r < a.rows ? r : a.rows - 1) * a.ld + c);
            if (r >= a.rows) word[k] = u4{0u, 0u, 0u, 0u};
        } else {
            word[k] = i8_word_at<T, false>(a, r, c);
        }
    }
    unsigned int top[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) top[i] = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) i8_raise_word<T>(top, word[k]);
#pragma unroll
    for (int i = 0; i < PER; ++i)
#pragma unroll
        for (int d = I8_ACROSS; d < 64; d *= 2) i8_raise(top[i], (unsigned int)__shfl_xor((int)top[i], d));
    if ((threadIdx.x & 63) < I8_ACROSS)
#pragma unroll
        for (int i = 0; i < PER; ++i) tops[wave * COLS + w * PER + i] = top[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int col = w * PER + i;
        unsigned int t = tops[col];
#pragma unroll
        for (int k = 1; k < 4 * TEAMS; ++k) i8_raise(t, tops[k * COLS + col]);
        const I8Scale s = i8_scale(t);
        const unsigned int keep = t >= 0x7f800000u ? 0u : ~0u;
        if (quad == 0 && c + i < a.cols) a.scales_t[c + i] = s.down;
        turn[col * COLUMN + ((quad >> 2 ^ (w * TURN & (PIECES - 1))) << 2) + (quad & 3)] = i8_pack_column<T>(word, i, s.up) & keep;
    }
    __syncthreads();
    const int pieces = (int)(a.ldct >> 4);
#pragma unroll
    for (int p = 0; p < COLS * PIECES / (256 * TEAMS); ++p) {
        const int e = threadIdx.x + p * 256 * TEAMS, col = e / PIECES, piece = e % PIECES;
        if (c0 + col < a.cols && piece < pieces)
            *(u4*)(a.codes_t + (c0 + col) * a.ldct + 16 * piece) = *(const u4*)(turn + col * COLUMN + ((piece ^ (col / PER * TURN & (PIECES - 1))) << 2));
    }
}

// Columns read their matrix twice.  What is larger than this goes past the caches both times (4096 x 25088 bf16 numbers that no cache
// holds: largest magnitudes 35 us and codes 72, through the caches 77 and 73), what is smaller is mostly found there the second time (past them and
// through them, us: 4096 x 1000 fp32 14.0 and 12.5, bf16 17.0 and 14.1; 4096 x 4096 fp32 36 and 32, bf16 22 and 24).
#define I8_PAST (64 << 20)

// ---- one or two matrices --------------------------------------------------------------------------------------------

struct I8Two {
    I8QuantArgs a[2];
};

// Rows of both and columns held whole: one launch.
template <typename T, int HOLD, int TEAMS>
__global__ __launch_bounds__(256 * TEAMS) void i8_once_kernel(I8Two m)
{
    constexpr int COLS = I8_ACROSS * 16 / sizeof(T);
    __shared__ __attribute__((aligned(16))) unsigned int turn[COLS * I8_DOWN / 4 * TEAMS];
    __shared__ unsigned int tops[4 * TEAMS * COLS];
    int block = blockIdx.x;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const I8QuantArgs& a = m.a[i];
        if (block < a.column_blocks) {
            i8_columns_once<T, TEAMS>(a, block, turn, tops);
            return;
        }
        block -= a.column_blocks;
        if (block < a.row_blocks) {
            if (a.ldc <= 2048) i8_rows<T, 1, 4, TEAMS>(a, block, tops);
            else i8_rows<T, 4, HOLD, TEAMS>(a, block, tops);
            return;
        }
        block -= a.row_blocks;
    }
}
// First the rows of both and the columns' largest magnitudes: none needs another's result.  HOLD: what the longer rows keep.
template <typename T, int HOLD>
__global__ __launch_bounds__(I8Q_THREADS) void i8_rows_kernel(I8Two m)
{
    __shared__ unsigned int part[4 * 64 * (16 / sizeof(T) + 1)];
    int block = blockIdx.x;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const I8QuantArgs& a = m.a[i];
        if (block < a.row_blocks) {
            if (a.ldc <= 2048) i8_rows<T, 1, 4>(a, block, part);
            else i8_rows<T, 4, HOLD>(a, block, part);
            return;
        }
        block -= a.row_blocks;
        if (block < a.peak_blocks) {
            i8_peaks<T>(a, block, part);
            return;
        }
        block -= a.peak_blocks;
    }
}
// Then the columns' codes.
template <typename T, bool PAST>
__global__ __launch_bounds__(I8Q_THREADS) void i8_columns_kernel(I8Two m)
{
    __shared__ __attribute__((aligned(16))) unsigned int turn[I8_COLUMNS<T> * 32];
    __shared__ unsigned int tops[I8Q_THREADS];
    const int block = tile_of_block(blockIdx.x, gridDim.x);
    if (block < m.a[0].column_blocks) i8_columns_of<T, PAST>(m.a[0], block, turn, tops);
    else i8_columns_of<T, PAST>(m.a[1], block - m.a[0].column_blocks, turn, tops);
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

template <typename T, int TEAMS>
static int launch_once(I8Two m, bool longer, hipStream_t st)
{
    constexpr int PER = 16 / sizeof(T);
    int64_t groups = 0;
    for (I8QuantArgs& a : m.a) {
        if (a.codes) a.row_blocks = (int)(((a.ldc <= 2048 ? (a.rows + 3) / 4 : a.rows) + TEAMS - 1) / TEAMS);
        if (a.codes_t) a.column_blocks = (int)((a.cols + I8_ACROSS * PER - 1) / (I8_ACROSS * PER));
        groups += a.row_blocks + a.column_blocks;
    }
    if (longer) hipLaunchKernelGGL((i8_once_kernel<T, 8, TEAMS>), dim3((unsigned)groups), dim3(256 * TEAMS), 0, st, m);
    else hipLaunchKernelGGL((i8_once_kernel<T, 4, TEAMS>), dim3((unsigned)groups), dim3(256 * TEAMS), 0, st, m);
    GVQ_HIP(hipGetLastError());
    return GVQ_OK;
}

template <typename T>
static int launch_quantize(const I8QuantArgs* matrices, int n, hipStream_t st)
{
    constexpr int PER = 16 / sizeof(T);
    I8Two m{};
    int64_t first = 0, second = 0, deepest = 0, largest = 0;   // (rows and numbers of what is wanted by columns)
    bool longer = false, past = false;
    for (int i = 0; i < n; ++i) {
        I8QuantArgs& a = m.a[i];
        a = matrices[i];
        a.ldc = gvq_i8_row_bytes(a.cols);
        a.ldct = gvq_i8_row_bytes(a.rows);
        a.words = (((uintptr_t)a.x | (uintptr_t)(a.ld * sizeof(T))) & 15) == 0;
        longer |= a.codes && a.ldc > 8192;
        if (a.codes_t) {
            deepest = a.rows > deepest ? a.rows : deepest;
            largest = a.rows * a.cols > largest ? a.rows * a.cols : largest;
        }
    }
    // Columns of few rows in one launch with the rows, or in two (us, a layer's gradients: x's columns and dy both ways): 16 x 4096 and 4096 fp32 7.7 and 12.8,
    // bf16 9.8 and 15; 500 x 4096 and 1000 8.8 and 14, 11 and 18; 1024 x 4096 and 4096 22 and 26, 21 and 22; 512 x 25088 and 4096 30 and 32, 27 and 29;
    // but 1024 x 25088 bf16 alone 40 and 29: pieces of 64 bytes of a row are slower where memory is what bounds it.
    if (deepest > 0 && deepest <= I8_DOWN) return launch_once<T, 1>(m, longer, st);
    if (deepest > 0 && deepest <= 2 * I8_DOWN) return launch_once<T, 2>(m, longer, st);
    if (deepest > 0 && deepest <= 4 * I8_DOWN && largest <= 1 << 23) return launch_once<T, 4>(m, longer, st);
    for (I8QuantArgs& a : m.a) {
        // a wave a row, or four (8192 rows of bf16, us: of 1024 numbers 6.6 and 11.0, of 2048 12.4 and 14.7, of 4096 22.7 and 21.3)
        if (a.codes) a.row_blocks = (int)(a.ldc <= 2048 ? (a.rows + 3) / 4 : a.rows);
        if (a.codes_t) {
            a.chunk_rows = gvq_i8_chunk_rows(a.rows);
            a.chunks = (int)((a.rows + a.chunk_rows - 1) / a.chunk_rows);
            a.stripes = (int)((a.cols + 64 * PER - 1) / (64 * PER));
            a.peak_blocks = a.stripes * a.chunks;
            a.across = (int)((a.cols + I8_COLUMNS<T> - 1) / I8_COLUMNS<T>);
            past |= a.rows * a.cols * (int64_t)sizeof(T) > I8_PAST;
            const int64_t tiles = a.across * (a.ldct >> 7);
            if (tiles > 0x3fffffff) return GVQ_EINVAL;
            a.column_blocks = (int)tiles;
            a.band = 16;
        }
        first += a.row_blocks + a.peak_blocks;
        second += a.column_blocks;
    }
    for (I8QuantArgs& a : m.a) a.past = past;
    // rows of up to 16384 numbers stay in registers; the shorter ones' kernel has half of those, and more waves (with all and with half of them, us:
    // 8192 x 4096 bf16 25 and 21, 4096 x 8192 fp32 34 and 32; 4096 x 16384 39 and 48, fp32 66 and 89)
    if (longer) hipLaunchKernelGGL((i8_rows_kernel<T, 8>), dim3((unsigned)first), dim3(I8Q_THREADS), 0, st, m);
    else hipLaunchKernelGGL((i8_rows_kernel<T, 4>), dim3((unsigned)first), dim3(I8Q_THREADS), 0, st, m);
    GVQ_HIP(hipGetLastError());
    if (second > 0) {
        if (past) hipLaunchKernelGGL((i8_columns_kernel<T, true>), dim3((unsigned)second), dim3(I8Q_THREADS), 0, st, m);
        else hipLaunchKernelGGL((i8_columns_kernel<T, false>), dim3((unsigned)second), dim3(I8Q_THREADS), 0, st, m);
        GVQ_HIP(hipGetLastError());
    }
    return GVQ_OK;
}

int gvq_launch_i8_quantize(const I8QuantArgs* matrices, int n, gvq_dtype_t dtype, hipStream_t st)
{
    return dtype == GVQ_BF16 ? launch_quantize<unsigned short>(matrices, n, st) : launch_quantize<float>(matrices, n, st);
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
