// Products of 8-bit integers, C = A B^T with a scale for every row of A and of B, on the int8 matrix pipe (v_mfma_i32_16x16x64_i8: exact
// products, exact 32-bit sums; (int)sum is rounded to fp32 once and multiplied by the product of both scales).  Gated: the second
// operand's rows are a gate's and another projection's, a wave has both sums of the same places, and what leaves is act(g) u, or, given the
// gradient of that, the gradients of g and u.
// Bound: the matrix pipe, at the rate that its power leaves.  The instruction alone, operands of normal numbers in registers, does 4.08 PFLOP/s
// (the 32 x 32 one 3.5); 4096 x 4096 x 16384 takes 181 us (3.0), and with the reads of the operands left out in a copy of the kernel 163 without the
// copies into LDS, 173 and 176 without the fragments of A or B, 133 without either.  Counters of the kernel itself: the clock at 1.86 of 2.4 GHz and the
// pipe busy 74 % of the cycles there, 2.03 GHz and 58 % on 8192 x 4096 x 4096, where a tile's beginning and end count four times as much.
// 8192 x 4096 x 4096 106 us (2.6), 8192^3 379 (2.9); with the quantiser's 20, gated 8192 x (2 * 8192) x 4096 443 to 453, its inner gradient 562.
#include "gvq_i8.h"
#include "gvq_i8_plan.h"
#include "gvq_tile.h"

#define I8_STEP 128   // bytes of a row per step: a line

// BM rows of A by BN of B, WM x WN waves.  A step's rows lie in LDS one behind the other, row r's piece c of 16 bytes in place
// c ^ (r & 7): the 16 lanes whose reads are served together then cover all banks.
// PARTS: teams of WM x WN waves that take the steps in turn, each with stages of its own; their sums, whole numbers, are added at the end.  One team
// alone on a compute unit waits for its barriers and reads most of the time.
template <int BM_, int BN_, int WM_, int WN_, int STAGES_, int PARTS_ = 1>
struct I8Shape {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, STAGES = STAGES_, PARTS = PARTS_;
    static constexpr int WAVES = WM * WN, THREADS = 64 * WAVES * PARTS, MI = BM / WM / 16, NI = BN / WN / 16;
    static constexpr int STAGE = (BM + BN) * I8_STEP, LDS = STAGE * STAGES * PARTS;
    static constexpr int GROUPS = (BM + BN) / 8, COPIES = GROUPS / WAVES;   // 1 KB copies of a step: eight rows each
    static_assert(GROUPS % WAVES == 0 && BM % 16 == 0 && LDS <= 160 * 1024 && COPIES * STAGES < 64, "whole copies, LDS and vmcnt");
    static_assert((PARTS - 1) * WAVES * MI * NI * 1024 <= LDS && WAVES * 4096 <= LDS, "the teams' sums, then the results");
};

// Row of B that the tile's row j is.  Gated: groups of 16 of the gate's and of the other's in turn.
template <I8Mode MODE>
__device__ __forceinline__ int64_t i8_row_of_b(int tn, int BN, int j, int n)
{
    if (MODE == I8_PLAIN) {
        const int r = tn * BN + j;
        return r < n ? r : n - 1;
    }
    const int r = tn * (BN / 2) + (j >> 5) * 16 + (j & 15);
    return (int64_t)(r < n ? r : n - 1) + ((j >> 4) & 1 ? n : 0);
}

// The first team's waves return true, with the sums.
template <typename T, I8Mode MODE>
__device__ __forceinline__ bool i8_tile(const I8ProductArgs& a, int tm, int tn, char* lds, i4v (&acc)[T::MI][T::NI])
{
    const int lane = threadIdx.x & 63, every = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), team = T::PARTS > 1 ? every / T::WAVES : 0,
              wave = T::PARTS > 1 ? every % T::WAVES : every;
    const int wm = wave / T::WN, wn = wave % T::WN, steps = (int)(a.ldk / I8_STEP);
    char* mine = lds + team * T::STAGES * T::STAGE;
    const unsigned int lds0 = lds_offset(mine);
    const char* base[T::COPIES];
    unsigned int voff[T::COPIES];
#pragma unroll
    for (int i = 0; i < T::COPIES; ++i) {
        const int j0 = (wave * T::COPIES + i) * 8, j = j0 + (lane >> 3), piece = (lane & 7) ^ (lane >> 3);
        if (j0 < T::BM) {
            const int64_t first = (int64_t)tm * T::BM + j0 < a.m ? (int64_t)tm * T::BM + j0 : a.m - 1;
            const int64_t r = (int64_t)tm * T::BM + j < a.m ? (int64_t)tm * T::BM + j : a.m - 1;
            base[i] = (const char*)a.a + first * a.ldk;
            voff[i] = (unsigned int)((r - first) * a.ldk) + 16 * piece;
        } else {
            const int64_t first = i8_row_of_b<MODE>(tn, T::BN, j0 - T::BM, a.n), r = i8_row_of_b<MODE>(tn, T::BN, j - T::BM, a.n);
            base[i] = (const char*)a.b + first * a.ldk;
            voff[i] = (unsigned int)((r - first) * a.ldk) + 16 * piece;
        }
    }
    // the team's turns: its t-th step is step t PARTS + team
    auto issue = [&](int t) {
        const unsigned int to = lds0 + (unsigned int)(t % T::STAGES) * T::STAGE + (unsigned int)(wave * T::COPIES) * 1024;
#pragma unroll
        for (int i = 0; i < T::COPIES; ++i) copy_rows_to_lds(base[i] + (int64_t)(t * T::PARTS + team) * I8_STEP, voff[i], to + i * 1024);
    };
    const int row = lane & 15, turns = (steps + T::PARTS - 1) / T::PARTS, own = steps > team ? (steps - team + T::PARTS - 1) / T::PARTS : 0;
    for (int t = 0; t < T::STAGES - 1 && t < own; ++t) issue(t);
    for (int t = 0; t < turns; ++t) {
        // this wave's copies of its step have arrived, and then everybody's; everybody is done with the place that is asked for next
        if (t + T::STAGES - 1 <= own) tile_barrier<T::COPIES * (T::STAGES - 2)>();
        else tile_barrier<0>();
        if (t + T::STAGES - 1 < own) issue(t + T::STAGES - 1);
        if (T::PARTS > 1 && t >= own) continue;
        const char* st = mine + (t % T::STAGES) * T::STAGE;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int piece = ((4 * k + (lane >> 4)) ^ (row & 7)) * 16;
            i4v fb[T::NI];
#pragma unroll
            for (int ni = 0; ni < T::NI; ++ni) fb[ni] = *(const i4v*)(st + (T::BM + (wn * T::NI + ni) * 16 + row) * I8_STEP + piece);
#pragma unroll
            for (int mi = 0; mi < T::MI; ++mi) {
                const i4v fa = *(const i4v*)(st + ((wm * T::MI + mi) * 16 + row) * I8_STEP + piece);
#pragma unroll
                for (int ni = 0; ni < T::NI; ++ni) acc[mi][ni] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[ni], fa, acc[mi][ni], 0, 0, 0);
            }
        }
    }
    if constexpr (T::PARTS > 1) {
        i4v* sums = (i4v*)lds + lane;
        __syncthreads();
        if (team > 0)
#pragma unroll
            for (int mi = 0; mi < T::MI; ++mi)
#pragma unroll
                for (int ni = 0; ni < T::NI; ++ni) sums[(((team - 1) * T::WAVES + wave) * T::MI * T::NI + mi * T::NI + ni) * 64] = acc[mi][ni];
        __syncthreads();
        if (team == 0)
#pragma unroll
            for (int p = 0; p < T::PARTS - 1; ++p)
#pragma unroll
                for (int mi = 0; mi < T::MI; ++mi)
#pragma unroll
                    for (int ni = 0; ni < T::NI; ++ni) acc[mi][ni] += sums[((p * T::WAVES + wave) * T::MI * T::NI + mi * T::NI + ni) * 64];
    }
    return team == 0;
}

// 256 x 256 by eight waves in two halves that take turns: while the four of one half multiply, one on each SIMD, the four of the other
// read fragments and ask for rows, and a barrier ends every turn of the two.  A step's products of a wave (128 x 64, 128 numbers of the
// sum) are four turns of 16 instructions, of half of its rows (A0, A1) and half of its columns each; F is the half of the columns that the
// step begins with, B0 and B1 by turns, G the other.  What a turn multiplies was asked of LDS one turn earlier at the latest, so that no
// turn waits for a read that it has just begun.  Each quarter of a stage (the rows of A0, A1, F or G of all waves, 16 KB) is in
// registers two turns after its read began, and its place then takes the rows of two steps later.
//   turn (step s)   reads        asks for     multiplies
//   0               G (s)        A0 (s + 2)   A0 F
//   1               A1 (s)       F (s + 2)    A0 G
//   2               A0 (s + 1)   G (s + 2)    A1 G
//   3               F (s + 1)    A1 (s + 2)   A1 F
// Five quarters, ten copies of a wave, are younger than the one that the next turn reads.
// Tried: work-groups that stay and ask for the next tile while they hand out the last one (no faster, and gated ones spill), reads spread over both turns of
// a pair (2 % slower), a turn's last products behind the barrier (8 to 17 % slower), all eight waves in step (no room for the reads ahead), and
// four waves of 128 x 128 each, one on a SIMD, that read a third less from LDS: 4096 x 4096 x 16384 203 us instead of 182, as fast as this one only without
// copies (163 both), which then hold up the one wave that multiplies.
struct I8Pong {
    static constexpr int BM = 256, BN = 256, WM = 2, WN = 4, WAVES = 8, THREADS = 512, MI = 8, NI = 4;
    static constexpr int STAGE = 512 * I8_STEP, LDS = 2 * STAGE;
};

// All but the youngest N copies are there, all but the youngest R reads in registers; then the other half's too.
template <int N, int R>
__device__ __forceinline__ void i8_turn_over()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(%1)\n\ts_barrier" ::"n"(N), "n"(R) : "memory");
}

template <I8Mode MODE>
__device__ __forceinline__ void i8_tile_pong(const I8ProductArgs& a, int tm, int tn, char* lds, i4v (&acc)[8][4])
{
    typedef I8Pong T;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int wm = wave / T::WN, wn = wave % T::WN, steps = (int)(a.ldk / I8_STEP);
    const unsigned int lds0 = lds_offset(lds);
    if (steps <= 0) return;
    // quarters: 0 A0, 1 B0, 2 B1, 3 A1; a wave has two of the 16 copies of eight rows of each
    const char* base[4][2];
    unsigned int voff[4][2], to[4][2];
    static_for<0, 8>([&](auto n) {
        constexpr int q = decltype(n)::value / 2, i = decltype(n)::value % 2;
        constexpr bool of_a = q == 0 || q == 3;
        constexpr int half = q >= 2 ? 1 : 0;
        const int c = 2 * wave + i, j0 = of_a ? (c >> 3) * 128 + half * 64 + (c & 7) * 8 : (c >> 2) * 64 + half * 32 + (c & 3) * 8;
        const int j = j0 + (lane >> 3), piece = (lane & 7) ^ (lane >> 3);
        int64_t first, r;
        if (of_a) {
            first = (int64_t)tm * T::BM + j0 < a.m ? (int64_t)tm * T::BM + j0 : a.m - 1;
            r = (int64_t)tm * T::BM + j < a.m ? (int64_t)tm * T::BM + j : a.m - 1;
        } else {
            first = i8_row_of_b<MODE>(tn, T::BN, j0, a.n);
            r = i8_row_of_b<MODE>(tn, T::BN, j, a.n);
        }
        base[q][i] = (const char*)(of_a ? a.a : a.b) + first * a.ldk;
        voff[q][i] = (unsigned int)((r - first) * a.ldk) + 16 * piece;
        to[q][i] = lds0 + (of_a ? 0 : T::BM * I8_STEP) + j0 * I8_STEP;
    });
    auto issue = [&](auto which, int s) {
        constexpr int q = decltype(which)::value;
#pragma unroll
        for (int i = 0; i < 2; ++i) copy_rows_to_lds(base[q][i] + (int64_t)s * I8_STEP, voff[q][i], to[q][i] + (unsigned int)(s & 1) * T::STAGE);
    };
    const int row = lane & 15, piece[2] = {((lane >> 4) ^ (row & 7)) * 16, ((4 + (lane >> 4)) ^ (row & 7)) * 16};
    i4v fa[2][4][2], fb[2][2][2];
    auto read_a = [&](auto which, int s) {
        constexpr int h = decltype(which)::value;
        const char* st = lds + (s & 1) * T::STAGE + (wm * 128 + h * 64 + row) * I8_STEP;
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int mi = 0; mi < 4; ++mi) fa[h][mi][k] = *(const i4v*)(st + piece[k] + mi * 16 * I8_STEP);
    };
    auto read_b = [&](auto which, int s) {
        constexpr int h = decltype(which)::value;
        const char* st = lds + (s & 1) * T::STAGE + (T::BM + wn * 64 + h * 32 + row) * I8_STEP;
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int ni = 0; ni < 2; ++ni) fb[h][ni][k] = *(const i4v*)(st + piece[k] + ni * 16 * I8_STEP);
    };
    auto multiply = [&](auto ha, auto hb) {
        constexpr int A = decltype(ha)::value, B = decltype(hb)::value;
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int mi = 0; mi < 4; ++mi)
#pragma unroll
                for (int ni = 0; ni < 2; ++ni)
                    acc[4 * A + mi][2 * B + ni] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[B][ni][k], fa[A][mi][k], acc[4 * A + mi][2 * B + ni], 0, 0, 0);
        __builtin_amdgcn_s_setprio(0);
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_barrier" ::: "memory");
    };
    typedef std::integral_constant<int, 0> C0;
    typedef std::integral_constant<int, 1> C1;
    typedef std::integral_constant<int, 3> C3;
    auto step = [&](int s, auto first) {
        constexpr int F = decltype(first)::value, G = 1 - F;
        typedef std::integral_constant<int, F> BF;
        typedef std::integral_constant<int, G> BG;
        const bool more = s + 2 < steps;
        auto turn_over = [&](auto reads) {
            if (more) i8_turn_over<10, decltype(reads)::value>();
            else i8_turn_over<0, decltype(reads)::value>();
        };
        typedef std::integral_constant<int, 4> R4;
        typedef std::integral_constant<int, 8> R8;
        read_b(BG{}, s);
        if (more) issue(C0{}, s + 2);
        turn_over(R4{});
        multiply(C0{}, BF{});
        read_a(C1{}, s);
        if (more) issue(std::integral_constant<int, 1 + F>{}, s + 2);
        turn_over(R8{});
        multiply(C0{}, BG{});
        read_a(C0{}, s + 1);   // (behind the last step: what is there, which nobody looks at)
        if (more) issue(std::integral_constant<int, 1 + G>{}, s + 2);
        turn_over(R8{});
        multiply(C1{}, BG{});
        read_b(BG{}, s + 1);
        if (more) issue(C3{}, s + 2);
        turn_over(R4{});
        multiply(C1{}, BF{});
    };
    auto ask = [&](int s, auto first) {
        constexpr int F = decltype(first)::value;
        issue(C0{}, s);
        issue(std::integral_constant<int, 1 + F>{}, s);
        issue(std::integral_constant<int, 2 - F>{}, s);
        issue(C3{}, s);
    };
    ask(0, C0{});
    if (steps > 1) ask(1, C1{});
    if (steps > 1) i8_turn_over<12, 0>();
    else i8_turn_over<0, 0>();
    read_a(C0{}, 0);
    read_b(C0{}, 0);
    if (steps > 1) i8_turn_over<10, 0>();
    else i8_turn_over<0, 0>();
    if (wave >= 4) asm volatile("s_barrier" ::: "memory");   // the second half is a turn behind
    for (int s = 0; s < steps; s += 2) {
        step(s, C0{});
        if (s + 1 >= steps) break;
        step(s + 1, C1{});
    }
    if (wave < 4) asm volatile("s_barrier" ::: "memory");
}

// A wave hands its results out through 4 KB of LDS, so that rows leave in 16-byte words side by side: straight from the accumulators
// they would leave in pieces of 32 or 64 bytes.  ROWS of C columns at a time; a row's 16-byte pieces are exchanged by the row.
template <typename OUT, int C>
struct I8Hand {
    static constexpr int ROW = C * (int)sizeof(OUT), PIECES = ROW / 16, ROWS = ROW >= 256 ? 16 : 32, PER = 16 / (int)sizeof(OUT);
    static constexpr int MASK = PIECES < 8 ? PIECES - 1 : 7;
    static_assert(ROWS * ROW <= 4096, "a wave's share");
    static __device__ __forceinline__ int place(int r, int byte) { return r * ROW + ((byte >> 4 ^ (r & MASK)) << 4) + (byte & 15); }
};
template <typename OUT, int C>
__device__ __forceinline__ void i8_put(char* w, int r, int c, f4 v)
{
    char* p = w + I8Hand<OUT, C>::place(r, c * (int)sizeof(OUT));
    if constexpr (sizeof(OUT) == 4) *(f4*)p = v;
    else *(u2*)p = u2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
}
// `wide`: rows are aligned to 16 bytes; otherwise a lane stores one number, next to its neighbours' (4095 x 4097 x 4096 104 us; four to a lane,
// straight from the accumulators, 129).
template <typename OUT, int C>
__device__ __forceinline__ void i8_hand_out(const char* w, OUT* out, int64_t ld, int rows, int cols, bool wide, int lane)
{
    typedef I8Hand<OUT, C> H;
    if (!wide) {
#pragma unroll 4
        for (int i = 0; i < H::ROWS * C / 64; ++i) {
            const int e = lane + 64 * i, r = e / C, c = e % C;
            if (r < rows && c < cols) out[(int64_t)r * ld + c] = *(const OUT*)(w + H::place(r, c * (int)sizeof(OUT)));
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < H::ROWS * H::PIECES / 64; ++i) {
        const int e = lane + 64 * i, r = e / H::PIECES, c = e % H::PIECES * H::PER, left = cols - c;
        const u4 v = *(const u4*)(w + H::place(r, 16 * (e % H::PIECES)));
        OUT* to = out + (int64_t)r * ld + c;
        if (r < rows && left >= H::PER) *(u4*)to = v;
        else if (r < rows)
#pragma unroll
            for (int k = 0; k < H::PER; ++k)
                if (k < left) {
                    if constexpr (sizeof(OUT) == 4) to[k] = __uint_as_float(v[k]);
                    else to[k] = (OUT)(v[k >> 1] >> (16 * (k & 1)));
                }
    }
}

template <typename T, I8Mode MODE>
__device__ __forceinline__ bool i8_sums(const I8ProductArgs& a, int tm, int tn, char* lds, i4v (&acc)[T::MI][T::NI])
{
#pragma unroll
    for (int mi = 0; mi < T::MI; ++mi)
#pragma unroll
        for (int ni = 0; ni < T::NI; ++ni) acc[mi][ni] = i4v{0, 0, 0, 0};
    bool first = true;
    if constexpr (std::is_same<T, I8Pong>::value) i8_tile_pong<MODE>(a, tm, tn, lds, acc);
    else first = i8_tile<T, MODE>(a, tm, tn, lds, acc);
    __syncthreads();
    return first;
}

template <typename T, I8Mode MODE, typename OUT>
__device__ __forceinline__ void i8_tile_out(const I8ProductArgs& a, int tm, int tn, char* lds, const i4v (&acc)[T::MI][T::NI])
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int r0 = tm * T::BM + wave / T::WN * (T::BM / T::WM);
    constexpr int PAIR = MODE == I8_PLAIN ? 1 : 2, COLS = T::BN / T::WN / PAIR, NJ = T::NI / PAIR;
    const int c0 = tn * (T::BN / PAIR) + wave % T::WN * COLS, cl = 4 * (lane >> 4);
    OUT* out = (OUT*)a.out;
    I8Columns s[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) s[j] = i8_columns<MODE>(a, c0 + cl + 16 * j);
    if (!a.accumulate) {
        typedef I8Hand<OUT, COLS> H;
        constexpr int AT = H::ROWS / 16;
        char* w = lds + wave * 4096;
        static_for<0, T::MI / AT>([&](auto turn) {
            constexpr int M = decltype(turn)::value * AT;
            f4 more[AT][NJ];
            const int rows = a.m - (r0 + 16 * M), cols = a.n - c0;
            if (MODE == I8_INNER && !a.dh_words) {   // dh comes the same way
                const OUT* dh = (const OUT*)a.dh + (int64_t)(r0 + 16 * M) * a.ld_dh + c0;
#pragma unroll 4
                for (int i = 0; i < H::ROWS * COLS / 64; ++i) {
                    const int e = lane + 64 * i, r = e / COLS, c = e % COLS;
                    if (r < rows && c < cols) *(OUT*)(w + H::place(r, c * (int)sizeof(OUT))) = dh[(int64_t)r * a.ld_dh + c];
                }
                wave_lds_sync();
#pragma unroll
                for (int mi = 0; mi < AT; ++mi)
#pragma unroll
                    for (int j = 0; j < NJ; ++j)
                        more[mi][j] = i8_load4((const OUT*)(w + H::place(16 * mi + (lane & 15), (cl + 16 * j) * (int)sizeof(OUT))), true, 4);
                wave_lds_sync();
            } else if (MODE == I8_INNER) {
#pragma unroll
                for (int mi = 0; mi < AT; ++mi)
#pragma unroll
                    for (int j = 0; j < NJ; ++j) {
                        const int r = r0 + 16 * (M + mi) + (lane & 15), c = c0 + cl + 16 * j;
                        more[mi][j] = i8_load4((const OUT*)a.dh + (int64_t)(r < a.m ? r : a.m - 1) * a.ld_dh + c, true, a.n - c);
                    }
            }
#pragma unroll
            for (int mi = 0; mi < AT; ++mi) {
                const int r = r0 + 16 * (M + mi) + (lane & 15), rr = r < a.m ? r : a.m - 1;
                const float scale = a.ldk > 0 ? a.a_scales[rr] : 0.f;
#pragma unroll
                for (int j = 0; j < NJ; ++j) {
                    const I8Results v = i8_results<MODE>(s[j], acc[M + mi][j * PAIR], acc[M + mi][j * PAIR + PAIR - 1], scale, a.activation, more[mi][j]);
                    i8_put<OUT, COLS>(w, 16 * mi + (lane & 15), cl + 16 * j, v.g);
                    more[mi][j] = v.u;
                }
            }
            OUT* to = out + (int64_t)(r0 + 16 * M) * a.ld + c0;
            wave_lds_sync();
            i8_hand_out<OUT, COLS>(w, to, a.ld, rows, cols, a.wide != 0, lane);
            wave_lds_sync();
            if constexpr (MODE == I8_INNER) {
#pragma unroll
                for (int mi = 0; mi < AT; ++mi)
#pragma unroll
                    for (int j = 0; j < NJ; ++j) i8_put<OUT, COLS>(w, 16 * mi + (lane & 15), cl + 16 * j, more[mi][j]);
                wave_lds_sync();
                i8_hand_out<OUT, COLS>(w, to + a.n, a.ld, rows, cols, a.wide != 0, lane);
                wave_lds_sync();
            }
        });
        return;
    }
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int mi = 0; mi < T::MI; ++mi) {
            const int r = r0 + 16 * mi + (lane & 15);
            if (r < a.m) i8_finish<MODE>(a, out, r, c0 + cl + 16 * j, s[j], acc[mi][j * PAIR], acc[mi][j * PAIR + PAIR - 1], a.ldk > 0 ? a.a_scales[r] : 0.f);
        }
}

template <typename T, I8Mode MODE, typename OUT>
__global__ __launch_bounds__(T::THREADS) void i8_tile_kernel(I8ProductArgs a)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    int tm, tn;
    tile_at(tile_of_block(blockIdx.x, a.nm * a.nn), a.nm, a.nn, a.band, tm, tn);
    i4v acc[T::MI][T::NI];
    if (i8_sums<T, MODE>(a, tm, tn, lds, acc)) i8_tile_out<T, MODE, OUT>(a, tm, tn, lds, acc);
}

// One plain product or two, whose tiles follow each other: the second's fill the round that the first's leave half empty.
struct I8Pair {
    I8ProductArgs a[2];
};
template <typename T>
__global__ __launch_bounds__(T::THREADS) void i8_pair_kernel(I8Pair p)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int first = p.a[0].nm * p.a[0].nn, second = (int)blockIdx.x >= first;
    const I8ProductArgs a = second ? p.a[1] : p.a[0];
    int tm, tn;
    tile_at(tile_of_block(blockIdx.x - (second ? first : 0), a.nm * a.nn), a.nm, a.nn, a.band, tm, tn);
    i4v acc[T::MI][T::NI];
    if (!i8_sums<T, I8_PLAIN>(a, tm, tn, lds, acc)) return;
    if (a.bf16) i8_tile_out<T, I8_PLAIN, unsigned short>(a, tm, tn, lds, acc);
    else i8_tile_out<T, I8_PLAIN, float>(a, tm, tn, lds, acc);
}

template <typename T, I8Mode MODE>
static int set_tiles(I8ProductArgs& a)
{
    constexpr int COLS = MODE == I8_PLAIN ? T::BN : T::BN / 2;
    a.nm = (a.m + T::BM - 1) / T::BM;
    a.nn = (a.n + COLS - 1) / COLS;
    a.band = 4;   // (rows of tiles that are swept together, so that what they read stays in a die's cache)
    return (int64_t)a.nm * a.nn > 0x3fffffff ? GVQ_EINVAL : GVQ_OK;
}
template <typename T, typename K, typename ARGS>
static int launch_kernel(K kernel, gvq_once_per_device& lds, const ARGS& args, int64_t tiles, hipStream_t st)
{
    int dev;
    GVQ_HIP(hipGetDevice(&dev));
    const int rc = lds.call(dev, [&] {
        GVQ_HIP(hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, T::LDS));
        return (int)GVQ_OK;
    });
    if (rc != GVQ_OK) return rc;
    hipLaunchKernelGGL(kernel, dim3((unsigned)tiles), dim3(T::THREADS), T::LDS, st, args);
    GVQ_HIP(hipGetLastError());
    return GVQ_OK;
}

template <typename T, I8Mode MODE, typename OUT>
static int launch_tile(I8ProductArgs a, hipStream_t st)
{
    static gvq_once_per_device lds;
    const int rc = set_tiles<T, MODE>(a);
    return rc != GVQ_OK ? rc : launch_kernel<T>(i8_tile_kernel<T, MODE, OUT>, lds, a, (int64_t)a.nm * a.nn, st);
}
template <typename T>
static int launch_pair(I8Pair p, hipStream_t st)
{
    static gvq_once_per_device lds;
    int64_t tiles = 0;
    for (I8ProductArgs& a : p.a) {
        if (a.m == 0) continue;
        const int rc = set_tiles<T, I8_PLAIN>(a);
        if (rc != GVQ_OK) return rc;
        tiles += (int64_t)a.nm * a.nn;
    }
    return launch_kernel<T>(i8_pair_kernel<T>, lds, p, tiles, st);
}

typedef I8Shape<64, 64, 2, 2, 2> I8Tile64;
typedef I8Shape<64, 64, 2, 2, 2, 2> I8Tile64Two;
typedef I8Shape<64, 64, 2, 2, 2, 4> I8Tile64Four;
typedef I8Shape<128, 128, 2, 2, 2> I8Tile128;

static int launch_plain(const I8Pair& p, int way, hipStream_t st)
{
    switch (way) {
    case I8_TILE_64: return launch_pair<I8Tile64>(p, st);
    case I8_TILE_64_TWO: return launch_pair<I8Tile64Two>(p, st);
    case I8_TILE_64_FOUR: return launch_pair<I8Tile64Four>(p, st);
    case I8_TILE_128: return launch_pair<I8Tile128>(p, st);
    default: return launch_pair<I8Pong>(p, st);
    }
}
template <I8Mode MODE, typename OUT>
static int launch_mode(const I8ProductArgs& a, int way, hipStream_t st)
{
    switch (way) {
    case I8_TILE_64: return launch_tile<I8Tile64, MODE, OUT>(a, st);
    case I8_TILE_64_TWO: return launch_tile<I8Tile64Two, MODE, OUT>(a, st);
    case I8_TILE_64_FOUR: return launch_tile<I8Tile64Four, MODE, OUT>(a, st);
    case I8_TILE_128: return launch_tile<I8Tile128, MODE, OUT>(a, st);
    default: return launch_tile<I8Pong, MODE, OUT>(a, st);
    }
}

static void set_words(I8ProductArgs& a, I8Mode mode, gvq_dtype_t dtype)
{
    const int64_t es = dtype == GVQ_BF16 ? 2 : 4;
    a.bf16 = dtype == GVQ_BF16;
    a.words = (((uintptr_t)a.out | (uintptr_t)(a.ld * es)) & (uintptr_t)(4 * es - 1)) == 0;
    a.dh_words = (((uintptr_t)a.dh | (uintptr_t)(a.ld_dh * es)) & (uintptr_t)(4 * es - 1)) == 0;
    a.wide = (((uintptr_t)a.out | (uintptr_t)(a.ld * es) | (mode == I8_INNER ? (uintptr_t)(a.n * es) : 0)) & 15) == 0;
}

int gvq_launch_i8_product(I8ProductArgs a, I8Mode mode, gvq_dtype_t dtype, hipStream_t st)
{
    set_words(a, mode, dtype);
    const int way = i8_pick(a.m, a.n, mode == I8_PLAIN ? 1 : 2, a.ldk / I8_STEP);
    if (way <= I8_FEW_32) return gvq_launch_i8_few(a, way == I8_FEW_16 ? 1 : 2, mode, dtype, st);
    if (mode == I8_PLAIN) {
        I8Pair p{};
        p.a[0] = a;
        return launch_plain(p, way, st);
    }
    if (dtype == GVQ_BF16)
        return mode == I8_GATED ? launch_mode<I8_GATED, unsigned short>(a, way, st) : launch_mode<I8_INNER, unsigned short>(a, way, st);
    return mode == I8_GATED ? launch_mode<I8_GATED, float>(a, way, st) : launch_mode<I8_INNER, float>(a, way, st);
}

int gvq_launch_i8_products(I8ProductArgs a, gvq_dtype_t a_dtype, I8ProductArgs b, gvq_dtype_t b_dtype, hipStream_t st)
{
    const int way = i8_pick_pair(a.m, a.n, a.ldk / I8_STEP, b.m, b.n, b.ldk / I8_STEP);
    if (way < 0) {
        const int rc = gvq_launch_i8_product(a, I8_PLAIN, a_dtype, st);
        return rc != GVQ_OK ? rc : gvq_launch_i8_product(b, I8_PLAIN, b_dtype, st);
    }
    set_words(a, I8_PLAIN, a_dtype);
    set_words(b, I8_PLAIN, b_dtype);
    // the longer tiles first
    I8Pair p{};
    p.a[0] = a.ldk >= b.ldk ? a : b;
    p.a[1] = a.ldk >= b.ldk ? b : a;
    return launch_plain(p, way, st);
}
