// A work-group's tile of a product of two matrices whose rows both run along the sum (C = A B^T), for the 4-bit products
// (gvq_mx_product.hip) and the Newton-Schulz products (gvq_muon.hip).  The two share everything but the matrix instruction: 128
// numbers of 4 bits and 32 of 16 bits are both 64 bytes of a row, 16 bytes a lane, and one 16 x 16 matrix instruction.
//
// Rows come global -> LDS without passing through registers, 64 bytes of every row of the tile per step, STAGES steps ahead;
// one barrier a step.  In LDS a 16-row group is 1 KB: row r's 16-byte chunk c sits in slot c ^ tile_swizzle(r / 4) of the row, so that
// the 16 lanes whose 16-byte reads the LDS serves together (0-3, 12-15, 20-23, 24-27 and the like) cover all 64 banks.
//
// What bounds it.  4 bits, 256 x 256: LDS, of which a step's 1024 cycles of products need 96 KB of fragments, 33 KB of copies in and
// 24 reads of scales a wave; 8192 x 8192 x 8192 3.7 PFLOP/s of the 8.0 that the pipe does alone.  f16, three products: power, the
// clock falls to 1.9 GHz with the pipe two thirds busy; a step of 4096 x 4096 x 4096 1.25 to 1.3 PFLOP/s where the library's f16 product of
// 8192 x 8192 x 8192 does 1.24.  256 x 256 is the largest tile whose sums leave registers for fragments (128 of 256; the f16 kernels that hand
// planes out keep 24 to 26 more in scratch), eight waves of 128 x 64 because four of 128 x 128 have their sums copied back and forth (four times slower).
#pragma once
#include "gvq_device.h"

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef _Float16 h4 __attribute__((ext_vector_type(4)));
typedef int i8v __attribute__((ext_vector_type(8)));

#define TILE_STEP 64   // bytes of a row per step

// global -> LDS, `voff` bytes behind the wave-uniform `base` for each lane, 16 (or 4) bytes a lane to consecutive places from the
// wave-uniform byte offset `lds` on.  Inline assembly: the compiler would otherwise wait for every such copy before any LDS read.
// m0 carries the LDS offset and is named as clobbered on purpose.  The compiler keeps `base` in vector registers where it likes and
// reads it into scalar ones right before the copy; a scalar register that a vector instruction wrote may be an address five wait
// states later at the earliest, and the compiler puts no such waits in front of inline assembly: the five are s_mov and s_nop 3.
__device__ __forceinline__ const void* in_scalars(const void* p)
{
    const uint64_t v = (uint64_t)p;
    const unsigned int lo = __builtin_amdgcn_readfirstlane((int)v), hi = __builtin_amdgcn_readfirstlane((int)(v >> 32));
    return (const void*)((uint64_t)hi << 32 | lo);
}
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void copy_rows_to_lds(const void* base, unsigned int voff, unsigned int lds)
{
    base = in_scalars(base);
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %0, %2" ::"v"(voff), "s"(lds), "s"(base)
                 : "memory", "m0");
}
__device__ __forceinline__ void copy_words_to_lds(const void* base, unsigned int voff, unsigned int lds)
{
    base = in_scalars(base);
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 3\n\tglobal_load_lds_dword %0, %2" ::"v"(voff), "s"(lds), "s"(base)
                 : "memory", "m0");
}
#pragma clang diagnostic pop

// Where a copy's destination lies among the work-group's LDS: `p` is not always the first of it.
__device__ __forceinline__ unsigned int lds_offset(const char* p)
{
    return (unsigned int)(uintptr_t)(__attribute__((address_space(3))) const char*)p;
}

// All but the youngest N copies of this wave have arrived and its LDS reads are done; then the other waves' too.
template <int N>
__device__ __forceinline__ void tile_barrier()
{
    static_assert(N >= 0 && N < 64, "vmcnt is a 6-bit counter");
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

__device__ __forceinline__ int tile_swizzle(int s) { return (0x78 >> (2 * s)) & 3; }   // 0 2 3 1

// One operand: `planes` matrices of the same layout, `plane` bytes apart; rows of `ld` bytes (a multiple of TILE_STEP).
struct TileOperand {
    const char* p;
    int64_t plane;
    int64_t ld;
    int rows;              // rows behind the last one are read as the last one (of the second operand in the other layout: columns)
    const char* scales;    // 4-bit operands: one byte per 32 numbers, rows of ld / 16 bytes
    int depth;             // second operand in the other layout: its rows (numbers of the sum); further ones are read as the last one
};

// What a lane holds of 16 rows and one step.
struct TileFragMx {
    u4 v;
    int k;   // scale
};
struct TileFragF16 {
    h8 hi, lo;
};

// BM x BN of C by WM x WN waves; PLANES = 1: 4-bit numbers with scales, 2: two f16 terms per number (three products).
// TURNED: the second operand's rows run across the sum instead of along it (C = A B; f16): a step is 32 of its rows, BN columns
// each, and a lane gets its eight numbers of one column by two transposing LDS reads.  Their 32-byte units (a fragment's 16 columns of
// one row) are exchanged within a row so that the eight rows that are read at one time lie in different banks.
// FLIP: a lane ends with four neighbouring rows of one column instead of four neighbouring columns of one row.
// Scales come for four steps at a time, 16 bytes of a row, into one of two places (a row's 4 bytes per step cost as many cache lines
// as its 16 would: 8192 x 4096 x 4096 73 us without them, 101 with): sums of four steps at least, unless NARROW, step by step.
template <int BM_, int BN_, int WM_, int WN_, int PLANES_, int STAGES_, bool TURNED_ = false, bool FLIP_ = false, bool NARROW_ = false>
struct TileShape {
    static constexpr bool TURNED = TURNED_, FLIP = FLIP_, WIDE = PLANES_ == 1 && !NARROW_;
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, PLANES = PLANES_, STAGES = STAGES_;
    static constexpr int WAVES = WM * WN, THREADS = 64 * WAVES;
    static constexpr int MI = BM / WM / 16, NI = BN / WN / 16;             // fragments of a wave
    static constexpr int GROUPS = PLANES * (BM + BN) / 16;                 // 1 KB copies of a step
    static constexpr int COPIES = GROUPS / WAVES;
    static constexpr int SCALE_GROUPS = PLANES == 1 ? (BM + BN) / 64 : 0;  // 64 rows' scales each
    static constexpr int SCALE_COPIES = (SCALE_GROUPS + WAVES - 1) / WAVES;
    static constexpr int STAGE = GROUPS * 1024 + (WIDE ? 0 : SCALE_GROUPS * 256);
    static constexpr int SCALE_PLACE = SCALE_GROUPS * 1024;                // WIDE: two of them behind the stages
    static constexpr int LDS = STAGE * STAGES + (WIDE ? 2 * SCALE_PLACE : 0);
    static constexpr int RING = (2 * MI) % 3 == 0 ? 3 : 4;                 // row fragments of A in registers
    static constexpr int BSETS = PLANES == 1 ? 2 : 1;                      // sets of column fragments
    static constexpr int UNROLL = BSETS == 2 || MI % RING ? 2 : 1;         // steps after which the registers' roles repeat
    typedef typename std::conditional<PLANES == 1, TileFragMx, TileFragF16>::type Frag;
    // Of a wave and a step.  WIDE: every fourth step has SCALE_COPIES more, which a wait for the youngest ones' predecessors then
    // counts in place of younger ones: it waits for a copy or two more than it has to.
    static constexpr int LOADS = COPIES + (WIDE ? 0 : SCALE_COPIES);
    static_assert(BM % (16 * WM) == 0 && BN % (16 * WN) == 0 && GROUPS % WAVES == 0, "whole fragments and copies");
    static_assert(SCALE_GROUPS * 64 == (PLANES == 1 ? BM + BN : 0), "whole copies of scales");
    static_assert(LDS <= 160 * 1024 && (LOADS + SCALE_COPIES) * STAGES < 64, "LDS and vmcnt");
    static_assert(!WIDE || STAGES <= 4, "a place of scales is free when the step that needs the next one is asked for");
    static_assert(!TURNED || (PLANES == 2 && (NI & (NI - 1)) == 0 && (BN & (BN - 1)) == 0 && BN >= 64), "exchange by exclusive or");
    static_assert(MI >= 2 && (2 * MI) % RING == 0, "rings turn whole in two steps");
};

typedef short s4v __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s4v* tile_turn_ptr;
// Four numbers each of one column: 16 lanes read four rows of 16 numbers, lane i four numbers of row i / 4 from column 4 (i % 4) on, and
// lane i gets column i.
__device__ __forceinline__ h4 turned4(const void* p)
{
    return __builtin_bit_cast(h4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((tile_turn_ptr)p));
}
template <typename T>
__device__ __forceinline__ int tile_exchange(int row)
{
    return T::BN >= 128 ? (row & 3) | (row >> 1 & 4) : (row >> 1 & 1) | (row >> 2 & 2);
}

// acc[mi][ni][i] += C[row0 + wave's rows + 16 mi + lane % 16][col0 + wave's columns + 16 ni + 4 (lane / 16) + i] (FLIP: row 4 (lane / 16) + i,
// column lane % 16), over the steps [step0, step0 + steps) of the sum.  Four neighbouring columns a lane come from giving the matrix
// instruction the operands in exchanged roles.  lds: T::LDS bytes, aligned to 16.
template <typename T>
__device__ __forceinline__ void tile_product(const TileOperand& A, const TileOperand& B, int row0, int col0, int step0, int steps,
                                             char* lds, f4 (&acc)[T::MI][T::NI])
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int wm = wave / T::WN, wn = wave % T::WN;
    const unsigned int lds0 = lds_offset(lds);
    const char* base[2] = {A.p + (int64_t)row0 * A.ld + (int64_t)step0 * TILE_STEP,
                           T::TURNED ? B.p + (int64_t)step0 * 32 * B.ld + (int64_t)col0 * 2
                                     : B.p + (int64_t)col0 * B.ld + (int64_t)step0 * TILE_STEP};
    const char* sbase[2] = {nullptr, nullptr};
    unsigned int voff[T::COPIES], soff[T::SCALE_COPIES > 0 ? T::SCALE_COPIES : 1];
    constexpr int GA = T::BM / 16, GB = T::BN / 16;   // groups of a plane
#pragma unroll
    for (int i = 0; i < T::COPIES; ++i) {
        // copies [0, PLANES GA) are A's planes, the rest B's
        const int g = wave * T::COPIES + i;
        const bool of_b = g >= T::PLANES * GA;
        const int gg = of_b ? g - T::PLANES * GA : g, per = of_b ? GB : GA;
        const int pl = gg / per;
        if (T::TURNED && of_b) {
            const int flat = (gg - pl * per) * 64 + lane, r = flat / (T::BN / 8), u = flat % (T::BN / 8);
            const int c = ((u >> 1) ^ tile_exchange<T>(r)) * 32 + (u & 1) * 16, most = (int)(B.ld - 16 - (int64_t)col0 * 2);
            voff[i] = (unsigned int)(pl * B.plane + (c < most ? c : most));
            continue;
        }
        const int r = (gg - pl * per) * 16 + (lane >> 2);
        const int last = of_b ? B.rows - 1 - col0 : A.rows - 1 - row0;
        const int c = (lane & 3) ^ tile_swizzle(lane >> 4);
        voff[i] = (unsigned int)((r < last ? r : last) * (of_b ? B.ld : A.ld) + pl * (of_b ? B.plane : A.plane)) + 16 * c;
    }
    if constexpr (T::PLANES == 1) {
        sbase[0] = A.scales + (int64_t)row0 * (A.ld / 16) + (int64_t)step0 * 4;
        sbase[1] = B.scales + (int64_t)col0 * (B.ld / 16) + (int64_t)step0 * 4;
#pragma unroll
        for (int i = 0; i < T::SCALE_COPIES; ++i) {
            const int g = (wave * T::SCALE_COPIES + i) % T::SCALE_GROUPS;
            const bool of_b = g >= T::BM / 64;
            const int r = (of_b ? g - T::BM / 64 : g) * 64 + lane;
            const int last = of_b ? B.rows - 1 - col0 : A.rows - 1 - row0;
            soff[i] = (unsigned int)((r < last ? r : last) * ((of_b ? B.ld : A.ld) / 16));
        }
    }
    auto issue = [&](int s) {
        const unsigned int to = lds0 + (unsigned int)(s % T::STAGES) * T::STAGE;
        if constexpr (T::WIDE) {
            if ((s & 3) == 0) {
                const int from = s + 4 <= steps ? s : steps - 4;
#pragma unroll
                for (int i = 0; i < T::SCALE_COPIES; ++i) {
                    const int g = (wave * T::SCALE_COPIES + i) % T::SCALE_GROUPS;
                    copy_rows_to_lds(sbase[g >= T::BM / 64] + (int64_t)from * 4, soff[i],
                                     lds0 + T::STAGE * T::STAGES + (s >> 2 & 1) * T::SCALE_PLACE + g * 1024);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < T::COPIES; ++i) {
            const int g = wave * T::COPIES + i;
            if (T::TURNED && g >= T::PLANES * GA) {
                const int left = B.depth - 1 - (step0 + s) * 32, r = (((g - T::PLANES * GA) % GB) * 64 + lane) / (T::BN / 8);
                copy_rows_to_lds(base[1] + (int64_t)s * 32 * B.ld, voff[i] + (unsigned int)(r < left ? r : left) * (unsigned int)B.ld,
                                 to + g * 1024);
            } else {
                copy_rows_to_lds(base[g >= T::PLANES * GA] + (int64_t)s * TILE_STEP, voff[i], to + g * 1024);
            }
        }
        if constexpr (T::PLANES == 1 && !T::WIDE) {
#pragma unroll
            for (int i = 0; i < T::SCALE_COPIES; ++i) {
                const int g = (wave * T::SCALE_COPIES + i) % T::SCALE_GROUPS;
                copy_words_to_lds(sbase[g >= T::BM / 64] + (int64_t)s * 4, soff[i], to + T::GROUPS * 1024 + g * 256);
            }
        }
    };
    // WIDE: the scales of steps s to s + 3, or of the last four
    auto scales_from = [&](int s) { return (s & ~3) + 4 <= steps ? s & ~3 : steps - 4; };
    auto scales_at = [&](int s, int row) {
        if constexpr (T::WIDE)
            return T::STAGE * T::STAGES + (s >> 2 & 1) * T::SCALE_PLACE + row * 16 + (s - scales_from(s)) * 4;
        else
            return (s % T::STAGES) * T::STAGE + T::GROUPS * 1024 + row * 4;
    };
    const int frag = (lane & 15) * 64 + ((lane >> 4) ^ tile_swizzle((lane >> 2) & 3)) * 16;
    const int turn_row = 8 * (lane >> 4) + ((lane & 15) >> 2);
    const int turn = turn_row * 2 * T::BN + (lane & 3) * 8, turn_unit = (wn * T::NI) ^ tile_exchange<T>(turn_row);
    typedef typename T::Frag Frag;
    constexpr int SCALE_ROW = T::WIDE ? 16 : 4;
    const char* lane_scale = lds + (lane >> 4);
    Frag fa[T::RING], fb[T::BSETS][T::NI];
    auto load_a = [&](const char* st, const char* sc, int mi, Frag& f) {
        if constexpr (T::PLANES == 1) {
            f.v = *(const u4*)(st + (wm * T::MI + mi) * 1024 + frag);
            f.k = *(const unsigned char*)(sc + (wm * T::MI + mi) * 16 * SCALE_ROW);
        } else {
            f.hi = *(const h8*)(st + (wm * T::MI + mi) * 1024 + frag);
            f.lo = *(const h8*)(st + (GA + wm * T::MI + mi) * 1024 + frag);
        }
    };
    auto load_b = [&](const char* st, const char* sc, int ni, Frag& f, auto which) {   // f16: 1 the first term, 2 the second
        constexpr int WHICH = decltype(which)::value;
        if constexpr (T::PLANES == 1) {
            f.v = *(const u4*)(st + (GA + wn * T::NI + ni) * 1024 + frag);
            f.k = *(const unsigned char*)(sc + (T::BM + (wn * T::NI + ni) * 16) * SCALE_ROW);
        } else if constexpr (T::TURNED) {
            // two transposing reads of four rows each; lane i of 16 gets column i of the fragment
            const char* p = st + 2 * GA * 1024 + turn + ((turn_unit ^ ni) << 5);
            if constexpr (WHICH & 1) {
                const h4 a = turned4(p), b = turned4(p + 8 * T::BN);
                f.hi = h8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
            }
            if constexpr (WHICH & 2) {
                const h4 a = turned4(p + GB * 1024), b = turned4(p + GB * 1024 + 8 * T::BN);
                f.lo = h8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
            }
        } else {
            if constexpr (WHICH & 1) f.hi = *(const h8*)(st + (2 * GA + wn * T::NI + ni) * 1024 + frag);
            if constexpr (WHICH & 2) f.lo = *(const h8*)(st + (2 * GA + GB + wn * T::NI + ni) * 1024 + frag);
        }
    };
    // One step, the P-th of UNROLL; the row fragments run two ahead.  Before its last two rows of products the wave has read all of
    // the step's rows: there it meets the others, asks for step s + STAGES into the place that is free now, and reads the beginning
    // of the next step beside the products that are left (f16: into the registers of B's fragments as their last products go out).
    auto step = [&](int s, auto parity) {
        constexpr int P = decltype(parity)::value, PB = P % T::BSETS, NB = (P + 1) % T::BSETS;
        const char* st = lds + (unsigned int)(s % T::STAGES) * T::STAGE;
        const char* next = lds + (unsigned int)((s + 1) % T::STAGES) * T::STAGE;
        const bool more = s + 1 < steps;
        const char* sc = T::PLANES == 1 ? lane_scale + scales_at(s, lane & 15) : nullptr;
        const char* next_sc = T::PLANES == 1 ? lane_scale + scales_at(more ? s + 1 : s, lane & 15) : nullptr;
        static_for<0, T::MI>([&](auto c) {
            constexpr int mi = decltype(c)::value;
            if constexpr (mi + 2 < T::MI) load_a(st, sc, mi + 2, fa[(P * T::MI + mi + 2) % T::RING]);
            if constexpr (mi == T::MI - 2) {
                if (more) {
                    if (s + T::STAGES <= steps) tile_barrier<T::LOADS * (T::STAGES - 2)>();
                    else tile_barrier<0>();
                    if (s + T::STAGES < steps) issue(s + T::STAGES);
                }
                // (behind the last step: read once more what is there, into registers that nobody looks at)
                if constexpr (T::BSETS == 2)
#pragma unroll
                    for (int ni = 0; ni < T::NI; ++ni) load_b(next, next_sc, ni, fb[NB][ni], std::integral_constant<int, 3>{});
            }
            if constexpr (mi >= T::MI - 2) load_a(next, next_sc, mi + 2 - T::MI, fa[(P * T::MI + mi + 2) % T::RING]);
            const Frag& a = fa[(P * T::MI + mi) % T::RING];
            if constexpr (T::PLANES == 1) {
#pragma unroll
                for (int ni = 0; ni < T::NI; ++ni) {
                    const Frag& b = fb[PB][ni];
                    acc[mi][ni] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
                        i8v{(int)b.v[0], (int)b.v[1], (int)b.v[2], (int)b.v[3], 0, 0, 0, 0},
                        i8v{(int)a.v[0], (int)a.v[1], (int)a.v[2], (int)a.v[3], 0, 0, 0, 0}, acc[mi][ni], 4, 4, 0, b.k, 0, a.k);
                }
            } else {
#pragma unroll
                for (int ni = 0; ni < T::NI; ++ni) acc[mi][ni] = T::FLIP ? __builtin_amdgcn_mfma_f32_16x16x32_f16(a.hi, fb[PB][ni].lo, acc[mi][ni], 0, 0, 0)
                                                                           : __builtin_amdgcn_mfma_f32_16x16x32_f16(fb[PB][ni].lo, a.hi, acc[mi][ni], 0, 0, 0);
                if constexpr (mi == T::MI - 1)
#pragma unroll
                    for (int ni = 0; ni < T::NI; ++ni) load_b(next, next_sc, ni, fb[PB][ni], std::integral_constant<int, 2>{});
#pragma unroll
                for (int ni = 0; ni < T::NI; ++ni) acc[mi][ni] = T::FLIP ? __builtin_amdgcn_mfma_f32_16x16x32_f16(a.lo, fb[PB][ni].hi, acc[mi][ni], 0, 0, 0)
                                                                           : __builtin_amdgcn_mfma_f32_16x16x32_f16(fb[PB][ni].hi, a.lo, acc[mi][ni], 0, 0, 0);
#pragma unroll
                for (int ni = 0; ni < T::NI; ++ni) acc[mi][ni] = T::FLIP ? __builtin_amdgcn_mfma_f32_16x16x32_f16(a.hi, fb[PB][ni].hi, acc[mi][ni], 0, 0, 0)
                                                                           : __builtin_amdgcn_mfma_f32_16x16x32_f16(fb[PB][ni].hi, a.hi, acc[mi][ni], 0, 0, 0);
                if constexpr (mi == T::MI - 1)
#pragma unroll
                    for (int ni = 0; ni < T::NI; ++ni) load_b(next, next_sc, ni, fb[PB][ni], std::integral_constant<int, 1>{});
            }
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    if (steps <= 0) return;
    for (int s = 0; s < T::STAGES && s < steps; ++s) issue(s);
    if (steps >= T::STAGES) tile_barrier<T::LOADS * (T::STAGES - 1)>();
    else tile_barrier<0>();
    const char* first_sc = T::PLANES == 1 ? lane_scale + scales_at(0, lane & 15) : nullptr;
#pragma unroll
    for (int ni = 0; ni < T::NI; ++ni) load_b(lds, first_sc, ni, fb[0][ni], std::integral_constant<int, 3>{});
    load_a(lds, first_sc, 0, fa[0]);
    load_a(lds, first_sc, 1, fa[1]);
    for (int s = 0; s < steps; s += T::UNROLL) {
        step(s, std::integral_constant<int, 0>{});
        if constexpr (T::UNROLL == 2) {
            if (s + 1 >= steps) break;
            step(s + 1, std::integral_constant<int, 1>{});
        }
    }
}

// Which tile a work-group takes.  Work-groups go round robin over the 8 XCDs, each with an L2 of its own: XCD x takes the x-th
// eighth of the tiles, in an order that sweeps groups of `band` tile rows column by column, so that the tiles in flight on one XCD
// share rows of both operands.
__device__ __forceinline__ int tile_of_block(int block, int tiles)
{
    const int per = tiles >> 3, more = tiles & 7, x = block & 7;
    return x * per + (x < more ? x : more) + (block >> 3);
}
__device__ __forceinline__ void tile_at(int t, int nm, int nn, int band, int& tm, int& tn)
{
    const int g = t / (band * nn), first = g * band, h = nm - first < band ? nm - first : band;
    const int r = t - g * band * nn;
    tn = r / h;
    tm = first + r - tn * h;
}
