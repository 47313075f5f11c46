// A work-group's tile of a product of two matrices whose rows both run along the sum (C = A B^T), for the 4-bit products
// (gvq_mx_product.hip) and the Newton-Schulz products (gvq_muon.hip).  The two share everything but the matrix instruction: 128
// numbers of 4 bits and 32 of 16 bits are both 64 bytes of a row, 16 bytes a lane, and one 16 x 16 matrix instruction.
//
// Rows come global -> LDS without passing through registers, 64 bytes of every row of the tile per step, STAGES - 1 steps ahead;
// one barrier a step.  In LDS a 16-row group is 1 KB: row r's 16-byte chunk c sits in slot c ^ ((r >> 2) & 3) of the row, so that
// the 16 rows of a fragment that are read at one time cover all 64 banks.
#pragma once
#include "gvq_device.h"

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef _Float16 h4 __attribute__((ext_vector_type(4)));
typedef int i8v __attribute__((ext_vector_type(8)));

#define TILE_STEP 64   // bytes of a row per step

// global -> LDS, `voff` bytes behind the wave-uniform `base` for each lane, 16 (or 4) bytes a lane to consecutive places from the
// wave-uniform byte offset `lds` on.  Inline assembly: the compiler would otherwise wait for every such copy before any LDS read.
// m0 carries the LDS offset and is named as clobbered on purpose.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void copy_rows_to_lds(const void* base, unsigned int voff, unsigned int lds)
{
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %2" ::"v"(voff), "s"(lds), "s"(base)
                 : "memory", "m0");
}
__device__ __forceinline__ void copy_words_to_lds(const void* base, unsigned int voff, unsigned int lds)
{
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, %2" ::"v"(voff), "s"(lds), "s"(base)
                 : "memory", "m0");
}
#pragma clang diagnostic pop

// All but the youngest N copies of this wave have arrived and its LDS reads are done; then the other waves' too.
template <int N>
__device__ __forceinline__ void tile_barrier()
{
    static_assert(N >= 0 && N < 64, "vmcnt is a 6-bit counter");
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// One operand: `planes` matrices of the same layout, `plane` bytes apart; rows of `ld` bytes (a multiple of TILE_STEP).
struct TileOperand {
    const char* p;
    int64_t plane;
    int64_t ld;
    int rows;              // rows behind the last one are read as the last one
    const char* scales;    // 4-bit operands: one byte per 32 numbers, rows of ld / 16 bytes
};

// BM x BN of C by WM x WN waves; PLANES = 1: 4-bit numbers with scales, 2: two f16 terms per number (three products).
template <int BM_, int BN_, int WM_, int WN_, int PLANES_, int STAGES_>
struct TileShape {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, PLANES = PLANES_, STAGES = STAGES_;
    static constexpr int WAVES = WM * WN, THREADS = 64 * WAVES;
    static constexpr int MI = BM / WM / 16, NI = BN / WN / 16;             // fragments of a wave
    static constexpr int GROUPS = PLANES * (BM + BN) / 16;                 // 1 KB copies of a step
    static constexpr int COPIES = GROUPS / WAVES;
    static constexpr int SCALE_GROUPS = PLANES == 1 ? (BM + BN) / 64 : 0;  // 64 rows' scales each
    static constexpr int SCALE_COPIES = (SCALE_GROUPS + WAVES - 1) / WAVES;
    static constexpr int STAGE = GROUPS * 1024 + SCALE_GROUPS * 256;
    static constexpr int LDS = STAGE * STAGES;
    static constexpr int LOADS = COPIES + SCALE_COPIES;                    // of a wave and a step
    static_assert(BM % (16 * WM) == 0 && BN % (16 * WN) == 0 && GROUPS % WAVES == 0, "whole fragments and copies");
    static_assert(SCALE_GROUPS * 64 == (PLANES == 1 ? BM + BN : 0), "whole copies of scales");
    static_assert(LDS <= 160 * 1024 && LOADS * (STAGES - 2) < 64, "LDS and vmcnt");
};

// acc[mi][ni][i] += C[row0 + wave's rows + 16 mi + lane % 16][col0 + wave's columns + 16 ni + 4 (lane / 16) + i], over the steps
// [step0, step0 + steps) of the sum.  The operands go into the matrix instruction in exchanged roles, so that a lane ends with four
// neighbouring columns of one row.
template <typename T>
__device__ __forceinline__ void tile_product(const TileOperand& A, const TileOperand& B, int row0, int col0, int step0, int steps,
                                             char* lds, f4 (&acc)[T::MI][T::NI])
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int wm = wave / T::WN, wn = wave % T::WN;
    const char* base[2] = {A.p + (int64_t)row0 * A.ld + (int64_t)step0 * TILE_STEP,
                           B.p + (int64_t)col0 * B.ld + (int64_t)step0 * TILE_STEP};
    const char* sbase[2] = {nullptr, nullptr};
    unsigned int voff[T::COPIES], soff[T::SCALE_COPIES > 0 ? T::SCALE_COPIES : 1];
    constexpr int GA = T::BM / 16, GB = T::BN / 16;   // groups of a plane
#pragma unroll
    for (int i = 0; i < T::COPIES; ++i) {
        // copies [0, PLANES GA) are A's planes, the rest B's
        const int g = wave * T::COPIES + i;
        const bool of_b = g >= T::PLANES * GA;
        const int gg = of_b ? g - T::PLANES * GA : g, per = of_b ? GB : GA;
        const int pl = gg / per, r = (gg - pl * per) * 16 + (lane >> 2);
        const int last = of_b ? B.rows - 1 - col0 : A.rows - 1 - row0;
        const int c = (lane & 3) ^ ((lane >> 4) & 3);
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
        const unsigned int to = (unsigned int)(s % T::STAGES) * T::STAGE;
#pragma unroll
        for (int i = 0; i < T::COPIES; ++i) {
            const int g = wave * T::COPIES + i;
            copy_rows_to_lds(base[g >= T::PLANES * GA] + (int64_t)s * TILE_STEP, voff[i], to + g * 1024);
        }
        if constexpr (T::PLANES == 1) {
#pragma unroll
            for (int i = 0; i < T::SCALE_COPIES; ++i) {
                const int g = (wave * T::SCALE_COPIES + i) % T::SCALE_GROUPS;
                copy_words_to_lds(sbase[g >= T::BM / 64] + (int64_t)s * 4, soff[i], to + T::GROUPS * 1024 + g * 256);
            }
        }
    };
    for (int s = 0; s < T::STAGES - 1 && s < steps; ++s) issue(s);
    const int frag = (lane & 15) * 64 + (((lane >> 4) ^ (lane >> 2)) & 3) * 16;
    for (int s = 0; s < steps; ++s) {
        if (s + T::STAGES - 1 <= steps) tile_barrier<T::LOADS * (T::STAGES - 2)>();
        else tile_barrier<0>();
        if (s + T::STAGES - 1 < steps) issue(s + T::STAGES - 1);
        const char* st = lds + (unsigned int)(s % T::STAGES) * T::STAGE;
        const char* pa = st + wm * T::MI * 1024 + frag;
        const char* pb = st + T::PLANES * GA * 1024 + wn * T::NI * 1024 + frag;
        if constexpr (T::PLANES == 1) {
            const char* sa = st + T::GROUPS * 1024 + (wm * T::MI * 16 + (lane & 15)) * 4 + (lane >> 4);
            const char* sb = st + T::GROUPS * 1024 + (T::BM + wn * T::NI * 16 + (lane & 15)) * 4 + (lane >> 4);
            i8v b[T::NI];
            int kb[T::NI];
#pragma unroll
            for (int ni = 0; ni < T::NI; ++ni) {
                const u4 v = *(const u4*)(pb + ni * 1024);
                b[ni] = i8v{(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0};
                kb[ni] = *(const unsigned char*)(sb + ni * 64);
            }
#pragma unroll
            for (int mi = 0; mi < T::MI; ++mi) {
                const u4 v = *(const u4*)(pa + mi * 1024);
                const i8v a = {(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0};
                const int ka = *(const unsigned char*)(sa + mi * 64);
#pragma unroll
                for (int ni = 0; ni < T::NI; ++ni)
                    acc[mi][ni] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b[ni], a, acc[mi][ni], 4, 4, 0, kb[ni], 0, ka);
            }
        } else {
            h8 b[T::NI][2];
#pragma unroll
            for (int ni = 0; ni < T::NI; ++ni) {
                b[ni][0] = *(const h8*)(pb + ni * 1024);
                b[ni][1] = *(const h8*)(pb + (GB + ni) * 1024);
            }
#pragma unroll
            for (int mi = 0; mi < T::MI; ++mi) {
                const h8 hi = *(const h8*)(pa + mi * 1024), lo = *(const h8*)(pa + (GA + mi) * 1024);
#pragma unroll
                for (int ni = 0; ni < T::NI; ++ni) acc[mi][ni] = __builtin_amdgcn_mfma_f32_16x16x32_f16(b[ni][1], hi, acc[mi][ni], 0, 0, 0);
#pragma unroll
                for (int ni = 0; ni < T::NI; ++ni) acc[mi][ni] = __builtin_amdgcn_mfma_f32_16x16x32_f16(b[ni][0], lo, acc[mi][ni], 0, 0, 0);
#pragma unroll
                for (int ni = 0; ni < T::NI; ++ni) acc[mi][ni] = __builtin_amdgcn_mfma_f32_16x16x32_f16(b[ni][0], hi, acc[mi][ni], 0, 0, 0);
            }
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
