// A tile of a product of two matrices whose rows lie along the sum, C[i][j] = sum over k of A[i][k] B[j][k], in 8-bit floating point with a scale for each 128 of a
// row, or in pairs of fp16.  Internal to the library.
//
// A step takes 128 bytes of every row of the tile, which go straight from memory into one of the buffers in LDS (no registers in between) while the matrix
// instructions work on another.  A load writes 64 x 16 bytes one behind the other, eight rows; which sixteen bytes of its row a lane fetches is turned by
// half the row's number, so that the sixteen lanes that read one place of as many rows together meet all 64 banks (turned by the row's number itself, each read
// took eight cycles instead of four).  One barrier per step; the first operands of a step are read
// behind it and ahead of the last products of the step before, so the matrix unit has work across it.
//
// The 8-bit matrix instruction multiplies exactly and sums in fp32, but of each eight products it adds up first it drops what lies 2^-13 below the largest: results
// are 1.3e-5 off in the root mean square of theirs, however long the sum (measured, 128 to 4096 terms of a normal distribution), and never by more than 2^-10 of the eights'
// largest products' sum.  That is a sixteenth of fp16's rounding and a hundredth of bf16's, but where large products cancel, and far below what the operands' own
// rounding to four significand bits, 2^-4 of each, has put into the same products; for fp32 results the numbers are turned into bf16, scales applied, both exactly, and the 16-bit instruction sums them in fp32 throughout.
//
// Pairs of fp16: x = h + l, l what the rounding to h left, rounded: 22 bits.  128 bytes of a row are 32 h and their 32 l, and a product is h h' + h l' + l h', what it
// leaves off 2^-22 of it or less.  Where 11 bits do, a step takes 64 h of a row out of 256 bytes.
#ifndef ADATOPK_ROW_TILES_H
#define ADATOPK_ROW_TILES_H

#include "stage_ops.h"

namespace adatopk_stage {
#if defined(__HIPCC__)

typedef float F16v __attribute__((ext_vector_type(16)));
typedef int I8v __attribute__((ext_vector_type(8)));
typedef int I4v __attribute__((ext_vector_type(4)));
typedef _Float16 H8v __attribute__((ext_vector_type(8)));
typedef __bf16 B8v __attribute__((ext_vector_type(8)));
typedef __bf16 B2v __attribute__((ext_vector_type(2)));

constexpr int SLICE = 128;  // bytes of a row in a step

// All lanes where a < b, none where not, for copies.  (By the scalar unit: a mask that comes out of vector instructions would have to wait before it is used.)
__device__ __forceinline__ uint64_t lanes_if_less(int a, int b) {
    uint64_t lanes;
    asm volatile("s_cmp_lt_i32 %1, %2\n\ts_cselect_b64 %0, -1, 0" : "=s"(lanes) : "s"(a), "s"(b) : "scc");
    return lanes;
}
// (The compiler has no value of its own in m0 but what it writes there right before a use, and warns that it would not keep one; that these write it is said all the same.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
// From global memory straight into LDS: 16 (4) bytes per lane of `lanes`, from base + offset, to `to` + 16 (4) * lane.  All lanes of the wavefront are active
// around it.  Not waited for.  (Written out because the compiler waits for all of them before any read from LDS; there is no register in it that could be
// taken for written too early.)
__device__ __forceinline__ void copy_16(uint64_t base, uint32_t offset, uint32_t to, uint64_t lanes) {
    asm volatile("s_mov_b32 m0, %0\n\ts_mov_b64 exec, %3\n\tglobal_load_lds_dwordx4 %1, %2\n\ts_mov_b64 exec, -1" ::"s"(to), "v"(offset), "s"(base), "s"(lanes)
                 : "memory", "m0");
}
__device__ __forceinline__ void copy_4(uint64_t base, uint32_t offset, uint32_t to, uint64_t lanes) {
    asm volatile("s_mov_b32 m0, %0\n\ts_mov_b64 exec, %3\n\tglobal_load_lds_dword %1, %2\n\ts_mov_b64 exec, -1" ::"s"(to), "v"(offset), "s"(base), "s"(lanes)
                 : "memory", "m0");
}
#pragma clang diagnostic pop
__device__ __forceinline__ uint32_t lds_address(const void *p) {
    return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((const __attribute__((address_space(3))) void *)p));
}
template <int MORE> __device__ __forceinline__ void wait_copies() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(MORE) : "memory"); }
// All that this wavefront has asked for but the last MORE copies is there, and (MEET) every wavefront has come here.
template <int MORE, bool MEET> __device__ __forceinline__ void wait_and_meet() {
    if constexpr (MEET)
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(MORE) : "memory");
    else
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(MORE) : "memory");
}

// Eight numbers as bf16, times a power of two.
__device__ __forceinline__ B8v bf16_of(int lo, int hi, float scale) {
    const B2v a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
    const B2v c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
    return __builtin_shufflevector(__builtin_shufflevector(a, b, 0, 1, 2, 3), __builtin_shufflevector(c, d, 0, 1, 2, 3), 0, 1, 2, 3, 4, 5, 6, 7);
}
__device__ __forceinline__ float power_of(int S) { return __uint_as_float(static_cast<uint32_t>(S < 254 ? S : 254) << 23); }  // (numbers under S = 255 are NaN themselves)

enum Kind { PAIRS, HIGH, FP8_FAST, FP8_EXACT };  // of fp16; of those, the h alone; 8 bits by their own instruction; 8 bits as bf16

// WM x WN wavefronts, an equal part of the tile each, in blocks of 32 x 32: of those, a lane holds column lane % 32 of B's side and, of A's, the rows
// 8 * (q / 4) + 4 * (lane / 32) + q % 4.
//
// ALONG: so many groups of WM x WN wavefronts take turns along the sum, each with buffers of its own; a group of one wavefront meets nobody before its end.
// What they have then is to be added up.  For few tiles: a wavefront's block may be larger, which halves the reads from LDS that bound the smallest tiles.
template <Kind KIND, int BM_, int BN_, int WM_, int WN_, int STAGES_, int ALONG_ = 1> struct RowTile {
    static constexpr Kind FORM = KIND;
    static constexpr bool FP8 = KIND == FP8_FAST || KIND == FP8_EXACT, EXACT = KIND == FP8_EXACT;
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, STAGES = STAGES_, ALONG = ALONG_;
    static constexpr int WAVES = WM * WN, NT = WAVES * ALONG * 64, MI = BM / WM / 32, NI = BN / WN / 32;
    static constexpr int STRIDE = KIND == HIGH ? 2 * SLICE : SLICE, STEPS = EXACT || KIND == HIGH ? 4 : 2, TIMES = EXACT ? 2 : KIND == PAIRS ? 3 : 1;  // bytes of a row from slice to slice; of a slice; matrix instructions of one
    static constexpr int SCALES = FP8 ? 256 : 0;  // bytes for either side's scales: what a copy writes
    static constexpr int BUFFER = (BM + BN) * SLICE + 2 * SCALES, GROUP_LDS = STAGES * BUFFER, LDS = ALONG * GROUP_LDS;
    static constexpr int PA = BM / 8 / WAVES, PB = BN / 8 / WAVES;  // copies of a wavefront per slice
    // One block to a wavefront: too few products in a step for the reads from LDS of the next one, so a slice's operands are read together, a slice ahead.
    static constexpr bool WHOLE = MI * NI == 1;
    static_assert(BM == BN || WAVES > 1, "scales of both sides from one offset");
    static_assert(ALONG == 1 || WAVES == 1, "a group that has to meet is the workgroup");
    static_assert(PA >= 1 && PB >= 1 && BM % (8 * WAVES) == 0 && BN % (8 * WAVES) == 0 && MI >= 1 && NI >= 1, "whole pieces");

    // `source`: a, b: address of the tile's first row, where its slices begin; pitch_a, pitch_b: bytes from one row to the next; left_a, left_b: rows from the
    // tile's first one on (those behind are read as the last one); for FP8 scales_a(t), scales_b(t): addresses of the tile's scales of slice t.
    template <typename Source> static __device__ __forceinline__ void run(char *lds, const Source &source, int all_slices, F16v (&acc)[MI][NI]) {
        const int lane = threadIdx.x % 64, place = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), wave = place % WAVES, wm = wave / WN, wn = wave % WN;
        const int turn = ALONG == 1 ? 0 : place / WAVES;  // slices turn, turn + ALONG, ...
        const int slices = ALONG == 1 ? all_slices : (all_slices - turn + ALONG - 1) / ALONG;
        uint32_t from_a[PA], from_b[PB];
        const auto chunk = [&](int eight) { return (lane % 8) ^ (4 * (eight % 2) + lane / 16); };  // of the rows 8 * eight + lane / 8
#pragma unroll
        for (int q = 0; q < PA; ++q) {
            const int r = (wave * PA + q) * 8 + lane / 8, last = static_cast<int>(source.left_a) - 1;
            from_a[q] = static_cast<uint32_t>(r < last ? r : last) * static_cast<uint32_t>(source.pitch_a) + chunk(wave * PA + q) * 16;
        }
#pragma unroll
        for (int q = 0; q < PB; ++q) {
            const int r = (wave * PB + q) * 8 + lane / 8, last = static_cast<int>(source.left_b) - 1;
            from_b[q] = static_cast<uint32_t>(r < last ? r : last) * static_cast<uint32_t>(source.pitch_b) + chunk(wave * PB + q) * 16;
        }
        const uint32_t lds0 = lds_address(lds) + turn * GROUP_LDS;
        constexpr int LEAST = BM < BN ? BM : BN;
        const uint32_t from_scales = lane * 4 < (WAVES == 1 ? LEAST : wave < WAVES / 2 ? BM : BN) ? lane * 4 : 0;  // (what lies behind the tile's is not looked at)
        // Copy number n of slice t's: the wavefront's eights of rows of A, of B, and the scales of A (half of the wavefronts write them, equal) or B, or both.
        constexpr int COPIES = PA + PB + (FP8 ? (WAVES == 1 ? 2 : 1) : 0);
        auto copy = [&](int n, int t, uint32_t to, uint64_t lanes) {
            if (n < PA) {
                copy_16(source.a + static_cast<uint64_t>(turn + t * ALONG) * STRIDE, from_a[n < PA ? n : 0], to + (wave * PA + n) * 1024, lanes);
            } else if (n < PA + PB) {
                copy_16(source.b + static_cast<uint64_t>(turn + t * ALONG) * STRIDE, from_b[n >= PA && n < PA + PB ? n - PA : 0], to + BM * SLICE + (wave * PB + n - PA) * 1024, lanes);
            } else if constexpr (FP8) {
                const bool a = WAVES == 1 ? n == PA + PB : wave < WAVES / 2;
                copy_4(a ? source.scales_a(turn + t * ALONG) : source.scales_b(turn + t * ALONG), from_scales, to + (BM + BN) * SLICE + (a ? 0 : SCALES), lanes);
            }
        };
        // An operand's place: row lane % 32 of its block, sixteen bytes at a time, of which a slice has the ones below for each half of the wavefront.  Addresses
        // move from buffer to buffer; what is not written so the compiler takes a register for.
        constexpr int PLACES = 4;
        uint32_t at[2][PLACES], scales = lds0 + (BM + BN) * SLICE + lane % 32;
        typedef const __attribute__((address_space(3))) char Lds;
#pragma unroll
        for (int k = 0; k < PLACES; ++k) {
            // (8 bits by their instruction: a step's 32 bytes one behind the other, in two places; pairs: place 2 * step + piece)
            const uint32_t c = KIND == FP8_FAST ? 4 * (k / 2) + 2 * (lane / 32) + k % 2 : EXACT || KIND == HIGH ? 2 * k + lane / 32 : 4 * (k % 2) + 2 * (k / 2) + lane / 32;
            at[0][k] = lds0 + (wm * (BM / WM) + lane % 32) * SLICE + (c ^ (lane / 2 % 8)) * 16;
            at[1][k] = lds0 + BM * SLICE + (wn * (BN / WN) + lane % 32) * SLICE + (c ^ (lane / 2 % 8)) * 16;
        }
        auto pin = [&](uint32_t by) {
#pragma unroll
            for (int k = 0; k < PLACES; ++k) {
                at[0][k] += by;
                at[1][k] += by;
                asm("" : "+v"(at[0][k]), "+v"(at[1][k]));
            }
            if constexpr (FP8) {
                scales += by;
                asm("" : "+v"(scales));
            }
        };
        // Slice t + 1 is there, for every wavefront (what has been asked for and need not be: the slices after it, if there are as many as buffers for them), and
        // reads go to its buffer from now on.
        auto advance = [&](int t, uint32_t now) {
            if (STAGES > 2 && t + STAGES <= slices)
                wait_and_meet<(STAGES - 2) * COPIES, (WAVES > 1)>();
            else
                wait_and_meet<0, (WAVES > 1)>();
            pin(now == (STAGES - 1) * BUFFER ? 0u - (STAGES - 1) * BUFFER : BUFFER);
        };
        auto read = [&](uint32_t where, int block) { return *(const __attribute__((address_space(3))) I4v *)((Lds *)(uintptr_t)where + block * 32 * SLICE); };
        auto read_scale = [&](bool a, int block) {
            return static_cast<int>(*(const __attribute__((address_space(3))) uint8_t *)((Lds *)(uintptr_t)(scales + (a ? wm * (BM / WM) : SCALES + wn * (BN / WN))) + block * 32));
        };
        constexpr bool FAST = KIND == FP8_FAST;
        asm volatile("s_nop 4" ::: "memory");  // (an address that came out of the vector unit may be read by a load so much later; in the loop addresses are scalar sums)
#pragma unroll
        for (int b = 0; b < STAGES; ++b) {
            const uint64_t lanes = lanes_if_less(b, slices);
#pragma unroll
            for (int n = 0; n < COPIES; ++n) copy(n, b, lds0 + b * BUFFER, lanes);
        }
        if (slices >= STAGES)
            wait_copies<(STAGES - 1) * COPIES>();
        else
            wait_copies<0>();
        if constexpr (WAVES > 1) asm volatile("s_barrier" ::: "memory");
        pin(0);
        if constexpr (WHOLE) {
            // Everything a slice holds for the wavefront's block: four times sixteen bytes of either side, and the scales.
            I4v x[2][2][PLACES];
            int scale[2][2];
            auto take = [&](int n, int set) {  // the n-th of ten
                if (n >= 8) {
                    if constexpr (FP8) scale[set][n - 8] = read_scale(n == 8, 0);
                } else {
                    x[set][n % 2][n / 2] = read(at[n % 2][n / 2], 0);
                }
            };
            constexpr int TAKES = FP8 ? 10 : 8, PRODUCTS = STEPS * TIMES;
            auto multiply = [&](int m, int set) {
                if constexpr (FAST) {
                    const I8v a = __builtin_shufflevector(x[set][0][2 * m], x[set][0][2 * m + 1], 0, 1, 2, 3, 4, 5, 6, 7);
                    const I8v b = __builtin_shufflevector(x[set][1][2 * m], x[set][1][2 * m + 1], 0, 1, 2, 3, 4, 5, 6, 7);
                    acc[0][0] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, acc[0][0], 0, 0, 0, scale[set][0], 0, scale[set][1]);
                } else if constexpr (EXACT) {
                    const I4v a = x[set][0][m / 2], b = x[set][1][m / 2];
                    const int h = 2 * (m % 2);
                    acc[0][0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bf16_of(a[h], a[h + 1], power_of(scale[set][0])), bf16_of(b[h], b[h + 1], power_of(scale[set][1])),
                                                                        acc[0][0], 0, 0, 0);
                } else {
                    const int step = KIND == HIGH ? 0 : m / 3, a = KIND == HIGH ? m : m % 3 == 2, b = KIND == HIGH ? m : m % 3 == 1;
                    acc[0][0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(H8v, x[set][0][2 * step + a]), __builtin_bit_cast(H8v, x[set][1][2 * step + b]),
                                                                       acc[0][0], 0, 0, 0);
                }
            };
            auto slice = [&](int t, uint32_t now, auto which) {
                constexpr int SET = decltype(which)::value;
                const uint64_t lanes = lanes_if_less(t + STAGES, slices);
#pragma unroll
                for (int m = 0; m < PRODUCTS; ++m) {
                    multiply(m, SET);
                    if (m == 0) advance(t, now);
#pragma unroll
                    for (int n = m * TAKES / PRODUCTS; n < (m + 1) * TAKES / PRODUCTS; ++n) take(n, 1 - SET);
#pragma unroll
                    for (int n = m * COPIES / PRODUCTS; n < (m + 1) * COPIES / PRODUCTS; ++n) copy(n, t + STAGES, lds0 + now, lanes);
                    __builtin_amdgcn_sched_barrier(0);
                }
            };
#pragma unroll
            for (int n = 0; n < TAKES; ++n) take(n, 0);
            uint32_t now = 0;
            auto after = [](uint32_t now) { return now == (STAGES - 1) * BUFFER ? 0 : now + BUFFER; };
            for (int t = 0; t < slices; t += 2) {
                slice(t, now, std::integral_constant<int, 0>());
                now = after(now);
                if (t + 1 == slices) break;
                slice(t + 1, now, std::integral_constant<int, 1>());
                now = after(now);
            }
            return;
        }
        I8v xa8[2][FAST ? MI : 1], xb8[2][FAST ? NI : 1];
        H8v xa[2][2][FP8 ? 1 : MI], xb[2][2][FP8 ? 1 : NI];
        I4v raw_a[EXACT ? MI : 1], raw_b[EXACT ? NI : 1];
        B8v ya[2][2][EXACT ? MI : 1], yb[2][2][EXACT ? NI : 1];
        int sa[FP8 ? MI : 1], sb[FP8 ? NI : 1], sa_next[FP8 ? MI : 1], sb_next[FP8 ? NI : 1];
        // Operand n of a step, in the order in which the products want them: A's first block, B's, A's others.
        constexpr int OPERANDS = MI + NI;
        auto take = [&](int n, int step, int set) {
            const bool a = n == 0 || n > NI;
            const int k = n == 0 ? 0 : a ? n - NI : n - 1, side = a ? 0 : 1;
            if (FP8 && step == 0)
                (a ? sa_next[a ? k : 0] : sb_next[a ? 0 : k]) = read_scale(a, k);
            if constexpr (FAST) {
                (a ? xa8[set][a ? k : 0] : xb8[set][a ? 0 : k]) =
                    __builtin_shufflevector(read(at[side][2 * step], k), read(at[side][2 * step + 1], k), 0, 1, 2, 3, 4, 5, 6, 7);
            } else if constexpr (EXACT) {
                (a ? raw_a[a ? k : 0] : raw_b[a ? 0 : k]) = read(at[side][step], k);
            } else {
#pragma unroll
                for (int piece = 0; piece < (KIND == HIGH ? 1 : 2); ++piece)
                    (a ? xa[set][piece][a ? k : 0] : xb[set][piece][a ? 0 : k]) = __builtin_bit_cast(H8v, read(at[side][KIND == HIGH ? step : 2 * step + piece], k));
            }
        };
        // The operand, once it is there, in the form in which it is multiplied.
        auto convert = [&](int n, int step, int set) {
            const bool a = n == 0 || n > NI;
            const int k = n == 0 ? 0 : a ? n - NI : n - 1;
            if constexpr (EXACT) {
                const I4v raw = a ? raw_a[a ? k : 0] : raw_b[a ? 0 : k];
                if (step == 0) (a ? sa[a ? k : 0] : sb[a ? 0 : k]) = a ? sa_next[a ? k : 0] : sb_next[a ? 0 : k];
                const float scale = power_of(a ? sa[a ? k : 0] : sb[a ? 0 : k]);
#pragma unroll
                for (int h = 0; h < 2; ++h) (a ? ya[set][h][a ? k : 0] : yb[set][h][a ? 0 : k]) = bf16_of(raw[2 * h], raw[2 * h + 1], scale);
            }
        };
        auto multiply = [&](int m, int set) {
            const int h = m / (MI * NI), i = m / NI % MI, j = m % NI;
            if constexpr (FAST)
                acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(xa8[set][i], xb8[set][j], acc[i][j], 0, 0, 0, sa[i], 0, sb[j]);
            else if constexpr (EXACT)
                acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ya[set][h][i], yb[set][h][j], acc[i][j], 0, 0, 0);
            else
                acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(xa[set][h == 2 ? 1 : 0][i], xb[set][h == 1 ? 1 : 0][j], acc[i][j], 0, 0, 0);
        };
        // A slice: between two matrix instructions go the reads of the next step's operands and the copies of the slice that comes into the buffer left, a few
        // at a time (behind the last slice: reads of what is not looked at, and no copies).
        auto slice = [&](int t, uint32_t now) {
            constexpr int PRODUCTS = TIMES * MI * NI;
            constexpr int BY = EXACT ? PRODUCTS / 2 : PRODUCTS > 4 ? PRODUCTS - 3 : PRODUCTS;  // the reads are done some products before their use
            const uint64_t lanes = lanes_if_less(t + STAGES, slices);
            if constexpr (FAST) {
#pragma unroll
                for (int i = 0; i < MI; ++i) sa[i] = sa_next[i];
#pragma unroll
                for (int j = 0; j < NI; ++j) sb[j] = sb_next[j];
            }
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                const bool last = s + 1 == STEPS;
#pragma unroll
                for (int m = 0; m < PRODUCTS; ++m) {
                    multiply(m, s % 2);
                    if (last && m == 0) advance(t, now);
                    if (m < BY)
#pragma unroll
                        for (int n = m * OPERANDS / BY; n < (m + 1) * OPERANDS / BY; ++n) take(n, last ? 0 : s + 1, (s + 1) % 2);
                    else if (EXACT)
#pragma unroll
                        for (int n = (m - BY) * OPERANDS / BY; n < (m - BY + 1) * OPERANDS / BY; ++n) convert(n, last ? 0 : s + 1, (s + 1) % 2);
                    if (last)
#pragma unroll
                        for (int n = m * COPIES / PRODUCTS; n < (m + 1) * COPIES / PRODUCTS; ++n) copy(n, t + STAGES, lds0 + now, lanes);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        };
#pragma unroll
        for (int n = 0; n < OPERANDS; ++n) take(n, 0, 0);
#pragma unroll
        for (int n = 0; n < OPERANDS; ++n) convert(n, 0, 0);
        uint32_t now = 0;
        for (int t = 0; t < slices; ++t) {
            slice(t, now);
            now = now == (STAGES - 1) * BUFFER ? 0 : now + BUFFER;
        }
    }
};

// Workgroup b of n works on place(b) of n: eight runs of neighbours, one for each XCD (workgroups go round the XCDs), so that tiles which read the same
// rows share an L2.
__device__ __forceinline__ int place(int b, int n) {
    const int xcd = b % 8, per = n / 8, more = n % 8;
    return xcd * per + (xcd < more ? xcd : more) + b / 8;
}
// Tiles in bands of eight along one side, band by band, the other side within a band: the workgroups of an XCD that run at a time form a rectangle.
constexpr int BAND = 8;
__device__ __forceinline__ void tile_at(int tile, int tiles_a, int tiles_b, int &a, int &b) {
    const int band = tile / (BAND * tiles_b), in = tile - band * BAND * tiles_b;
    const int width = tiles_a - band * BAND < BAND ? tiles_a - band * BAND : BAND;
    b = in / width;
    a = band * BAND + in - b * width;
}
#endif  // __HIPCC__
}  // namespace adatopk_stage
#endif
