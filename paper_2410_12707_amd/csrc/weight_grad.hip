// The gradient of a projection's weight and bias: dW[n][k] = sum over tokens r of dY[r][n] * X[r][k], db[n] = sum of dY[r][n], with X kept in 8 bits.
//
// A matrix product whose long axis is the slow one of both operands.  Tiles of dY and X go through LDS as bf16, [token][feature], and come out
// transposed (ds_read_b64_tr_b16), which is what the matrix instruction wants.  A number of the 8-bit form times its step, a power of two, is
// exact in bf16; dY is taken apart into as many bf16 pieces as its type needs (bf16 one, fp16 two, fp32 three: the leading 8 bits, the next 8, the
// rest), so every product is exact and the sums are 32-bit (fp32 from 2^-110 on: below, the third piece ends at bf16's smallest number, 2^-133).
//
// With weight and bias of the layer norm whose normalised rows X holds, the projection's input was weight[k] * X + bias[k], so
// dW[n][k] = weight[k] * (dY^T X)[n][k] + db[n] * bias[k]: two operations per result instead of a rounding per element of X.
//
// Few tiles and many tokens: the tokens are split, partial products go to the workspace and k_weight_join adds them up in a fixed order.
#include <hip/hip_runtime.h>

#ifdef ADATOPK_MEASURE_BUILD
#include "adatopk_measure.h"
#endif
#include "stage_ops.h"

namespace {

using namespace adatopk_stage;

typedef __bf16 B4 __attribute__((ext_vector_type(4)));
typedef __bf16 B8 __attribute__((ext_vector_type(8)));
typedef float F16v __attribute__((ext_vector_type(16)));
typedef short S4 __attribute__((ext_vector_type(4)));

template <typename T> constexpr int pieces_of() { return sizeof(T) == 4 ? 3 : (__is_same(T, Bf16) ? 1 : 2); }

typedef __bf16 Pair __attribute__((ext_vector_type(2)));

constexpr int PAD = 32;  // elements behind a row of a tile in LDS: the four rows that one transposing read takes lie in different banks

struct Product {
    const void *dy;
    int64_t dy_stride;
    Act8 x;
    int64_t rows, n_out, n_in;
    int64_t rows_per_split;
    int tiles_in, tiles, split;  // of n_in, in all
    const void *weight, *bias;
    bool wide_weight;
    float *dw, *db;
    int accumulate;
    float *partial, *partial_db;  // [split][n_out][n_in], [split][n_out]
};

// The leading piece of each of two floats (bits cut off, so what is left is exact), and what is left.
__device__ __forceinline__ uint32_t cut(float &lo, float &hi, bool first) {
    const uint32_t a = __float_as_uint(lo) & 0xFFFF0000u, b = __float_as_uint(hi) & 0xFFFF0000u;
    // (of an infinity nothing is left, and nothing of what is left is one; of a NaN, a NaN)
    const bool inf_a = first && __builtin_fabsf(lo) == __builtin_inff(), inf_b = first && __builtin_fabsf(hi) == __builtin_inff();
    lo = inf_a ? 0.f : lo - __uint_as_float(a);
    hi = inf_b ? 0.f : hi - __uint_as_float(b);
    return a >> 16 | b;
}

__device__ __forceinline__ float weight_at(const void *p, bool wide, int dt_is_f16, int64_t i, float absent) {
    if (p == nullptr) return absent;
    if (wide) return static_cast<const float *>(p)[i];
    return dt_is_f16 ? to_f32(static_cast<const F16 *>(p)[i]) : to_f32(static_cast<const Bf16 *>(p)[i]);
}

// Workgroup b of n works on place(b) of n: eight runs of neighbours, one for each XCD (workgroups go round the XCDs), so that tiles which read the
// same columns share an L2.
__device__ __forceinline__ int place(int b, int n) {
    const int xcd = b % 8, per = n / 8, more = n % 8;
    return xcd * per + (xcd < more ? xcd : more) + b / 8;
}

// A tile's results to where they belong: the weight's gradient, or with the tokens split the partial products.  A register holds four rows' results of 32
// columns in each half of the wavefront, so a store's address is a scalar and an offset per lane.
// Results that are added to what is there (accumulate) wait for a read each, behind the last product and with nothing beside it: 2048 tokens, 4096 x 1024,
// bf16, 39.8 us without and 62.6 with; 16384 tokens, 6400 x 1600, 357 and 409.
template <typename T, int BM, int BN, int WM, int WN, int MI, int NI, typename Block>
__device__ __forceinline__ void finish(const Product &f, const F16v (&acc)[MI][NI], const float *sums, Block &&block, int64_t out0, int64_t own_out, int64_t in0,
                                       int64_t own_in, int part) {
    const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64), wm = wave / WN, wn = wave % WN;
    const bool last = f.split == 1;
    if (own_in == 0) {
        float *to = last ? f.db : f.partial_db + part * f.n_out;
        if (to != nullptr)
            for (int i = tid; i < BM && out0 + i < f.n_out; i += WM * WN * 64)
                if (out0 + i >= own_out) to[out0 + i] = sums[i] + (last && f.accumulate != 0 ? to[out0 + i] : 0.f);
    }
    const int64_t row0 = out0 + wm * (BM / WM), col0 = in0 + wn * (BN / WN);
    float *const to = (last ? f.dw : f.partial + part * f.n_out * f.n_in) + row0 * f.n_in + col0;
    const uint32_t offset = static_cast<uint32_t>(4 * (lane / 32)) * static_cast<uint32_t>(f.n_in) + lane % 32;
    const bool inside = out0 == own_out && out0 + BM <= f.n_out && in0 == own_in && in0 + BN <= f.n_in;
    const bool plain = !last || (f.weight == nullptr && f.bias == nullptr && f.accumulate == 0);
    if (inside && plain) {
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int q = 0; q < 16; ++q) {
                float *const row = to + (block(i) * 32 + 8 * (q / 4) + q % 4) * f.n_in;
#pragma unroll
                for (int j = 0; j < NI; ++j) row[offset + j * 32] = acc[i][j][q];
            }
        return;
    }
    float w[NI], v[NI];
    bool mine[NI];
#pragma unroll
    for (int j = 0; j < NI; ++j) {
        const int64_t c = col0 + j * 32 + lane % 32;
        mine[j] = c >= own_in && c < f.n_in;
        const bool there = last && mine[j];
        w[j] = there ? weight_at(f.weight, f.wide_weight || sizeof(T) == 4, __is_same(T, F16), c, 1.f) : 1.f;
        v[j] = there ? weight_at(f.bias, f.wide_weight || sizeof(T) == 4, __is_same(T, F16), c, 0.f) : 0.f;
    }
    const bool scaled = last && f.weight != nullptr, shifted = last && f.bias != nullptr, add = last && f.accumulate != 0;
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int q = 0; q < 16; ++q) {
            const int m = block(i) * 32 + 8 * (q / 4) + q % 4;
            const int64_t r = row0 + m + 4 * (lane / 32);
            if (!inside && (r >= f.n_out || r < own_out)) continue;
            float *const row = to + m * f.n_in;
            const float sum = shifted ? sums[wm * (BM / WM) + m + 4 * (lane / 32)] : 0.f;
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                if (!inside && !mine[j]) continue;
                float t = acc[i][j][q];
                if (scaled) t *= w[j];
                if (shifted) t = __builtin_fmaf(sum, v[j], t);
                if (add) t += row[offset + j * 32];
                row[offset + j * 32] = t;
            }
        }
}

// One tile of BM x BN results over one share of the tokens, WM x WN wavefronts, an equal part of the tile each.  Tiles of BK tokens go through two buffers in
// LDS: while the matrix instructions work on one, the next is converted into the other and the one behind it is on its way into registers.  One
// barrier per tile, and the last step's operands are in registers when it comes, so the matrix unit has work across it.
//
// 16384 tokens, 6400 x 1600, bf16 (tiles of 256 x 192): 368 us, 910 TFLOP/s.  Parts of the loop alone: the matrix instructions and the barrier 200 us, with
// the reads from LDS 235 to 257; the rest is dY and the 8-bit numbers on their way into LDS, whose conversion and stores share the issue slots and LDS
// with them.  512 tokens, 768 x 768, fp32 (three products): 11.5 us; 2049 tokens, 777 x 1000, fp16 (two): 29 us, both of them one workgroup
// to a compute unit, with its start and end and 8 steps of 0.85 us and 33 of 0.64.
//
// The last tile of a row or column of tiles begins so far ahead that it ends with the matrix (it stores what is its own), so loads need no bounds but
// those of the tokens.  SMALL: the matrix is narrower than the tile, or its rows too far apart for 32-bit offsets; every load is bounded.
template <typename T, int BM, int BN, int BK, int WM, int WN, int PER_CU, int AHEAD, bool SMALL>
__global__ __launch_bounds__(WM *WN * 64, PER_CU * WM * WN / 4) void k_weight_grad(Product f) {
    constexpr int NT = WM * WN * 64;
    constexpr int P = pieces_of<T>(), MI = BM / WM / 32, NI = BN / WN / 32, STEPS = BK / 16;
    constexpr int A_PITCH = BM + PAD, B_PITCH = BN + PAD, A_SIZE = BK * A_PITCH, BUFFER = P * A_SIZE + BK * B_PITCH;
    constexpr int A_OCTETS = BK * BM / 8 / NT, BW = BK * BN / 16 % NT == 0 ? 16 : 8, B_PIECES = BK * BN / BW / NT;
    constexpr int A_ROWS = NT / (BM / 8), B_ROWS = NT / (BN / BW);  // tokens from one of a thread's pieces of a tile to the next
    static_assert(BK * BM % (8 * NT) == 0 && BK * BN % (BW * NT) == 0 && NT % (BM / 8) == 0 && MI >= 1 && NI >= 1, "whole pieces");
    __shared__ __attribute__((aligned(16))) uint16_t lds[2 * BUFFER];
    __shared__ float sums[BM];
    const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64, wm = wave / WN, wn = wave % WN;
    const int b = place(blockIdx.x, gridDim.x);
    const int part = b / f.tiles, tile = b % f.tiles;
    const int64_t own_out = static_cast<int64_t>(tile / f.tiles_in) * BM, own_in = static_cast<int64_t>(tile % f.tiles_in) * BN;
    const int64_t out0 = SMALL || own_out + BM <= f.n_out ? own_out : f.n_out - BM, in0 = SMALL || own_in + BN <= f.x.pitch ? own_in : f.x.pitch - BN;
    const int64_t row0 = part * f.rows_per_split, row_end = row0 + f.rows_per_split < f.rows ? row0 + f.rows_per_split : f.rows;

    Raw<T> ra[AHEAD][A_OCTETS];  // of the AHEAD tiles behind the one in the next buffer
    typedef uint32_t Numbers __attribute__((ext_vector_type(BW / 4)));
    Numbers rb[AHEAD][B_PIECES];
    uint32_t re[AHEAD][B_PIECES];
    const int a_row = tid / (BM / 8), a_col = tid % (BM / 8) * 8;
    const uint32_t e_pitch = static_cast<uint32_t>(f.x.pitch / GROUP);
    const uint32_t a_at = (static_cast<uint32_t>(a_row) * static_cast<uint32_t>(f.dy_stride) + a_col) * sizeof(T);  // bytes from a tile's first element
    // (BN / BW need not divide NT: then a thread's pieces lie in different columns)
    constexpr bool B_EVEN = NT % (BN / BW) == 0;
    auto b_row = [&](int i) { return B_EVEN ? tid / (BN / BW) + i * B_ROWS : (tid + i * NT) / (BN / BW); };
    auto b_col = [&](int i) { return (B_EVEN ? tid : tid + i * NT) % (BN / BW) * BW; };
    uint32_t b_at[B_EVEN ? 1 : B_PIECES], e_at[B_EVEN ? 1 : B_PIECES];
#pragma unroll
    for (int i = 0; i < (B_EVEN ? 1 : B_PIECES); ++i) {
        b_at[i] = static_cast<uint32_t>(b_row(i)) * static_cast<uint32_t>(f.x.pitch) + b_col(i);
        e_at[i] = b_row(i) * e_pitch + b_col(i) / GROUP;
    }
    // Part `which` of `parts` of the tile that begins with token `row`, into registers.  WITHIN: all of its tokens are there.
    auto fetch = [&](auto within, int set, int64_t row, int which, int parts) {
        constexpr bool WITHIN = decltype(within)::value;
        typedef const __attribute__((address_space(1))) char Global;
        if (!WITHIN && row >= row_end) return;  // (what the registers hold goes into a buffer that nobody reads)
        if (WITHIN || (!SMALL && row + BK <= row_end)) {
            // (scalar bases that the optimiser cannot see through: an address is a base and a 32-bit offset, not a 64-bit variable of its own)
#pragma unroll
            for (int i = 0; i < B_PIECES; ++i) {
                if (i % parts != which) continue;
                const int64_t r = row + (B_EVEN ? i * B_ROWS : 0);
                uint64_t q = reinterpret_cast<uint64_t>(f.x.q + r * f.x.pitch + in0), e = reinterpret_cast<uint64_t>(f.x.e + r * e_pitch + in0 / GROUP);
                asm("" : "+s"(q), "+s"(e));
                rb[set][i] = *(const __attribute__((address_space(1))) Numbers *)((Global *)q + b_at[B_EVEN ? 0 : i]);
                re[set][i] = *(const __attribute__((address_space(1))) uint8_t *)((Global *)e + e_at[B_EVEN ? 0 : i]);
            }
#pragma unroll
            for (int i = 0; i < A_OCTETS; ++i) {
                if (i % parts != which) continue;
                uint64_t a = reinterpret_cast<uint64_t>(static_cast<const T *>(f.dy) + (row + i * A_ROWS) * f.dy_stride + out0);
                asm("" : "+s"(a));
                const auto at = (Global *)a + a_at;
                if constexpr (sizeof(T) == 4) {
                    ra[set][i].w[0] = *(const __attribute__((address_space(1))) U4a4 *)at;
                    ra[set][i].w[1] = *(const __attribute__((address_space(1))) U4a4 *)(at + 16);
                } else {
                    ra[set][i].w[0] = *(const __attribute__((address_space(1))) U4a2 *)at;
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < B_PIECES; ++i) {
                if (i % parts != which) continue;
                const int64_t r = row + b_row(i), c = in0 + b_col(i);
                const bool there = r < row_end && c < f.x.pitch;
                rb[set][i] = there ? *reinterpret_cast<const Numbers *>(f.x.q + r * f.x.pitch + c) : Numbers{};
                re[set][i] = there ? f.x.e[r * (f.x.pitch / GROUP) + c / GROUP] : 7;
            }
#pragma unroll
            for (int i = 0; i < A_OCTETS; ++i) {
                if (i % parts != which) continue;
                const int64_t r = row + a_row + i * A_ROWS, c = out0 + a_col;
                ra[set][i] = load_row(static_cast<const T *>(f.dy) + r * f.dy_stride + c, r < row_end ? f.n_out - c : 0, c > 0);
            }
        }
    };
    // Part `which` of `parts` of the tile in registers, into a buffer.
    auto stage = [&](int set, uint16_t *to, int which, int parts) {
        uint16_t *const a = to + a_row * A_PITCH + a_col, *const x = to + P * A_SIZE;
#pragma unroll
        for (int i = 0; i < A_OCTETS; ++i) {
            if (i % parts != which) continue;
            if constexpr (P == 1) {
                *reinterpret_cast<U4 *>(a + i * A_ROWS * A_PITCH) = ra[set][i].w[0];
            } else {
                float v[8];
                unpack(ra[set][i], v);
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    U4 d;
#pragma unroll
                    for (int j = 0; j < 4; ++j) d[j] = cut(v[2 * j], v[2 * j + 1], p == 0);
                    *reinterpret_cast<U4 *>(a + p * A_SIZE + i * A_ROWS * A_PITCH) = d;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < B_PIECES; ++i) {
            if (i % parts != which) continue;
#pragma unroll
            for (int h = 0; h < BW / 8; ++h) {
                float v[8];
                values_of(U2{rb[set][i][2 * h], rb[set][i][2 * h + 1]}, re[set][i], v);
                *reinterpret_cast<U4 *>(x + b_row(i) * B_PITCH + b_col(i) + 8 * h) = pack<Bf16>(v).w[0];
            }
        }
    };
    // What a lane holds of a 32 x 16 operand: feature lane % 32, tokens 8 * (lane / 32) and the seven behind it.  A transposing read works on blocks of
    // 16 lanes: lane i reads four features of token i / 4, and gets four tokens of feature i.
    //
    // The WN wavefronts along the tile's second side hold the same blocks of dY, each in an order that puts first the blocks whose sums over the tokens
    // it takes: block(i).
    constexpr int CI = (MI + WN - 1) / WN, TURN = MI < WN ? (MI > 1 ? 1 : 0) : MI / WN;
    const int token = 8 * (lane / 32) + lane % 16 / 4, feature = 16 * (lane / 16 % 2) + 4 * (lane % 4);
    auto block = [&](int i) { return (i + wn * TURN) % MI; };
    int a_lane[MI];
#pragma unroll
    for (int i = 0; i < MI; ++i) a_lane[i] = token * A_PITCH + wm * (BM / WM) + feature + block(i) * 32;
    const int b_lane = P * A_SIZE + token * B_PITCH + wn * (BN / WN) + feature;
    auto operand = [&](const uint16_t *at, int pitch) {
        typedef __attribute__((address_space(3))) S4 Lds;
        const S4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds *)(at));
        const S4 c = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds *)(at + 4 * pitch));
        const B4 x = __builtin_bit_cast(B4, a), y = __builtin_bit_cast(B4, c);
        return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    B8 xa[2][P][MI], xb[2][NI];
    auto take = [&](const uint16_t *from, int step, int set) {
#pragma unroll
        for (int j = 0; j < NI; ++j) xb[set][j] = operand(from + b_lane + step * 16 * B_PITCH + j * 32, B_PITCH);
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int i = 0; i < MI; ++i)
                xa[set][p][i] = operand(from + a_lane[i] + p * A_SIZE + step * 16 * A_PITCH, A_PITCH);
    };
    F16v acc[MI][NI] = {};
    float colsum[CI] = {};
    auto multiply = [&](int set) {
#pragma unroll
        for (int p = 0; p < P; ++p) {
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int j = 0; j < NI; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(xa[set][p][i], xb[set][j], acc[i][j], 0, 0, 0);
#pragma unroll
            for (int i = 0; i < CI; ++i) {
                const U4 d = __builtin_bit_cast(U4, xa[set][p][i]);
                const Pair one = {static_cast<__bf16>(1.f), static_cast<__bf16>(1.f)};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t two = d[j];
                    colsum[i] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(Pair, two), one, colsum[i], false);
                }
            }
        }
    };

    using Yes = std::true_type;
    using No = std::false_type;
    int64_t row = row0;
    fetch(No(), 0, row, 0, 1);
    stage(0, lds, 0, 1);
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) fetch(No(), i, row + (i + 1) * BK, 0, 1);
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): in the loop the loads come back in the loop's own order, and waits there count on it
    __syncthreads();
    take(lds, 0, 0);
    int cur = 0;
    // A tile: operands of the step after next are read, a part of the next tile is converted and the same part of the one behind it asked for, while
    // the matrix instructions of a step run.
    auto tile_of = [&](auto within, int set) {
        uint16_t *const now = lds + cur, *const next = lds + (BUFFER - cur);
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            if (s + 1 < STEPS) {
                take(now, s + 1, (s + 1) % 2);
                stage(set, next, s, STEPS - 1);
                fetch(within, set, row + (AHEAD + 1) * BK, s, STEPS - 1);
            } else {
                __syncthreads();
                take(next, 0, (s + 1) % 2);
            }
            multiply(s % 2);
#pragma unroll
            for (int g = 0; g < P * MI * NI; ++g) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
                __builtin_amdgcn_sched_group_barrier(0x002, 6, 0);
                __builtin_amdgcn_sched_group_barrier(0x200, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
            }
        }
        cur = BUFFER - cur;
        row += BK;
    };
    if constexpr (!SMALL)
        while (row + (2 * AHEAD + 1) * BK <= row_end) {
#pragma unroll
            for (int set = 0; set < AHEAD; ++set) tile_of(Yes(), set);
        }
    while (row < row_end) {
#pragma unroll
        for (int set = 0; set < AHEAD; ++set)
            if (set == 0 || row < row_end) tile_of(No(), set);
    }
#pragma unroll
    for (int i = 0; i < CI; ++i) {
        const float t = colsum[i] + __shfl_xor(colsum[i], 32);
        if (lane < 32 && wn * CI < MI) sums[wm * (BM / WM) + block(i) * 32 + lane] = t;
    }
    __syncthreads();
    finish<T, BM, BN, WM, WN>(f, acc, sums, block, out0, own_out, in0, own_in, part);
}

// The partial products added up in the order of the tokens, weight and bias applied.  Four results per thread, wherever rows end.  Bound by memory, and on
// small matrices by the launch: the planner counts 5 us and 0.4 us for each MB of a share's results.
struct Join {
    Product f;
    Divisor per_row;  // n_in
    int f16;
};
__global__ __launch_bounds__(256) void k_weight_join(Join w) {
    const Product &f = w.f;
    typedef float F4 __attribute__((ext_vector_type(4), aligned(4)));
    const int64_t all = f.n_out * f.n_in;
    const uint32_t first = (blockIdx.x * 256u + threadIdx.x) * 4u;
    if (first < f.n_out && f.db != nullptr) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (first + j >= f.n_out) break;
            float t = 0.f;
            for (int s = 0; s < f.split; ++s) t += f.partial_db[s * f.n_out + first + j];
            f.db[first + j] = t + (f.accumulate != 0 ? f.db[first + j] : 0.f);
        }
    }
    if (first >= all) return;
    float t[4] = {};
    const bool whole = first + 4 <= all;
    for (int s = 0; s < f.split; ++s) {
        const float *from = f.partial + s * all + first;
        if (whole) {
            const F4 v = *reinterpret_cast<const F4 *>(from);
#pragma unroll
            for (int j = 0; j < 4; ++j) t[j] += v[j];
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (first + j < all) t[j] += from[j];
        }
    }
    if (f.weight != nullptr || f.bias != nullptr) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t n = w.per_row.quotient(first + j), k = first + j - n * w.per_row.d;
            if (first + j >= all) break;
            if (f.weight != nullptr) t[j] *= weight_at(f.weight, f.wide_weight, w.f16, k, 1.f);
            if (f.bias != nullptr) {
                float sum = 0.f;
                for (int s = 0; s < f.split; ++s) sum += f.partial_db[s * f.n_out + n];
                t[j] = __builtin_fmaf(sum, weight_at(f.bias, f.wide_weight, w.f16, k, 0.f), t[j]);
            }
        }
    }
    float *to = f.dw + first;
    if (whole) {
        F4 v = {t[0], t[1], t[2], t[3]};
        if (f.accumulate != 0) v += *reinterpret_cast<const F4 *>(to);
        *reinterpret_cast<F4 *>(to) = v;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (first + j < all) to[j] = t[j] + (f.accumulate != 0 ? to[j] : 0.f);
    }
}

// Tiles that there are kernels for, as (BM, BN).
enum Tile { TILE_256_256, TILE_256_192, TILE_256_128, TILE_128_128, TILE_64_64, TILE_SMALL, TILES };
constexpr int TILE_BM[TILES] = {256, 256, 256, 128, 64, 64}, TILE_BN[TILES] = {256, 192, 128, 128, 64, 64};
constexpr int64_t MAX_STRIDE = 1 << 22;  // elements between rows of dY for 32-bit offsets within a tile
constexpr int SHARE = 64;  // tokens of the shortest share; shares are whole multiples of it

struct Cut {
    Tile tile;
    int tiles_in, tiles, split;
    int64_t rows_per_split;
};
// What a step of 64 tokens takes, us, with one workgroup on a compute unit and with as many as fit (two of the smaller tiles, but for fp32), by the
// pieces of dY (bf16, fp16, fp32) and by tile; and what a workgroup takes beside its steps.  Measured over 1024 and 4096 tokens with 256 and 512
// workgroups.  The larger tiles do two and a half times the work per time of the 64 x 64, but there are fewer of them: which tile and how many shares
// of the tokens are best is the least of the sums below.
constexpr float STEP_ALONE[3][TILES] = {{1.9f, 1.45f, 1.06f, 1.07f, 0.39f, 0.5f}, {3.25f, 0.f, 2.4f, 1.6f, 0.64f, 0.9f}, {4.55f, 0.f, 2.95f, 1.9f, 0.85f, 1.2f}};
constexpr float STEP_FULL[3][TILES] = {{1.9f, 1.45f, 1.06f, 1.31f, 0.58f, 0.8f}, {3.25f, 0.f, 2.4f, 2.46f, 1.01f, 1.4f}, {4.55f, 0.f, 2.95f, 1.9f, 0.85f, 1.2f}};
constexpr float BESIDE[TILES] = {14.f, 13.f, 8.f, 5.f, 4.5f, 5.f};
constexpr int SPLIT_MAX = 16;
int per_unit(int tile, int pieces) { return tile < TILE_128_128 || pieces == 3 ? 1 : 2; }  // (fp32's tiles take the LDS of one)

Cut cut_of(int64_t rows, int64_t n_out, int64_t n_in, adatopk_dtype dt, bool far) {
    Cut best{};
    double least = 0;
    const int pieces = dt == ADATOPK_BF16 ? 1 : (dt == ADATOPK_F16 ? 2 : 3);
    const int64_t steps = rows > 0 ? (rows + SHARE - 1) / SHARE : 1;
    for (int t = 0; t < TILES; ++t) {
        const bool fits = n_out >= TILE_BM[t] && adatopk_internal::act8_pitch(n_in) >= TILE_BN[t] && !far;
        if (t == TILE_SMALL ? best.split != 0 : !fits) continue;
        if (t == TILE_256_192 && pieces != 1) continue;  // (its octets do not divide evenly in the shorter tiles of the other types)
        const int64_t in = (n_in + TILE_BN[t] - 1) / TILE_BN[t], tiles = in * ((n_out + TILE_BM[t] - 1) / TILE_BM[t]);
        const int64_t places = 256 * per_unit(t, pieces);
        for (int64_t split = 1; split <= SPLIT_MAX && split <= steps && (split == 1 || n_out * n_in < (static_cast<int64_t>(1) << 31)); ++split) {
            const int64_t per = (steps + split - 1) / split;
            if ((steps + per - 1) / per != split) continue;
            const int64_t full = tiles * split / places, rest = tiles * split % places;
            const double alone = BESIDE[t] + static_cast<double>(STEP_ALONE[pieces - 1][t]) * per, together = BESIDE[t] + static_cast<double>(STEP_FULL[pieces - 1][t]) * per;
            // partial products written and read, and a launch: 5 us and 0.4 us for each MB of a share's
            const double join = split == 1 ? 0. : 5. + 0.4e-6 * 4. * static_cast<double>(split) * static_cast<double>(n_out * n_in);
            // workgroups that share a compute unit do not end together: their rounds run into one another
            const double rounds = per_unit(t, pieces) == 1 || full == 0 ? full * together + (rest == 0 ? 0. : rest <= 256 ? alone : together)
                                                                        : static_cast<double>(tiles * split) / places * together;
            const double cost = rounds + join;
            if (best.split == 0 || cost < least) {
                least = cost;
                best = Cut{static_cast<Tile>(t), static_cast<int>(in), static_cast<int>(tiles), static_cast<int>(split), per * SHARE};
            }
        }
    }
    return best;
}

constexpr int64_t MAX_FEATURES = 1 << 17;  // of either side: tiles, and rows of them, are counted in 32 bits

// Whether rows of dY lie too far apart for them.
bool far_apart(int64_t rows, int64_t dy_stride) { return rows > 1 && dy_stride >= MAX_STRIDE; }

bool product_ok(int64_t rows, int64_t n_out, int64_t n_in) {
    return shape_ok(rows, n_in) && n_out >= 0 && n_out <= MAX_FEATURES && n_in <= MAX_FEATURES && rows < (static_cast<int64_t>(1) << 31);
}

}  // namespace

extern "C" {

size_t adatopk_weight_grad_workspace_bytes(int64_t rows, int64_t n_out, int64_t n_in, adatopk_dtype dt) {
    if (!dtype_ok(dt) || !product_ok(rows, n_out, n_in)) return 0;
    if (n_out == 0 || n_in == 0) return 256;
    size_t most = 256;
    for (const bool far : {false, true}) {
        const Cut c = cut_of(rows, n_out, n_in, dt, far);
        const size_t bytes = static_cast<size_t>(c.split) * static_cast<size_t>(n_out) * (static_cast<size_t>(n_in) + 1) * sizeof(float);
        if (c.split > 1 && bytes > most) most = bytes;
    }
    return align_up(most, 256);
}

adatopk_status adatopk_weight_grad(const void *dy, int64_t dy_stride, const void *act8_x, int64_t rows, int64_t n_out, int64_t n_in, adatopk_dtype dt,
                                   const void *weight, const void *bias, adatopk_dtype weight_dt, float *dw, float *db, int32_t accumulate,
                                   void *workspace, size_t workspace_bytes, void *hip_stream) {
    if (!dtype_ok(dt) || !(weight_dt == dt || weight_dt == ADATOPK_F32) || !product_ok(rows, n_out, n_in)) return ADATOPK_EINVAL;
    if (n_out == 0 || n_in == 0) return ADATOPK_OK;
    const size_t weight_size = static_cast<size_t>(elem_size(weight_dt));
    if (!pointer_ok(dw, 4) || !pointer_ok_or_null(db, 4) || !pointer_ok_or_null(weight, weight_size) || !pointer_ok_or_null(bias, weight_size) ||
        !pointer_ok(workspace, 256) || (rows > 0 && (!matrix_ok(dy, dy_stride, rows, n_out, dt) || !pointer_ok(act8_x, 16))))
        return ADATOPK_EINVAL;
    if (workspace_bytes < adatopk_weight_grad_workspace_bytes(rows, n_out, n_in, dt)) return ADATOPK_EWORKSPACE;
    const Cut c = cut_of(rows, n_out, n_in, dt, far_apart(rows, dy_stride));
    float *partial = static_cast<float *>(workspace);
    const bool wide = weight_dt == ADATOPK_F32;
    const Product f{dy,     dy_stride, act8_of(const_cast<void *>(act8_x), rows, n_in), rows, n_out, n_in, c.rows_per_split, c.tiles_in, c.tiles, c.split,
                    weight, bias,      wide, dw, db, accumulate, partial, partial + static_cast<int64_t>(c.split) * n_out * n_in};
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    with_type(dt, [&](auto *null) {
        using T = std::remove_pointer_t<decltype(null)>;
        constexpr int DEEP = pieces_of<T>() == 1 ? 64 : 32;  // tokens of a tile: what two buffers have room for
        const auto launch = [&](auto kernel, int threads) {
            hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(c.tiles * c.split)), dim3(static_cast<unsigned>(threads)), 0, st, f);
        };
        if (c.tile == TILE_256_256)
            launch(k_weight_grad<T, 256, 256, DEEP, 4, 2, 1, 1, false>, 512);
        else if (c.tile == TILE_256_128)
            launch(k_weight_grad<T, 256, 128, DEEP, 4, 2, 1, 1, false>, 512);
        else if (c.tile == TILE_256_192) {
            if constexpr (pieces_of<T>() == 1) launch(k_weight_grad<T, 256, 192, DEEP, 2, 2, 1, 1, false>, 256);
        } else if (c.tile == TILE_128_128)
            launch(k_weight_grad<T, 128, 128, 32, 2, 2, pieces_of<T>() < 3 ? 2 : 1, 1, false>, 256);
        else if (c.tile == TILE_64_64)
            launch(k_weight_grad<T, 64, 64, 64, 2, 2, pieces_of<T>() < 3 ? 2 : 1, 2, false>, 256);
        else
            launch(k_weight_grad<T, 64, 64, 64, 2, 2, pieces_of<T>() < 3 ? 2 : 1, 2, true>, 256);
    });
    if (c.split > 1)
        hipLaunchKernelGGL(k_weight_join, dim3(static_cast<unsigned>((n_out * n_in + 1023) / 1024)), dim3(256), 0, st,
                           Join{f, Divisor(static_cast<uint32_t>(n_in)), weight_dt == ADATOPK_F16 ? 1 : 0});
    return launched();
}

#ifdef ADATOPK_MEASURE_BUILD
adatopk_status adatopk_measure_weight_grad_cut(int64_t rows, int64_t n_out, int64_t n_in, adatopk_dtype dt, int64_t dy_stride, int32_t *out) {
    if (!dtype_ok(dt) || !product_ok(rows, n_out, n_in) || n_out == 0 || n_in == 0) return ADATOPK_EINVAL;
    const Cut c = cut_of(rows, n_out, n_in, dt, far_apart(rows, dy_stride));
    out[0] = TILE_BM[c.tile];
    out[1] = TILE_BN[c.tile];
    out[2] = c.tile == TILE_SMALL ? 1 : 0;
    out[3] = c.split;
    return ADATOPK_OK;
}
#endif

}  // extern "C"
