// The product of two matrices in 8-bit floating point, y = x W^T + bias + add.
//
// The scales are powers of two, a byte for 128 of a row: the matrix instruction applies them as it goes, or the conversion to bf16 where results are fp32
// (row_tiles.h says why); products are exact and sums are fp32, one chain over the sum's axis per share of it.  The weights are the instruction's first operand, so that
// a lane's results are neighbours in a row of y.  Three forms: tiles of row_tiles.h, each workgroup one; the same with the sum's axis shared out where tiles are few,
// partial sums to the workspace and k_fp8_join behind; and for a few tokens k_fp8_few, which reads the weights once and straight into registers.
//
// Measured, us, 16-bit results and fp32 ones: one token 1600 -> 6400 4.2 to 4.6, 4.7; 512 tokens 768 -> 768 5.8, 6.8; 2048 x 2048 x 2048 16.5, 24.8; 4096 x 4096 x 4096 56 to 62, 106 (2.2 to 2.5
// and 1.3 PFLOP/s); 16384 tokens 1600 -> 6400 175 to 188, 310 (1.8 to 1.9 and 1.1), where a library's product with one scale for each matrix takes 200.  Large products are bound by the
// matrix unit's power (of zeros 4096 x 4096 x 8192 takes 87, of noise 107), small ones by the launch and the latency of the first slices, a few tokens' by the
// weights' bytes.
#include <hip/hip_runtime.h>

#ifdef ADATOPK_MEASURE_BUILD
#include "adatopk_measure.h"
#endif
#include "fp8_form.h"
#include "row_tiles.h"

namespace {

using namespace adatopk_stage;

struct Product {
    Fp8 x, w;
    int64_t rows, n_out;
    int slices, split, slices_per_split;  // of the sum's axis
    int tiles_out, tiles_rows;            // along features and tokens
    const void *bias, *add;
    bool wide_bias;
    int64_t add_stride, y_stride;
    void *y;
    float *partial;  // [split][rows][n_out]
};

// Eight results to y: bias and summand added, one rounding.
template <typename T> __device__ __forceinline__ void put(const Product &f, int64_t row, int64_t col, const float (&bias)[8], float (&v)[8]) {
    const int64_t left = f.n_out - col;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] += bias[j];
    if (f.add != nullptr) {
        float t[8];
        unpack(load_row(static_cast<const T *>(f.add) + row * f.add_stride + col, left, col > 0), t);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += t[j];
    }
    store_row(static_cast<T *>(f.y) + row * f.y_stride + col, left, pack<T>(v));
}
template <typename T> __device__ __forceinline__ void load_bias(const Product &f, int64_t col, float (&b)[8]) {
    const int64_t left = f.n_out - col;
    if (f.bias == nullptr) {
#pragma unroll
        for (int j = 0; j < 8; ++j) b[j] = 0.f;
    } else if (f.wide_bias) {
        unpack(load_row(static_cast<const float *>(f.bias) + col, left, col > 0), b);
    } else {
        unpack(load_row(static_cast<const T *>(f.bias) + col, left, col > 0), b);
    }
}

struct Source {
    uint64_t a, b, sa, sb;  // of the first slice
    int64_t pitch_a, pitch_b, left_a, left_b, scale_pitch_a, scale_pitch_b;
    __device__ __forceinline__ uint64_t scales_a(int t) const { return sa + static_cast<uint64_t>(t) * scale_pitch_a; }
    __device__ __forceinline__ uint64_t scales_b(int t) const { return sb + static_cast<uint64_t>(t) * scale_pitch_b; }
};

// Bytes of LDS: the tile's buffers, and behind the sums its results.
template <typename Tile> constexpr int RESULTS_PITCH = Tile::MI * 32 + 4;  // floats from one token's results to the next
template <typename Tile> constexpr int LDS_BYTES = Tile::LDS > Tile::WAVES * 32 * RESULTS_PITCH<Tile> * 4 ? Tile::LDS : Tile::WAVES * 32 * RESULTS_PITCH<Tile> * 4;

// The tile from feature out0 and token row0 on, of share `part` of the sum.
template <typename T, typename Tile> __device__ __forceinline__ void product_of_tile(const Product &f, char *lds, int64_t out0, int64_t row0, int part) {
    constexpr int MI = Tile::MI, NI = Tile::NI, PITCH = RESULTS_PITCH<Tile>;
    static_assert(Tile::ALONG == 1 || Tile::BN * PITCH * 4 <= Tile::GROUP_LDS, "a group's results fit its buffers");
    const int first = part * f.slices_per_split, slices = f.slices - first < f.slices_per_split ? f.slices - first : f.slices_per_split;
    const Source source{reinterpret_cast<uint64_t>(f.w.q + out0 * f.w.pitch + first * static_cast<int64_t>(SLICE)),
                        reinterpret_cast<uint64_t>(f.x.q + row0 * f.x.pitch + first * static_cast<int64_t>(SLICE)),
                        reinterpret_cast<uint64_t>(f.w.s + first * f.w.scale_pitch + out0),
                        reinterpret_cast<uint64_t>(f.x.s + first * f.x.scale_pitch + row0),
                        f.w.pitch, f.x.pitch, f.n_out - out0 < Tile::BM ? f.n_out - out0 : Tile::BM, f.rows - row0 < Tile::BN ? f.rows - row0 : Tile::BN,
                        f.w.scale_pitch, f.x.scale_pitch};
    F16v acc[MI][NI] = {};
    Tile::run(lds, source, slices, acc);
    __syncthreads();  // the buffers have been read

    // Results through LDS: rows of y are written in whole lines.  AT: octets that a thread has under way at a time.
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), wm = wave % Tile::WAVES / Tile::WN, wn = wave % Tile::WN;
    const auto lay = [&](float *to, int j) {  // a wavefront's results of 32 tokens
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                typedef float F4 __attribute__((ext_vector_type(4)));
                *reinterpret_cast<F4 *>(to + lane % 32 * PITCH + i * 32 + q * 8 + lane / 32 * 4) =
                    F4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
            }
    };
    constexpr int OCTETS = MI * 4, AT = 4;
    // Lines first, first + step, ... below `lines` of what `from` holds, GROUPS sums of each a distance apart; line 0 is token `row_at`.
    const auto write = [&](auto groups, const float *from, int first, int step, int lines, int64_t row_at, int octet, int64_t col) {
        constexpr int GROUPS = decltype(groups)::value, APART = Tile::GROUP_LDS / 4;
        if (col >= f.n_out) return;
        const int64_t left = f.n_out - col;
        float bias[8] = {};
        if (f.split == 1) load_bias<T>(f, col, bias);
#pragma unroll 1
        for (int k = first; k < lines; k += AT * step) {
            float v[AT][8];
            Raw<T> add[AT];
#pragma unroll
            for (int u = 0; u < AT; ++u) {
                const int64_t row = row_at + k + u * step;
                if (f.split == 1 && f.add != nullptr)
                    add[u] = fetch_row(static_cast<const T *>(f.add) + row * f.add_stride + col, k + u * step < lines && row < f.rows ? left : 0, col > 0);
                if (k + u * step >= lines) continue;
#pragma unroll
                for (int g = 0; g < GROUPS; ++g) {
                    const U4 *const at = reinterpret_cast<const U4 *>(from + g * APART + (k + u * step) * PITCH + octet * 8);
                    float t[8];
                    unpack(Raw<float>{{at[0], at[1]}}, t);
#pragma unroll
                    for (int x = 0; x < 8; ++x) v[u][x] = g == 0 ? t[x] : v[u][x] + t[x];
                }
            }
#pragma unroll
            for (int u = 0; u < AT; ++u) {
                const int64_t row = row_at + k + u * step;
                if (k + u * step >= lines || row >= f.rows) continue;
                if (f.split > 1) {
                    store_row(f.partial + (part * f.rows + row) * f.n_out + col, left, pack<float>(v[u]));
                    continue;
                }
#pragma unroll
                for (int x = 0; x < 8; ++x) v[u][x] += bias[x];
                if (f.add != nullptr) {
                    float t[8];
                    unpack(settle(add[u], left, col > 0), t);
#pragma unroll
                    for (int x = 0; x < 8; ++x) v[u][x] += t[x];
                }
                store_row(static_cast<T *>(f.y) + row * f.y_stride + col, left, pack<T>(v[u]));
            }
        }
    };
    if constexpr (Tile::ALONG > 1) {  // the groups' sums, added up in their order; the workgroup goes through the tile together
        float *const sums = reinterpret_cast<float *>(lds);
#pragma unroll
        for (int j = 0; j < NI; ++j) lay(sums + wave * (Tile::GROUP_LDS / 4) + j * 32 * PITCH, j);
        __syncthreads();
        const int octet = threadIdx.x % OCTETS;
        write(std::integral_constant<int, Tile::ALONG>(), sums, threadIdx.x / OCTETS, Tile::NT / OCTETS, Tile::BN, row0, octet, out0 + octet * 8);
    } else {
        float *const mine = reinterpret_cast<float *>(lds) + wave * 32 * PITCH;
        const auto together = [] {  // (a wavefront's lanes read what others of them have written)
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        };
        const int octet = lane % OCTETS;
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            lay(mine, j);
            together();
            write(std::integral_constant<int, 1>(), mine, lane / OCTETS, 64 / OCTETS, 32, row0 + wn * (Tile::BN / Tile::WN) + j * 32, octet,
                  out0 + wm * (Tile::BM / Tile::WM) + octet * 8);
            together();
        }
    }
}

template <typename T, typename Tile, int PER_CU> __global__ __launch_bounds__(Tile::NT, PER_CU * Tile::NT / 256) void k_fp8_product(Product f) {
    __shared__ __attribute__((aligned(16))) char lds[LDS_BYTES<Tile>];
    const int tiles = f.tiles_out * f.tiles_rows, b = place(blockIdx.x, gridDim.x), part = b / tiles;
    int tile_out, tile_row;
    tile_at(b - part * tiles, f.tiles_out, f.tiles_rows, tile_out, tile_row);
    product_of_tile<T, Tile>(f, lds, static_cast<int64_t>(tile_out) * Tile::BM, static_cast<int64_t>(tile_row) * Tile::BN, part);
}

// The same with the first `whole` tiles as they are and each of the others in four, so that what is left behind the last full round of the chip is done in a
// part of a round's time.
template <typename T, typename Tile, typename Quarter> __global__ __launch_bounds__(Tile::NT, Tile::NT / 256) void k_fp8_product_quartered(Product f, int whole) {
    static_assert(Quarter::NT == Tile::NT && 2 * Quarter::BM == Tile::BM && 2 * Quarter::BN == Tile::BN && LDS_BYTES<Quarter> <= LDS_BYTES<Tile>, "a quarter");
    __shared__ __attribute__((aligned(16))) char lds[LDS_BYTES<Tile>];
    const int b = blockIdx.x;
    const bool all = b < whole;
    const int at = all ? place(b, whole) : place(b - whole, gridDim.x - whole);
    int tile_out, tile_row;
    tile_at(all ? at : whole + at / 4, f.tiles_out, f.tiles_rows, tile_out, tile_row);
    int64_t out0 = static_cast<int64_t>(tile_out) * Tile::BM, row0 = static_cast<int64_t>(tile_row) * Tile::BN;
    if (all) return product_of_tile<T, Tile>(f, lds, out0, row0, 0);
    out0 += at % 2 * Quarter::BM;
    row0 += at % 4 / 2 * Quarter::BN;
    if (out0 < f.n_out && row0 < f.rows) product_of_tile<T, Quarter>(f, lds, out0, row0, 0);
}

// Partial sums added up in the order of the sum's axis.  An octet of a row per thread.
template <typename T> __global__ __launch_bounds__(256) void k_fp8_join(Product f, Divisor per_row, uint32_t octets) {
    const uint32_t t = blockIdx.x * 256u + threadIdx.x;
    if (t >= octets) return;
    const uint32_t row = per_row.quotient(t);
    const int64_t col = (t - row * per_row.d) * static_cast<int64_t>(8), left = f.n_out - col;
    float v[8] = {}, bias[8];
    for (int s = 0; s < f.split; ++s) {
        float p[8];
        unpack(load_row(f.partial + (s * f.rows + row) * f.n_out + col, left, col > 0), p);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += p[j];
    }
    load_bias<T>(f, col, bias);
    put<T>(f, row, col, bias, v);
}

// A few tokens: a workgroup takes sixteen features, its wavefronts take turns along the sum's axis.  A lane reads 32 bytes of a row, four neighbours a line.
// The wavefronts' sums are added up in their order.
constexpr int FEW_WAVES = 8, FEW_AHEAD = 4;
template <typename T, int TJ> __global__ __launch_bounds__(FEW_WAVES * 64) void k_fp8_few(Product f) {
    typedef float F4 __attribute__((ext_vector_type(4)));
    __shared__ F4 share[FEW_WAVES][TJ][64];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int64_t out0 = static_cast<int64_t>(blockIdx.x) * 16;
    const int64_t feature = out0 + lane % 16 < f.n_out ? out0 + lane % 16 : f.n_out - 1;
    const uint8_t *const w = f.w.q + feature * f.w.pitch + lane / 16 * 32;
    int64_t token[TJ];
#pragma unroll
    for (int j = 0; j < TJ; ++j) token[j] = j * 16 + lane % 16 < f.rows ? j * 16 + lane % 16 : f.rows - 1;
    F4 acc[TJ] = {};
    for (int t0 = wave; t0 < f.slices; t0 += FEW_WAVES * FEW_AHEAD) {
        I4v a[FEW_AHEAD][2], b[FEW_AHEAD][TJ][2];
        int sa[FEW_AHEAD], sb[FEW_AHEAD][TJ];
#pragma unroll
        for (int u = 0; u < FEW_AHEAD; ++u) {
            const int t = t0 + u * FEW_WAVES;
            if (t >= f.slices) break;
            const I4v *const from = reinterpret_cast<const I4v *>(w + t * static_cast<int64_t>(SLICE));
            a[u][0] = from[0];
            a[u][1] = from[1];
            sa[u] = f.w.s[t * f.w.scale_pitch + feature];
#pragma unroll
            for (int j = 0; j < TJ; ++j) {
                const I4v *const at = reinterpret_cast<const I4v *>(f.x.q + token[j] * f.x.pitch + lane / 16 * 32 + t * static_cast<int64_t>(SLICE));
                b[u][j][0] = at[0];
                b[u][j][1] = at[1];
                sb[u][j] = f.x.s[t * f.x.scale_pitch + token[j]];
            }
        }
#pragma unroll
        for (int u = 0; u < FEW_AHEAD; ++u) {
            if (t0 + u * FEW_WAVES >= f.slices) break;
#pragma unroll
            for (int j = 0; j < TJ; ++j) {
                if constexpr (sizeof(T) == 4) {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bf16_of(a[u][k / 2][k % 2 * 2], a[u][k / 2][k % 2 * 2 + 1], power_of(sa[u])),
                                                                         bf16_of(b[u][j][k / 2][k % 2 * 2], b[u][j][k / 2][k % 2 * 2 + 1], power_of(sb[u][j])), acc[j],
                                                                         0, 0, 0);
                } else {
                    acc[j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
                        __builtin_shufflevector(a[u][0], a[u][1], 0, 1, 2, 3, 4, 5, 6, 7), __builtin_shufflevector(b[u][j][0], b[u][j][1], 0, 1, 2, 3, 4, 5, 6, 7),
                        acc[j], 0, 0, 0, sa[u], 0, sb[u][j]);
                }
            }
        }
    }
#pragma unroll
    for (int j = 0; j < TJ; ++j) share[wave][j][lane] = acc[j];
    __syncthreads();
    // a lane of the sums holds token lane % 16, features 4 * (lane / 16) ... + 3
    for (int i = threadIdx.x; i < TJ * 256; i += FEW_WAVES * 64) {
        const int j = i / 256, which = i % 16, mine = i % 256 / 16;  // feature, token
        const int64_t row = j * 16 + mine, col = out0 + which;
        if (row >= f.rows || col >= f.n_out) continue;
        float v = 0.f;
#pragma unroll
        for (int k = 0; k < FEW_WAVES; ++k) v += share[k][j][which / 4 * 16 + mine][which % 4];
        if (f.bias != nullptr) v += f.wide_bias ? static_cast<const float *>(f.bias)[col] : to_f32(static_cast<const T *>(f.bias)[col]);
        if (f.add != nullptr) v += to_f32(static_cast<const T *>(f.add)[row * f.add_stride + col]);
        from_f32(v, static_cast<T *>(f.y) + row * f.y_stride + col);
    }
}

enum Form { LARGE, MIDDLE, SMALL, DEEP, TILED, FEW = TILED, NONE };
template <Kind KIND> struct Tiles {
    using Large = RowTile<KIND, 256, 256, 2, 4, 2>;
    using Quarter = RowTile<KIND, 128, 128, 2, 4, 2>;  // of Large, by as many wavefronts
    using Middle = RowTile<KIND, 128, 128, 2, 2, 2>;
    using Small = RowTile<KIND, 64, 64, 2, 2, 2>;
    using Deep = RowTile<KIND, 64, 64, 1, 1, 2, 4>;
};
constexpr int SIDE[TILED] = {256, 128, 64, 64}, SLOTS[TILED] = {256, 512, 1024, 256};  // of the chip

struct Cut {
    Form form;
    int tiles_out, tiles_rows, slices, split, per;
    int whole;  // tiles; the others in quarters
};
// us: of a slice of 128 for a workgroup with a few others on the chip and on a full one, and what a workgroup takes beside; by the 8-bit instruction, and as bf16 for fp32
// results.  Measured at 14 sizes (and ten of 1 to 64 tokens for FEW_ROWS below), 65 x 768 x 768 to 16384 x 1600 x 6400: by tile 193, 216, 302, 550 us there, 57, 69, 115, 140 for 4096 x 4096 x 4096, 17, 8.6, 6.0, 6.4
// for 1024 x 1024 x 1024, 57, 24, 17, 11 for 128 x 6400 x 1600.
constexpr double STEP_ALONE[2][TILED] = {{1.0, 0.38, 0.25, 0.125}, {1.95, 0.66, 0.38, 0.2}}, STEP_FULL[2][TILED] = {{1.5, 0.88, 0.69, 0.16}, {3.1, 1.7, 1.1, 0.26}};
constexpr double BESIDE[2][TILED] = {{8., 6., 4.8, 5.}, {10., 8., 5.5, 5.3}};
// Up to so many of the largest tiles behind the last full round are done in quarters, all at a time.  16384 x 6400 by 512, 1600, 4096 (64 of them): 109, 191, 364 us
// without, 99, 185, 353 with; of 160 and 224, where the quarters go round, 53 without and 58 with, 54 and 63 (8192 x 3328 and 3840 by 1600).
constexpr int64_t QUARTERED = 64;
constexpr double QUARTER_STEP[2] = {0.5, 0.9}, QUARTER_BESIDE[2] = {6., 8.};
// Up to so many tokens k_fp8_few is as quick or quicker: 16 tokens, 1600 x 6400, 5.3 us against 6.6, 32 tokens, 6400 x 1600, 10.9 against 12.2; 48, 1600 x 6400, 10.5
// against 7.0.
constexpr int64_t FEW_ROWS = 32;
constexpr int SPLIT_MAX = 16;
Cut cut_of(int64_t rows, int64_t n_out, int64_t n_in, bool exact) {
    const int slices = static_cast<int>(adatopk_internal::fp8_pitch(n_in) / SLICE);
    Cut best{FEW, 0, 0, slices, 1, slices, 0};
    if (slices == 0) best.form = NONE;  // (nothing to add up: what the join adds to no shares)
    if (rows <= FEW_ROWS || slices == 0) return best;
    double least = 0;
    for (int t = 0; t < TILED; ++t) {
        const int64_t out = (n_out + SIDE[t] - 1) / SIDE[t], along = (rows + SIDE[t] - 1) / SIDE[t], tiles = out * along;
        for (int split = 1; split <= SPLIT_MAX && split <= slices; ++split) {
            const int per = (slices + split - 1) / split;
            if ((slices + per - 1) / per != split) continue;
            const double filled = static_cast<double>(tiles * split) / SLOTS[t], some = filled < 1. ? filled : 1.;
            // workgroups that share a compute unit do not end together: their rounds run into one another
            const double rounds = filled <= 1. ? 1. : SLOTS[t] > 256 ? filled : static_cast<double>((tiles * split + 255) / 256);
            const double step = STEP_ALONE[exact][t] + some * (STEP_FULL[exact][t] - STEP_ALONE[exact][t]);
            const double join = split == 1 ? 0. : 4.5 + 0.4e-6 * 4. * split * static_cast<double>(rows) * static_cast<double>(n_out);
            const double one = BESIDE[exact][t] + step * per;
            double cost = rounds * one + join;
            int64_t left = 0;  // tiles in quarters
            if (t == LARGE && split == 1 && tiles > 256 && tiles % 256 != 0 && tiles % 256 <= QUARTERED) {
                left = tiles % 256;
                cost -= one - QUARTER_BESIDE[exact] - QUARTER_STEP[exact] * per;
            }
            if (best.form == FEW || cost < least) {
                least = cost;
                best = Cut{static_cast<Form>(t), static_cast<int>(out), static_cast<int>(along), slices, split, per, static_cast<int>(tiles - left)};
            }
        }
    }
    return best;
}
size_t shares_bytes(const Cut &c, int64_t rows, int64_t n_out) {
    return c.split == 1 ? 0 : align_up(static_cast<size_t>(c.split) * static_cast<size_t>(rows) * static_cast<size_t>(n_out) * sizeof(float), 256);
}

constexpr int64_t MAX_FEATURES = 1 << 17;
bool product_ok(int64_t rows, int64_t n_out, int64_t n_in) {
    return n_out >= 0 && n_in >= 0 && n_out <= MAX_FEATURES && n_in <= MAX_FEATURES && rows >= 0 && rows < (static_cast<int64_t>(1) << 31) && fp8_shape_ok(rows, n_in) &&
           fp8_shape_ok(n_out, n_in) && shape_ok(rows, n_out);
}

}  // namespace

extern "C" {

size_t adatopk_fp8_product_workspace_bytes(int64_t rows, int64_t n_out, int64_t n_in) {
    if (!product_ok(rows, n_out, n_in) || rows == 0 || n_out == 0) return 0;
    const size_t one = shares_bytes(cut_of(rows, n_out, n_in, false), rows, n_out), other = shares_bytes(cut_of(rows, n_out, n_in, true), rows, n_out);
    return one > other ? one : other;
}

adatopk_status adatopk_fp8_product(const void *fp8_x, const void *fp8_w, int64_t rows, int64_t n_out, int64_t n_in, const void *bias, adatopk_dtype bias_dt,
                                   const void *add, int64_t add_stride, void *y, int64_t y_stride, adatopk_dtype dt, void *workspace, size_t workspace_bytes,
                                   void *hip_stream) {
    if (!dtype_ok(dt) || !(bias_dt == dt || bias_dt == ADATOPK_F32) || !product_ok(rows, n_out, n_in)) return ADATOPK_EINVAL;
    if (rows == 0 || n_out == 0) return ADATOPK_OK;
    if (!matrix_ok(y, y_stride, rows, n_out, dt) || !pointer_ok_or_null(bias, static_cast<size_t>(elem_size(bias_dt))) ||
        (add != nullptr && !matrix_ok(add, add_stride, rows, n_out, dt)) || (n_in > 0 && (!pointer_ok(fp8_x, 16) || !pointer_ok(fp8_w, 16))))
        return ADATOPK_EINVAL;
    const size_t need = adatopk_fp8_product_workspace_bytes(rows, n_out, n_in);
    if (need > 0 && !pointer_ok(workspace, 256)) return ADATOPK_EINVAL;
    if (workspace_bytes < need) return ADATOPK_EWORKSPACE;
    const Cut c = cut_of(rows, n_out, n_in, dt == ADATOPK_F32);
    const Product f{fp8_of(const_cast<void *>(fp8_x), rows, n_in), fp8_of(const_cast<void *>(fp8_w), n_out, n_in), rows, n_out, c.slices, c.split, c.per, c.tiles_out,
                    c.tiles_rows, bias, add, bias_dt != dt, add_stride, y_stride, y, static_cast<float *>(workspace)};
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    with_type(dt, [&](auto *null) {
        using T = std::remove_pointer_t<decltype(null)>;
        const auto join = [&](int split) {
            Product of = f;
            of.split = split;
            const int64_t per_row = (n_out + 7) / 8;
            const uint32_t octets = static_cast<uint32_t>(rows * per_row);
            hipLaunchKernelGGL(k_fp8_join<T>, dim3((octets + 255) / 256), dim3(256), 0, st, of, Divisor(static_cast<uint32_t>(per_row)), octets);
        };
        if (c.form == NONE) return join(0);
        if (c.form == FEW) {
            const dim3 groups(static_cast<unsigned>((n_out + 15) / 16)), threads(FEW_WAVES * 64);
            hipLaunchKernelGGL((rows <= 16 ? k_fp8_few<T, 1> : k_fp8_few<T, 2>), groups, threads, 0, st, f);
            return;
        }
        using Of = Tiles<sizeof(T) == 4 ? FP8_EXACT : FP8_FAST>;
        const dim3 groups(static_cast<unsigned>(c.tiles_out * c.tiles_rows * c.split));
        if (c.form == LARGE && c.whole < c.tiles_out * c.tiles_rows)
            hipLaunchKernelGGL((k_fp8_product_quartered<T, typename Of::Large, typename Of::Quarter>), dim3(static_cast<unsigned>(c.whole + 4 * (c.tiles_out * c.tiles_rows - c.whole))),
                               dim3(Of::Large::NT), 0, st, f, c.whole);
        else if (c.form == LARGE)
            hipLaunchKernelGGL((k_fp8_product<T, typename Of::Large, 1>), groups, dim3(Of::Large::NT), 0, st, f);
        else if (c.form == MIDDLE)
            hipLaunchKernelGGL((k_fp8_product<T, typename Of::Middle, 2>), groups, dim3(Of::Middle::NT), 0, st, f);
        else if (c.form == SMALL)
            hipLaunchKernelGGL((k_fp8_product<T, typename Of::Small, 4>), groups, dim3(Of::Small::NT), 0, st, f);
        else
            hipLaunchKernelGGL((k_fp8_product<T, typename Of::Deep, 1>), groups, dim3(Of::Deep::NT), 0, st, f);
        if (c.split > 1) join(c.split);
    });
    return launched();
}

#ifdef ADATOPK_MEASURE_BUILD
adatopk_status adatopk_measure_fp8_product_cut(int64_t rows, int64_t n_out, int64_t n_in, adatopk_dtype dt, int32_t *out) {
    if (!dtype_ok(dt) || !product_ok(rows, n_out, n_in) || rows == 0 || n_out == 0 || n_in == 0) return ADATOPK_EINVAL;
    const Cut c = cut_of(rows, n_out, n_in, dt == ADATOPK_F32);
    out[0] = c.form == FEW ? 0 : SIDE[c.form];
    out[1] = c.form == DEEP ? 1 : 0;
    out[2] = c.split;
    out[3] = c.form == LARGE && c.whole < c.tiles_out * c.tiles_rows ? 1 : 0;
    return ADATOPK_OK;
}
#endif

}  // extern "C"
