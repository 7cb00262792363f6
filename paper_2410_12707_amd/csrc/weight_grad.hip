// The gradient of a projection's weight and bias: dW[n][k] = sum over tokens r of dY[r][n] * X[r][k], db[n] = sum of dY[r][n], with X kept in 8 bits.
//
// A matrix product whose long axis is the slow one of both operands.  Tiles of dY and X go through LDS as bf16, [token][feature], and come out
// transposed (ds_read_b64_tr_b16), which is what the matrix instruction wants.  A number of the 8-bit form times its step, a power of two, is
// exact in bf16; dY is taken apart into as many bf16 pieces as its type needs (bf16 one, fp16 two, fp32 three: the leading 8 bits, the next 8, the
// rest), so every product is exact and the sums are 32-bit.
//
// With weight and bias of the layer norm whose normalised rows X holds, the projection's input was weight[k] * X + bias[k], so
// dW[n][k] = weight[k] * (dY^T X)[n][k] + db[n] * bias[k]: two operations per result instead of a rounding per element of X.
//
// Few tiles and many tokens: the tokens are split, partial products go to the workspace and k_weight_join adds them up in a fixed order.
#include <hip/hip_runtime.h>

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
constexpr int WM = 2, WN = 2, NT = WM * WN * 64;  // wavefronts along the tile's two sides

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
__device__ __forceinline__ uint32_t cut(float &lo, float &hi) {
    const uint32_t a = __float_as_uint(lo) & 0xFFFF0000u, b = __float_as_uint(hi) & 0xFFFF0000u;
    const bool inf_a = __builtin_fabsf(lo) == __builtin_inff(), inf_b = __builtin_fabsf(hi) == __builtin_inff();
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

// One tile of BM x BN results over one share of the tokens, four wavefronts, a quarter of the tile each.  Tiles of BK tokens go through two buffers in
// LDS: while the matrix instructions work on one, the next is converted into the other and the one behind it is on its way into registers.  One
// barrier per tile, and the last step's operands are in registers when it comes, so the matrix unit has work across it.
//
// The last tile of a row or column of tiles begins so far ahead that it ends with the matrix (it stores what is its own), so loads need no bounds but
// those of the tokens.  SMALL: the matrix is narrower than the tile, or its rows too far apart for 32-bit offsets; every load is bounded.
template <typename T, int BM, int BN, int BK, bool SMALL> __global__ __launch_bounds__(NT, 1) void k_weight_grad(Product f) {
    constexpr int P = pieces_of<T>(), MI = BM / WM / 32, NI = BN / WN / 32, STEPS = BK / 16;
    constexpr int A_PITCH = BM + PAD, B_PITCH = BN + PAD, A_SIZE = BK * A_PITCH, BUFFER = P * A_SIZE + BK * B_PITCH;
    constexpr int A_OCTETS = BK * BM / 8 / NT, B_ALL = BK * BN / 16, B_PIECES = (B_ALL + NT - 1) / NT;
    static_assert(BK * BM % (8 * NT) == 0 && MI >= 1 && NI >= 1, "whole octets");
    static_assert(NT % (BM / 8) == 0 && NT % 4 == 0, "an octet's column is the same in all of a thread's tokens");
    __shared__ __attribute__((aligned(16))) uint16_t lds[2 * BUFFER];
    __shared__ float sums[BM];
    const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64, wm = wave / WN, wn = wave % WN;
    const int b = place(blockIdx.x, gridDim.x);
    const int part = b / f.tiles, tile = b % f.tiles;
    const int64_t own_out = static_cast<int64_t>(tile / f.tiles_in) * BM, own_in = static_cast<int64_t>(tile % f.tiles_in) * BN;
    const int64_t out0 = SMALL || own_out + BM <= f.n_out ? own_out : f.n_out - BM, in0 = SMALL || own_in + BN <= f.x.pitch ? own_in : f.x.pitch - BN;
    const int64_t row0 = part * f.rows_per_split, row_end = row0 + f.rows_per_split < f.rows ? row0 + f.rows_per_split : f.rows;

    Raw<T> ra[A_OCTETS];
    U4 rb[B_PIECES];
    uint32_t re[B_PIECES];
    const uint32_t e_pitch = static_cast<uint32_t>(f.x.pitch / GROUP);
    uint32_t a_at[A_OCTETS], b_at[B_PIECES], e_at[B_PIECES];  // bytes from a tile's first element
#pragma unroll
    for (int i = 0; i < A_OCTETS; ++i) {
        const int at = tid + i * NT;
        a_at[i] = (static_cast<uint32_t>(at / (BM / 8)) * static_cast<uint32_t>(f.dy_stride) + at % (BM / 8) * 8) * sizeof(T);
    }
#pragma unroll
    for (int i = 0; i < B_PIECES; ++i) {
        const uint32_t at = B_ALL % NT != 0 && tid + i * NT >= B_ALL ? 0 : tid + i * NT;
        b_at[i] = at / (BN / 16) * static_cast<uint32_t>(f.x.pitch) + at % (BN / 16) * 16;
        e_at[i] = at / (BN / 16) * e_pitch + at % (BN / 16) / 2;
    }
    auto fetch = [&](int64_t row) {
        if (!SMALL && row + BK <= row_end) {
            const char *const a = reinterpret_cast<const char *>(static_cast<const T *>(f.dy) + row * f.dy_stride + out0);
            const char *const q = reinterpret_cast<const char *>(f.x.q + row * f.x.pitch + in0);
            const uint8_t *const e = f.x.e + row * e_pitch + in0 / GROUP;
#pragma unroll
            for (int i = 0; i < B_PIECES; ++i) {
                rb[i] = *reinterpret_cast<const U4 *>(q + b_at[i]);
                re[i] = e[e_at[i]];
            }
#pragma unroll
            for (int i = 0; i < A_OCTETS; ++i) ra[i] = load_octet(reinterpret_cast<const T *>(a + a_at[i]));
            return;
        }
#pragma unroll
        for (int i = 0; i < A_OCTETS; ++i) {
            const int at = tid + i * NT;
            const int64_t r = row + at / (BM / 8), c = out0 + at % (BM / 8) * 8;
            ra[i] = load_row(static_cast<const T *>(f.dy) + r * f.dy_stride + c, r < row_end ? f.n_out - c : 0);
        }
#pragma unroll
        for (int i = 0; i < B_PIECES; ++i) {
            const int at = tid + i * NT;
            const int64_t r = row + at / (BN / 16), c = in0 + at % (BN / 16) * 16;
            const bool there = r < row_end && c < f.x.pitch && (B_ALL % NT == 0 || at < B_ALL);
            rb[i] = there ? *reinterpret_cast<const U4 *>(f.x.q + r * f.x.pitch + c) : U4{0, 0, 0, 0};
            re[i] = there ? f.x.e[r * (f.x.pitch / GROUP) + c / GROUP] : 7;
        }
    };
    // Part `which` of `parts` of the tile in registers, into a buffer.
    auto stage = [&](uint16_t *to, int which, int parts) {
#pragma unroll
        for (int i = 0; i < A_OCTETS; ++i) {
            if (i % parts != which) continue;
            const int at = tid + i * NT, k = at / (BM / 8), m = at % (BM / 8) * 8;
            if constexpr (P == 1) {
                *reinterpret_cast<U4 *>(to + k * A_PITCH + m) = ra[i].w[0];
            } else {
                float v[8];
                unpack(ra[i], v);
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    U4 d;
#pragma unroll
                    for (int j = 0; j < 4; ++j) d[j] = cut(v[2 * j], v[2 * j + 1]);
                    *reinterpret_cast<U4 *>(to + p * A_SIZE + k * A_PITCH + m) = d;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < B_PIECES; ++i) {
            if (i % parts != which) continue;
            const int at = tid + i * NT, k = at / (BN / 16), n = at % (BN / 16) * 16;
            if (B_ALL % NT != 0 && at >= B_ALL) continue;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float v[8];
                values_of(U2{rb[i][2 * h], rb[i][2 * h + 1]}, re[i], v);
                *reinterpret_cast<U4 *>(to + P * A_SIZE + k * B_PITCH + n + 8 * h) = pack<Bf16>(v).w[0];
            }
        }
    };
    // What a lane holds of a 32 x 16 operand: feature lane % 32, tokens 8 * (lane / 32) and the seven behind it.  A transposing read works on blocks of
    // 16 lanes: lane i reads four features of token i / 4, and gets four tokens of feature i.
    const int token = 8 * (lane / 32) + lane % 16 / 4, feature = 16 * (lane / 16 % 2) + 4 * (lane % 4);
    const int a_lane = token * A_PITCH + wm * (BM / WM) + feature, b_lane = P * A_SIZE + token * B_PITCH + wn * (BN / WN) + feature;
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
            for (int i = 0; i < MI; ++i) xa[set][p][i] = operand(from + a_lane + p * A_SIZE + step * 16 * A_PITCH + i * 32, A_PITCH);
    };
    F16v acc[MI][NI] = {};
    // Sums of dY over the tokens.  Two wavefronts hold the same operands: of two blocks of 32 features the one sums the first, the other the second.
    constexpr int CI = (MI + 1) / 2;
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
                const U4 first = __builtin_bit_cast(U4, xa[set][p][2 * i]), second = __builtin_bit_cast(U4, xa[set][p][2 * i + 1 < MI ? 2 * i + 1 : 2 * i]);
                const Pair one = {static_cast<__bf16>(1.f), static_cast<__bf16>(1.f)};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t d = wn == 0 ? first[j] : second[j];
                    colsum[i] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(Pair, d), one, colsum[i], false);
                }
            }
        }
    };

    fetch(row0);
    stage(lds, 0, 1);
    fetch(row0 + BK);
    __syncthreads();
    take(lds, 0, 0);
    int cur = 0;
    for (int64_t row = row0; row < row_end; row += BK) {
        uint16_t *const now = lds + cur, *const next = lds + (BUFFER - cur);
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            if (s + 1 < STEPS) {
                take(now, s + 1, (s + 1) % 2);
                stage(next, s, STEPS - 1);
            } else {
                fetch(row + 2 * BK);
                __syncthreads();
                take(next, 0, (s + 1) % 2);
            }
            multiply(s % 2);
        }
        cur = BUFFER - cur;
    }
#pragma unroll
    for (int i = 0; i < CI; ++i) {
        const float t = colsum[i] + __shfl_xor(colsum[i], 32);
        if (lane < 32 && (wn == 0 || 2 * i + 1 < MI)) sums[wm * (BM / WM) + (2 * i + wn) * 32 + lane] = t;
    }
    __syncthreads();
    const bool last = f.split == 1;
    if (own_in == 0) {
        float *to = last ? f.db : f.partial_db + part * f.n_out;
        if (to != nullptr)
            for (int i = tid; i < BM && out0 + i < f.n_out; i += NT)
                if (out0 + i >= own_out) to[out0 + i] = sums[i] + (last && f.accumulate != 0 ? to[out0 + i] : 0.f);
    }
    float *to = last ? f.dw : f.partial + part * f.n_out * f.n_in;
#pragma unroll
    for (int j = 0; j < NI; ++j) {
        const int64_t c = in0 + wn * (BN / WN) + j * 32 + lane % 32;
        if (c >= f.n_in || c < own_in) continue;
        const float w = last ? weight_at(f.weight, f.wide_weight || sizeof(T) == 4, __is_same(T, F16), c, 1.f) : 1.f;
        const float v = last ? weight_at(f.bias, f.wide_weight || sizeof(T) == 4, __is_same(T, F16), c, 0.f) : 0.f;
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int q = 0; q < 16; ++q) {
                const int m = wm * (BM / WM) + i * 32 + 8 * (q / 4) + 4 * (lane / 32) + q % 4;
                if (out0 + m >= f.n_out || out0 + m < own_out) continue;
                float *at = to + (out0 + m) * f.n_in + c;
                float t = acc[i][j][q];
                if (last) {
                    if (f.weight != nullptr) t *= w;
                    if (f.bias != nullptr) t = __builtin_fmaf(sums[m], v, t);
                    if (f.accumulate != 0) t += *at;
                }
                *at = t;
            }
    }
}

// The partial products added up, weight and bias applied.
__global__ __launch_bounds__(256) void k_weight_join(Product f, int dt_is_f16, int wide) {
    const unsigned blocks = static_cast<unsigned>((f.n_in + 255) / 256);  // of a row
    const int64_t n = blockIdx.x / blocks, k = static_cast<int64_t>(blockIdx.x % blocks) * 256 + threadIdx.x;
    float bias_sum = 0.f;
    for (int s = 0; s < f.split; ++s) bias_sum += f.partial_db[s * f.n_out + n];
    if (k == 0 && f.db != nullptr) f.db[n] = bias_sum + (f.accumulate != 0 ? f.db[n] : 0.f);
    if (k >= f.n_in) return;
    float t = 0.f;
    for (int s = 0; s < f.split; ++s) t += f.partial[(s * f.n_out + n) * f.n_in + k];
    if (f.weight != nullptr) t *= weight_at(f.weight, wide != 0, dt_is_f16, k, 1.f);
    if (f.bias != nullptr) t = __builtin_fmaf(bias_sum, weight_at(f.bias, wide != 0, dt_is_f16, k, 0.f), t);
    float *at = f.dw + n * f.n_in + k;
    *at = t + (f.accumulate != 0 ? *at : 0.f);
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
Cut cut_of(int64_t rows, int64_t n_out, int64_t n_in, bool far) {
    Cut best{};
    double least = 0;
    const int64_t steps = rows > 0 ? (rows + SHARE - 1) / SHARE : 1;
    for (int t = 0; t < TILES; ++t) {
        const bool fits = n_out >= TILE_BM[t] && adatopk_internal::act8_pitch(n_in) >= TILE_BN[t] && !far;
        if (t != TILE_SMALL && !fits) continue;
        if (t == TILE_SMALL && best.split != 0) continue;
        const int64_t in = (n_in + TILE_BN[t] - 1) / TILE_BN[t], tiles = in * ((n_out + TILE_BM[t] - 1) / TILE_BM[t]);
        for (int64_t split = 1; split <= 16 && split <= steps; ++split) {
            const int64_t per = (steps + split - 1) / split;
            if ((steps + per - 1) / per != split) continue;
            const int per_unit = t >= TILE_64_64 ? 4 : t == TILE_128_128 ? 2 : 1;
            const double area = static_cast<double>(TILE_BM[t]) * TILE_BN[t] / 65536.;
            const double rounds = static_cast<double>((tiles * split + 256 * per_unit - 1) / (256 * per_unit));
            const double step = (0.4 + 0.9 * area * per_unit) * per;
            const double join = split == 1 ? 0 : 4.0 + static_cast<double>(split) * n_out * n_in * 8 / 4e6;
            const double cost = rounds * (step + 4.0) + join;
            if (least == 0 || cost < least) {
                least = cost;
                best = Cut{static_cast<Tile>(t), static_cast<int>(in), static_cast<int>(tiles), static_cast<int>(split), per * SHARE};
            }
        }
    }
    return best;
}

constexpr int64_t MAX_FEATURES = 1 << 17;  // of either side: tiles, and rows of them, are counted in 32 bits

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
        const Cut c = cut_of(rows, n_out, n_in, far);
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
    const Cut c = cut_of(rows, n_out, n_in, rows > 1 && dy_stride >= MAX_STRIDE);
    float *partial = static_cast<float *>(workspace);
    const bool wide = weight_dt == ADATOPK_F32;
    const Product f{dy,     dy_stride, act8_of(const_cast<void *>(act8_x), rows, n_in), rows, n_out, n_in, c.rows_per_split, c.tiles_in, c.tiles, c.split,
                    weight, bias,      wide, dw, db, accumulate, partial, partial + static_cast<int64_t>(c.split) * n_out * n_in};
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    with_type(dt, [&](auto *null) {
        using T = std::remove_pointer_t<decltype(null)>;
        constexpr int DEEP = pieces_of<T>() == 1 ? 64 : 32;  // tokens of a tile: what two buffers have room for
        const auto kernel = c.tile == TILE_256_256   ? k_weight_grad<T, 256, 256, DEEP, false>
                            : c.tile == TILE_256_192 ? k_weight_grad<T, 256, 192, DEEP, false>
                            : c.tile == TILE_256_128 ? k_weight_grad<T, 256, 128, DEEP, false>
                            : c.tile == TILE_128_128 ? k_weight_grad<T, 128, 128, DEEP, false>
                            : c.tile == TILE_64_64   ? k_weight_grad<T, 64, 64, DEEP, false>
                                                     : k_weight_grad<T, 64, 64, DEEP, true>;
        hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(c.tiles * c.split)), dim3(NT), 0, st, f);
    });
    if (c.split > 1)
        hipLaunchKernelGGL(k_weight_join, dim3(static_cast<unsigned>((n_in + 255) / 256 * n_out)), dim3(256), 0, st, f,
                           weight_dt == ADATOPK_F16 ? 1 : 0, wide ? 1 : 0);
    return launched();
}

}  // extern "C"
