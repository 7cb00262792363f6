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

constexpr int PAD = 32;  // elements behind a row of a tile in LDS: the four rows that one transposing read takes lie in different banks
constexpr int BM = 128, BN = 128, BK = 32;
constexpr int WM = 2, WN = 2, NT = WM * WN * 64;
constexpr int MI = BM / WM / 32, NI = BN / WN / 32;

struct Product {
    const void *dy;
    int64_t dy_stride;
    Act8 x;
    int64_t rows, n_out, n_in;
    int64_t rows_per_split;
    int tiles_out, tiles_in, split;
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

template <typename T> __global__ __launch_bounds__(NT) void k_weight_grad(Product f) {
    constexpr int P = pieces_of<T>();
    constexpr int A_OCTETS = BK * BM / 8 / NT, B_PIECES = BK * BN / 16 / NT;
    __shared__ __attribute__((aligned(16))) uint16_t sa[P][BK][BM + PAD], sb[BK][BN + PAD];
    __shared__ float sums[BM];
    const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64, wm = wave / WN, wn = wave % WN;
    int b = blockIdx.x;
    const int tile_in = b % f.tiles_in;
    b /= f.tiles_in;
    const int tile_out = b % f.tiles_out, part = b / f.tiles_out;
    const int64_t out0 = static_cast<int64_t>(tile_out) * BM, in0 = static_cast<int64_t>(tile_in) * BN;
    const int64_t row0 = part * f.rows_per_split, row_end = row0 + f.rows_per_split < f.rows ? row0 + f.rows_per_split : f.rows;

    Raw<T> ra[A_OCTETS];
    U4 rb[B_PIECES];
    uint32_t re[B_PIECES];
    auto fetch = [&](int64_t row) {
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
            const bool there = r < row_end && c < f.x.pitch;
            rb[i] = there ? *reinterpret_cast<const U4 *>(f.x.q + r * f.x.pitch + c) : U4{0, 0, 0, 0};
            re[i] = there ? f.x.e[r * (f.x.pitch / GROUP) + c / GROUP] : 7;
        }
    };
    auto stage = [&]() {
#pragma unroll
        for (int i = 0; i < A_OCTETS; ++i) {
            const int at = tid + i * NT, k = at / (BM / 8), m = at % (BM / 8) * 8;
            if constexpr (P == 1) {
                *reinterpret_cast<U4 *>(&sa[0][k][m]) = ra[i].w[0];
            } else {
                float v[8];
                unpack(ra[i], v);
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    U4 d;
#pragma unroll
                    for (int j = 0; j < 4; ++j) d[j] = cut(v[2 * j], v[2 * j + 1]);
                    *reinterpret_cast<U4 *>(&sa[p][k][m]) = d;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < B_PIECES; ++i) {
            const int at = tid + i * NT, k = at / (BN / 16), n = at % (BN / 16) * 16;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float v[8];
                values_of(U2{rb[i][2 * h], rb[i][2 * h + 1]}, re[i], v);
                *reinterpret_cast<U4 *>(&sb[k][n + 8 * h]) = pack<Bf16>(v).w[0];
            }
        }
    };
    // What a lane holds of a 32 x 16 operand: feature lane % 32, tokens 8 * (lane / 32) and the seven behind it.  A transposing read works on blocks of
    // 16 lanes: lane i reads four features of token i / 4, and gets four tokens of feature i.
    const int token = 8 * (lane / 32) + lane % 16 / 4, feature = 16 * (lane / 16 % 2) + 4 * (lane % 4);
    auto operand = [&](const uint16_t *tile, int pitch) {
        typedef __attribute__((address_space(3))) S4 Lds;
        const S4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds *)(tile + token * pitch + feature));
        const S4 c = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds *)(tile + (token + 4) * pitch + feature));
        const B4 x = __builtin_bit_cast(B4, a), y = __builtin_bit_cast(B4, c);
        return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
    };

    F16v acc[MI][NI] = {};
    float colsum[MI] = {};
    fetch(row0);
    for (int64_t row = row0; row < row_end; row += BK) {
        __syncthreads();  // the tile before has been read
        stage();
        __syncthreads();
        if (row + BK < row_end) fetch(row + BK);
#pragma unroll
        for (int k = 0; k < BK; k += 16) {
            B8 x[NI];
#pragma unroll
            for (int j = 0; j < NI; ++j) x[j] = operand(&sb[k][wn * (BN / WN) + j * 32], BN + PAD);
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int i = 0; i < MI; ++i) {
                    const B8 a = operand(&sa[p][k][wm * (BM / WM) + i * 32], BM + PAD);
#pragma unroll
                    for (int j = 0; j < NI; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, x[j], acc[i][j], 0, 0, 0);
                    if (i % WN == wn) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) colsum[i] += static_cast<float>(a[j]);
                    }
                }
        }
    }
#pragma unroll
    for (int i = 0; i < MI; ++i) {
        if (i % WN == wn) {
            const float t = colsum[i] + __shfl_xor(colsum[i], 32);
            if (lane < 32) sums[wm * (BM / WM) + i * 32 + lane] = t;
        }
    }
    __syncthreads();
    const bool last = f.split == 1;
    if (tile_in == 0) {
        float *to = last ? f.db : f.partial_db + part * f.n_out;
        if (to != nullptr)
            for (int i = tid; i < BM && out0 + i < f.n_out; i += NT) to[out0 + i] = sums[i] + (last && f.accumulate != 0 ? to[out0 + i] : 0.f);
    }
    float *to = last ? f.dw : f.partial + part * f.n_out * f.n_in;
#pragma unroll
    for (int j = 0; j < NI; ++j) {
        const int64_t c = in0 + wn * (BN / WN) + j * 32 + lane % 32;
        if (c >= f.n_in) continue;
        const float w = last ? weight_at(f.weight, f.wide_weight || sizeof(T) == 4, __is_same(T, F16), c, 1.f) : 1.f;
        const float v = last ? weight_at(f.bias, f.wide_weight || sizeof(T) == 4, __is_same(T, F16), c, 0.f) : 0.f;
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int q = 0; q < 16; ++q) {
                const int m = wm * (BM / WM) + i * 32 + 8 * (q / 4) + 4 * (lane / 32) + q % 4;
                if (out0 + m >= f.n_out) continue;
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

struct Cut {
    int tiles_out, tiles_in, split;
    int64_t rows_per_split;
};
Cut cut_of(int64_t rows, int64_t n_out, int64_t n_in) {
    Cut c;
    c.tiles_out = static_cast<int>((n_out + BM - 1) / BM);
    c.tiles_in = static_cast<int>((n_in + BN - 1) / BN);
    const int64_t tiles = static_cast<int64_t>(c.tiles_out) * c.tiles_in, steps = (rows + BK - 1) / BK;
    int64_t split = (512 + tiles - 1) / tiles;
    if (split > steps / 4) split = steps / 4;
    if (split < 1) split = 1;
    const int64_t per = (steps + split - 1) / split;
    c.split = steps == 0 ? 1 : static_cast<int>((steps + per - 1) / per);
    c.rows_per_split = per * BK;
    return c;
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
    const Cut c = cut_of(rows, n_out, n_in);
    return c.split == 1 ? 256 : align_up(static_cast<size_t>(c.split) * static_cast<size_t>(n_out) * (static_cast<size_t>(n_in) + 1) * sizeof(float), 256);
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
    const Cut c = cut_of(rows, n_out, n_in);
    float *partial = static_cast<float *>(workspace);
    const bool wide = weight_dt == ADATOPK_F32;
    const Product f{dy,     dy_stride, act8_of(const_cast<void *>(act8_x), rows, n_in), rows, n_out, n_in, c.rows_per_split, c.tiles_out, c.tiles_in, c.split,
                    weight, bias,      wide, dw, db, accumulate, partial, partial + static_cast<int64_t>(c.split) * n_out * n_in};
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    with_type(dt, [&](auto *null) {
        using T = std::remove_pointer_t<decltype(null)>;
        hipLaunchKernelGGL(k_weight_grad<T>, dim3(static_cast<unsigned>(c.tiles_out * c.tiles_in * c.split)), dim3(NT), 0, st, f);
    });
    if (c.split > 1)
        hipLaunchKernelGGL(k_weight_join, dim3(static_cast<unsigned>((n_in + 255) / 256 * n_out)), dim3(256), 0, st, f,
                           weight_dt == ADATOPK_F16 ? 1 : 0, wide ? 1 : 0);
    return launched();
}

}  // extern "C"
