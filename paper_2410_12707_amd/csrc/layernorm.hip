// Layer norm over the rows of a matrix, forward and backward, with the residual addition before it and the normalised rows kept in 8 bits.
//
//   forward   s = x + residual, rounded to the type (the next block reads it);  mean = sum s / n;  rstd = 1 / sqrt(sum (s - mean)^2 / n + eps);
//             h = (s - mean) * rstd;  y = weight * h + bias
//   backward  g = dy * weight;  dx = rstd * (g - sum g / n - h * (sum g h) / n) + dsum;  dweight = sum over rows dy * h;  dbias = sum over rows dy
//             with h from the kept 8-bit rows, or from x, mean and rstd
//
// A row is read once and held in registers between the sums and their use: W wavefronts share it, an octet per lane and slot.  All sums are
// in 32 bits and in a fixed order.
#include <hip/hip_runtime.h>

#include "stage_ops.h"

namespace {

using namespace adatopk_stage;

constexpr int SLOTS = 4;                   // octets per lane at most: 2048 elements per wavefront
constexpr int WIDE_WAVES = 16;             // wavefronts of a row at most
constexpr int64_t MAX_COLS = static_cast<int64_t>(SLOTS) * 512 * WIDE_WAVES;  // 32768
constexpr int ROWS_PER_GROUP = 4;          // rows of a workgroup of one-wavefront rows
constexpr int PARTS = 256;                 // workgroups that leave partial sums of the weight's gradient, at most

// Sum over the W wavefronts of a row, in every lane.  `scratch`: W floats per value in LDS.
template <int W, int N> __device__ __forceinline__ void row_sum(float (&v)[N], float *scratch) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = wave_sum(v[i]);
    if constexpr (W > 1) {
        const int wave = threadIdx.x / 64;
        __syncthreads();  // the scratch of the sum before has been read
        if (threadIdx.x % 64 == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) scratch[i * W + wave] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float t = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) t += scratch[i * W + w];
            v[i] = t;
        }
    }
}

struct Forward {
    const void *x, *residual, *weight, *bias;
    void *sum, *y;
    float *mean, *rstd;
    int64_t x_stride, residual_stride, sum_stride, y_stride;
    int64_t rows, cols;
    float eps;
    bool wide_weight;  // weight and bias in fp32 beside 16-bit rows
    Act8 act8;
};

template <typename T> __device__ __forceinline__ void load_weight(const void *p, bool wide, int64_t at, int64_t left, float absent, float (&v)[8]) {
    if (p == nullptr) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = absent;
    } else if (wide) {
        unpack(load_row(static_cast<const float *>(p) + at, left), v);
    } else {
        unpack(load_row(static_cast<const T *>(p) + at, left), v);
    }
}

// One row per W wavefronts (W > 1: per workgroup).
template <typename T, int W, int S> __global__ __launch_bounds__(W > 1 ? W * 64 : ROWS_PER_GROUP * 64) void k_layernorm_forward(Forward f) {
    __shared__ float scratch[2 * W];
    const int lane = threadIdx.x % (W * 64);
    const int64_t row = W > 1 ? blockIdx.x : static_cast<int64_t>(blockIdx.x) * ROWS_PER_GROUP + threadIdx.x / 64;
    if (row >= f.rows) return;  // (a whole wavefront, or W == 1)
    const float inverse = 1.f / static_cast<float>(f.cols);
    float v[S][8];
    float sums[1] = {0.f};
#pragma unroll
    for (int s = 0; s < S; ++s) {
        const int64_t at = (static_cast<int64_t>(s) * W * 64 + lane) * 8, left = f.cols - at;
        unpack(load_row(static_cast<const T *>(f.x) + row * f.x_stride + at, left), v[s]);
        if (f.residual != nullptr) {
            float r[8];
            unpack(load_row(static_cast<const T *>(f.residual) + row * f.residual_stride + at, left), r);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[s][j] += r[j];
            const Raw<T> out = pack<T>(v[s]);
            if (f.sum != nullptr) store_row(static_cast<T *>(f.sum) + row * f.sum_stride + at, left, out);
            unpack(out, v[s]);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) sums[0] += v[s][j];
    }
    row_sum<W>(sums, scratch);
    const float mean = sums[0] * inverse;
    sums[0] = 0.f;
#pragma unroll
    for (int s = 0; s < S; ++s) {
        const int64_t at = (static_cast<int64_t>(s) * W * 64 + lane) * 8;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[s][j] = at + j < f.cols ? v[s][j] - mean : 0.f;
            sums[0] = __builtin_fmaf(v[s][j], v[s][j], sums[0]);
        }
    }
    row_sum<W>(sums, scratch);
    const float rstd = 1.f / __fsqrt_rn(sums[0] * inverse + f.eps);
    if (lane == 0) {
        if (f.mean != nullptr) f.mean[row] = mean;
        if (f.rstd != nullptr) f.rstd[row] = rstd;
    }
#pragma unroll
    for (int s = 0; s < S; ++s) {
        const int64_t at = (static_cast<int64_t>(s) * W * 64 + lane) * 8, left = f.cols - at;
        float w[8], b[8];
        load_weight<T>(f.weight, f.wide_weight, at, left, 1.f, w);
        load_weight<T>(f.bias, f.wide_weight, at, left, 0.f, b);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[s][j] *= rstd;
            b[j] = __builtin_fmaf(v[s][j], w[j], b[j]);
        }
        store_row(static_cast<T *>(f.y) + row * f.y_stride + at, left, pack<T>(b));
        if (f.act8.q != nullptr) act8_put(f.act8, row, static_cast<int>(at / 8), v[s]);
    }
}

struct Backward {
    const void *dy, *x, *weight, *dsum;
    const float *mean, *rstd;
    void *dx;
    float *partial;  // [parts][2][cols]: sums of dy * h and of dy over the rows of a workgroup
    int64_t dy_stride, x_stride, dsum_stride, dx_stride;
    int64_t rows, cols;
    bool wide_weight;
    Act8 act8;
};

// A workgroup takes rows blockIdx.x, blockIdx.x + gridDim.x, ... (W == 1: four at a time) and keeps its share of the weight's gradient in registers.
template <typename T, int W, int S> __global__ __launch_bounds__(W > 1 ? W * 64 : ROWS_PER_GROUP * 64) void k_layernorm_backward(Backward f) {
    __shared__ float scratch[2 * W];
    const int lane = threadIdx.x % (W * 64);
    const int64_t first = W > 1 ? blockIdx.x : static_cast<int64_t>(blockIdx.x) * ROWS_PER_GROUP + threadIdx.x / 64;
    const int64_t step = W > 1 ? gridDim.x : static_cast<int64_t>(gridDim.x) * ROWS_PER_GROUP;
    const float inverse = 1.f / static_cast<float>(f.cols);
    float dw[S][8] = {}, db[S][8] = {};
    for (int64_t row = first; row < f.rows; row += step) {
        float g[S][8], h[S][8];
        float sums[2] = {0.f, 0.f};
        const float rstd = f.rstd[row], mean = f.x != nullptr ? f.mean[row] : 0.f;
#pragma unroll
        for (int s = 0; s < S; ++s) {
            const int64_t at = (static_cast<int64_t>(s) * W * 64 + lane) * 8, left = f.cols - at;
            unpack(load_row(static_cast<const T *>(f.dy) + row * f.dy_stride + at, left), g[s]);
            if (f.x != nullptr) {
                unpack(load_row(static_cast<const T *>(f.x) + row * f.x_stride + at, left), h[s]);
#pragma unroll
                for (int j = 0; j < 8; ++j) h[s][j] = j < left ? (h[s][j] - mean) * rstd : 0.f;
            } else {
                U2 d;
                uint32_t E;
                act8_get(f.act8, row, static_cast<int>(at / 8), d, E);
                values_of(d, E, h[s]);
#pragma unroll
                for (int j = 0; j < 8; ++j) h[s][j] = j < left ? h[s][j] : 0.f;
            }
            float w[8];
            load_weight<T>(f.weight, f.wide_weight, at, left, 1.f, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                dw[s][j] = __builtin_fmaf(g[s][j], h[s][j], dw[s][j]);
                db[s][j] += g[s][j];
                g[s][j] *= w[j];
                sums[0] += g[s][j];
                sums[1] = __builtin_fmaf(g[s][j], h[s][j], sums[1]);
            }
        }
        row_sum<W>(sums, scratch);
        const float level = sums[0] * inverse, along = sums[1] * inverse;
#pragma unroll
        for (int s = 0; s < S; ++s) {
            const int64_t at = (static_cast<int64_t>(s) * W * 64 + lane) * 8, left = f.cols - at;
            float add[8] = {};
            if (f.dsum != nullptr) unpack(load_row(static_cast<const T *>(f.dsum) + row * f.dsum_stride + at, left), add);
#pragma unroll
            for (int j = 0; j < 8; ++j) add[j] += rstd * (g[s][j] - level - h[s][j] * along);
            store_row(static_cast<T *>(f.dx) + row * f.dx_stride + at, left, pack<T>(add));
        }
    }
    if (f.partial == nullptr) return;
    if constexpr (W == 1) {  // the four rows' shares, in a fixed order
        __shared__ float share[ROWS_PER_GROUP][512 + 8];
        const int wave = threadIdx.x / 64;
        for (int which = 0; which < 2; ++which)
#pragma unroll
            for (int s = 0; s < S; ++s) {
                __syncthreads();
#pragma unroll
                for (int j = 0; j < 8; ++j) share[wave][j * 64 + lane] = which == 0 ? dw[s][j] : db[s][j];
                __syncthreads();
                for (int i = threadIdx.x; i < 512; i += ROWS_PER_GROUP * 64) {
                    const int64_t col = static_cast<int64_t>(s) * 512 + (i % 64) * 8 + i / 64;
                    float t = 0.f;
#pragma unroll
                    for (int w = 0; w < ROWS_PER_GROUP; ++w) t += share[w][i];
                    if (col < f.cols) f.partial[(blockIdx.x * static_cast<int64_t>(2) + which) * f.cols + col] = t;
                }
            }
    } else {
#pragma unroll
        for (int s = 0; s < S; ++s) {
            const int64_t at = (static_cast<int64_t>(s) * W * 64 + lane) * 8, left = f.cols - at;
            float *to = f.partial + blockIdx.x * static_cast<int64_t>(2) * f.cols + at;
            if (left > 0) {
                store_row(to, left, pack<float>(dw[s]));
                store_row(to + f.cols, left, pack<float>(db[s]));
            }
        }
    }
}

// Columns of the partial sums added up, in a fixed order: 64 columns per workgroup, 16 lanes of parts for each.
__global__ __launch_bounds__(1024) void k_layernorm_join(const float *partial, int parts, int64_t cols, float *dweight, float *dbias, int accumulate) {
    __shared__ float share[16][64];
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 64 + threadIdx.x % 64;  // column of the [2][cols] sums
    const int lane = threadIdx.x / 64;
    float t = 0.f;
    if (i < 2 * cols)
        for (int p = lane; p < parts; p += 16) t += partial[static_cast<int64_t>(p) * 2 * cols + i];
    share[lane][threadIdx.x % 64] = t;
    __syncthreads();
    if (lane != 0 || i >= 2 * cols) return;
    t = 0.f;
#pragma unroll
    for (int k = 0; k < 16; ++k) t += share[k][threadIdx.x];
    float *to = i < cols ? dweight : dbias;
    if (to == nullptr) return;
    to += i < cols ? i : i - cols;
    *to = accumulate != 0 ? *to + t : t;
}

// The smallest of the shapes that hold a row: f is called with W and S as types.
template <int N> using Int = std::integral_constant<int, N>;
template <typename F> void with_shape(int64_t cols, F &&f) {
    if (cols <= 512)
        f(Int<1>(), Int<1>());
    else if (cols <= 1024)
        f(Int<1>(), Int<2>());
    else if (cols <= 2048)
        f(Int<1>(), Int<4>());
    else if (cols <= 4096)
        f(Int<4>(), Int<2>());
    else if (cols <= 8192)
        f(Int<4>(), Int<4>());
    else if (cols <= 16384)
        f(Int<16>(), Int<2>());
    else
        f(Int<16>(), Int<4>());
}

bool wave_rows(int64_t cols) { return cols <= 2048; }
// Workgroups of the backward pass, which is also how many partial sums there are.
int64_t parts_of(int64_t rows, int64_t cols) {
    const int64_t groups = wave_rows(cols) ? (rows + ROWS_PER_GROUP - 1) / ROWS_PER_GROUP : rows;
    return groups < PARTS * 2 ? groups : PARTS * 2;
}

bool weights_ok(const void *p, adatopk_dtype wdt) { return pointer_ok_or_null(p, static_cast<size_t>(elem_size(wdt))); }

}  // namespace

extern "C" {

adatopk_status adatopk_layernorm_forward(const void *x, int64_t x_stride, const void *residual, int64_t residual_stride, const void *weight,
                                         const void *bias, adatopk_dtype weight_dt, int64_t rows, int64_t cols, adatopk_dtype dt, float eps, void *sum,
                                         int64_t sum_stride, void *y, int64_t y_stride, float *mean, float *rstd, void *act8, void *hip_stream) {
    if (!dtype_ok(dt) || !(weight_dt == dt || weight_dt == ADATOPK_F32) || !shape_ok(rows, cols) || cols > MAX_COLS || !(eps >= 0.f)) return ADATOPK_EINVAL;
    if (rows == 0 || cols == 0) return ADATOPK_OK;
    if (!matrix_ok(x, x_stride, rows, cols, dt) || !matrix_ok(y, y_stride, rows, cols, dt) || !weights_ok(weight, weight_dt) || !weights_ok(bias, weight_dt) ||
        (residual != nullptr && !matrix_ok(residual, residual_stride, rows, cols, dt)) || (sum != nullptr && residual == nullptr) ||
        (sum != nullptr && !matrix_ok(sum, sum_stride, rows, cols, dt)) || !pointer_ok_or_null(mean, 4) || !pointer_ok_or_null(rstd, 4) ||
        !pointer_ok_or_null(act8, 16))
        return ADATOPK_EINVAL;
    const Forward f{x,        residual,        weight,     bias,     sum,  y,    mean, rstd,
                    x_stride, residual_stride, sum_stride, y_stride, rows, cols, eps,  weight_dt != dt, act8_of(act8, rows, cols)};
    const int64_t groups = wave_rows(cols) ? (rows + ROWS_PER_GROUP - 1) / ROWS_PER_GROUP : rows;
    with_type(dt, [&](auto *null) {
        using T = std::remove_pointer_t<decltype(null)>;
        with_shape(cols, [&](auto waves, auto slots) {
            constexpr int W = decltype(waves)::value, S = decltype(slots)::value;
            hipLaunchKernelGGL((k_layernorm_forward<T, W, S>), dim3(static_cast<unsigned>(groups)), dim3(W > 1 ? W * 64 : ROWS_PER_GROUP * 64), 0,
                               static_cast<hipStream_t>(hip_stream), f);
        });
    });
    return launched();
}

size_t adatopk_layernorm_backward_workspace_bytes(int64_t rows, int64_t cols) {
    if (!shape_ok(rows, cols) || cols > MAX_COLS) return 0;
    return align_up(static_cast<size_t>(parts_of(rows, cols)) * 2 * static_cast<size_t>(cols) * sizeof(float), 256);
}

adatopk_status adatopk_layernorm_backward(const void *dy, int64_t dy_stride, const void *x, int64_t x_stride, const void *act8, const float *mean,
                                          const float *rstd, const void *weight, adatopk_dtype weight_dt, const void *dsum, int64_t dsum_stride,
                                          int64_t rows, int64_t cols, adatopk_dtype dt, void *dx, int64_t dx_stride, float *dweight, float *dbias,
                                          int32_t accumulate, void *workspace, size_t workspace_bytes, void *hip_stream) {
    if (!dtype_ok(dt) || !(weight_dt == dt || weight_dt == ADATOPK_F32) || !shape_ok(rows, cols) || cols > MAX_COLS) return ADATOPK_EINVAL;
    const bool weights = dweight != nullptr || dbias != nullptr;
    if (cols == 0) return ADATOPK_OK;
    if (!pointer_ok_or_null(dweight, 4) || !pointer_ok_or_null(dbias, 4)) return ADATOPK_EINVAL;
    if (rows > 0 && (!matrix_ok(dy, dy_stride, rows, cols, dt) || !matrix_ok(dx, dx_stride, rows, cols, dt) || (x == nullptr) == (act8 == nullptr) ||
                     (x != nullptr && (!matrix_ok(x, x_stride, rows, cols, dt) || !pointer_ok(mean, 4))) || !pointer_ok_or_null(act8, 16) ||
                     !pointer_ok(rstd, 4) || !weights_ok(weight, weight_dt) || (dsum != nullptr && !matrix_ok(dsum, dsum_stride, rows, cols, dt)) ||
                     (weights && !pointer_ok(workspace, 256))))
        return ADATOPK_EINVAL;
    if (weights && rows > 0 && workspace_bytes < adatopk_layernorm_backward_workspace_bytes(rows, cols)) return ADATOPK_EWORKSPACE;
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const int64_t parts = parts_of(rows, cols);
    float *partial = weights ? static_cast<float *>(workspace) : nullptr;
    if (rows > 0) {
        const Backward f{dy,        x,        weight,      dsum,      mean, rstd, dx,
                         partial,   dy_stride, x_stride,   dsum_stride, dx_stride, rows, cols, weight_dt != dt, act8_of(const_cast<void *>(act8), rows, cols)};
        with_type(dt, [&](auto *null) {
            using T = std::remove_pointer_t<decltype(null)>;
            with_shape(cols, [&](auto waves, auto slots) {
                constexpr int W = decltype(waves)::value, S = decltype(slots)::value;
                hipLaunchKernelGGL((k_layernorm_backward<T, W, S>), dim3(static_cast<unsigned>(parts)), dim3(W > 1 ? W * 64 : ROWS_PER_GROUP * 64), 0, st, f);
            });
        });
    }
    if (weights)  // (no rows: the sums are zero)
        hipLaunchKernelGGL(k_layernorm_join, dim3(static_cast<unsigned>((2 * cols + 63) / 64)), dim3(1024), 0, st, partial, static_cast<int>(parts), cols,
                           dweight, dbias, accumulate);
    return launched();
}

}  // extern "C"
