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

constexpr int64_t MAX_COLS = 32768;        // 16 wavefronts with four octets per lane
constexpr int COMPUTE_UNITS = 256;
constexpr int WAVES = 8;                   // wavefronts of a workgroup, at most, where a row takes eight or fewer

// Threads of the largest workgroup, and rows that one works on at a time: a team of W wavefronts to a row.
template <int W> constexpr int threads_of() { return (W > WAVES ? W : WAVES) * 64; }
template <int W> constexpr int teams_of() { return W > WAVES ? 1 : WAVES / W; }

// Sum over the W wavefronts of a row, in every lane.  `scratch`: W floats per value in LDS, the team's own.  Every wavefront of the workgroup calls it.
template <int W, int N> __device__ __forceinline__ void row_sum(float (&v)[N], float *scratch) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = wave_sum(v[i]);
    if constexpr (W > 1) {
        const int wave = threadIdx.x / 64 % W;
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

// A workgroup's teams of W wavefronts take a row each, and rows come round in steps of the grid: weight and bias stay in registers, and the next row is on
// its way while this one is summed up.
template <typename T, int W, int S> __global__ __launch_bounds__(threads_of<W>()) void k_layernorm_forward(Forward f) {
    __shared__ float scratch[teams_of<W>()][W];
    const int lane = threadIdx.x % (W * 64), team = threadIdx.x / (W * 64);
    const int64_t teams = blockDim.x / (W * 64), step = gridDim.x * teams;
    const float inverse = 1.f / static_cast<float>(f.cols);
    int64_t row = blockIdx.x * teams + team;
    Raw<T> x[S], r[S];
    auto fetch = [&](int64_t of) {
#pragma unroll
        for (int s = 0; s < S; ++s) {
            const int64_t at = (static_cast<int64_t>(s) * W * 64 + lane) * 8, left = of < f.rows ? f.cols - at : 0;
            x[s] = load_row(static_cast<const T *>(f.x) + of * f.x_stride + at, left);
            if (f.residual != nullptr) r[s] = load_row(static_cast<const T *>(f.residual) + of * f.residual_stride + at, left);
        }
    };
    fetch(row);
    float w[S][8], b[S][8];
#pragma unroll
    for (int s = 0; s < S; ++s) {
        const int64_t at = (static_cast<int64_t>(s) * W * 64 + lane) * 8, left = f.cols - at;
        load_weight<T>(f.weight, f.wide_weight, at, left, 1.f, w[s]);
        load_weight<T>(f.bias, f.wide_weight, at, left, 0.f, b[s]);
    }
    for (; row - team < f.rows; row += step) {  // (the workgroup's teams go round together, one without a row along with the others)
        const bool there = row < f.rows;
        float v[S][8];
        float sums[1] = {0.f};
#pragma unroll
        for (int s = 0; s < S; ++s) {
            const int64_t at = (static_cast<int64_t>(s) * W * 64 + lane) * 8, left = there ? f.cols - at : 0;
            unpack(x[s], v[s]);
            if (f.residual != nullptr) {
                float t[8];
                unpack(r[s], t);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[s][j] += t[j];
                const Raw<T> out = pack<T>(v[s]);
                if (f.sum != nullptr) store_row(static_cast<T *>(f.sum) + row * f.sum_stride + at, left, out);
                unpack(out, v[s]);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) sums[0] += v[s][j];
        }
        fetch(row + step);
        row_sum<W>(sums, scratch[team]);
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
        row_sum<W>(sums, scratch[team]);
        const float rstd = 1.f / __fsqrt_rn(sums[0] * inverse + f.eps);
        if (lane == 0 && there) {
            if (f.mean != nullptr) f.mean[row] = mean;
            if (f.rstd != nullptr) f.rstd[row] = rstd;
        }
#pragma unroll
        for (int s = 0; s < S; ++s) {
            const int64_t at = (static_cast<int64_t>(s) * W * 64 + lane) * 8, left = there ? f.cols - at : 0;
            float y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[s][j] *= rstd;
                y[j] = __builtin_fmaf(v[s][j], w[s][j], b[s][j]);
            }
            store_row(static_cast<T *>(f.y) + row * f.y_stride + at, left, pack<T>(y));
            if (f.act8.q != nullptr && there) act8_put(f.act8, row, static_cast<int>(at / 8), v[s]);
        }
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

// Rows come round as in the forward pass.  A row's operands stay as they were loaded and are taken apart twice, for the sums and for dx: half the
// registers of keeping them as floats, which the next row's operands take.  KEEP: h comes from the 8-bit rows.
template <typename T, int W, int S, bool KEEP> __global__ __launch_bounds__(threads_of<W>()) void k_layernorm_backward(Backward f) {
    constexpr bool AHEAD = W <= WAVES;  // (sixteen wavefronts have half the registers each: they load a row when it is its turn)
    __shared__ float scratch[teams_of<W>()][2 * W];
    const int lane = threadIdx.x % (W * 64), team = threadIdx.x / (W * 64);
    const int64_t teams = blockDim.x / (W * 64), step = gridDim.x * teams;
    const float inverse = 1.f / static_cast<float>(f.cols);
    struct Row {
        Raw<T> dy[S], ds[S], x[KEEP ? 1 : S];
        U2 q[KEEP ? S : 1];
        uint32_t e[KEEP ? S : 1];
        float mean, rstd;
    };
    auto fetch = [&](Row &to, int64_t row) {
        const bool there = row < f.rows;
        to.rstd = there ? f.rstd[row] : 0.f;
        to.mean = !KEEP && there ? f.mean[row] : 0.f;
#pragma unroll
        for (int s = 0; s < S; ++s) {
            const int64_t at = (static_cast<int64_t>(s) * W * 64 + lane) * 8, left = there ? f.cols - at : 0;
            to.dy[s] = load_row(static_cast<const T *>(f.dy) + row * f.dy_stride + at, left);
            if constexpr (KEEP) {
                if (left > 0) {
                    act8_get(f.act8, row, static_cast<int>(at / 8), to.q[s], to.e[s]);
                } else {
                    to.q[s] = U2{0, 0};
                    to.e[s] = 7;
                }
            } else {
                to.x[s] = load_row(static_cast<const T *>(f.x) + row * f.x_stride + at, left);
            }
            if (f.dsum != nullptr) to.ds[s] = load_row(static_cast<const T *>(f.dsum) + row * f.dsum_stride + at, left);
        }
    };
    float dw[S][8] = {}, db[S][8] = {}, w[S][8];
    int64_t row = blockIdx.x * teams + team;
    Row now;
    if constexpr (AHEAD) fetch(now, row);
#pragma unroll
    for (int s = 0; s < S; ++s) {
        const int64_t at = (static_cast<int64_t>(s) * W * 64 + lane) * 8;
        load_weight<T>(f.weight, f.wide_weight, at, f.cols - at, 1.f, w[s]);
    }
    auto take = [&](const Row &from, int s, float (&g)[8], float (&h)[8]) {
        unpack(from.dy[s], g);
        if constexpr (KEEP) {
            values_of(from.q[s], from.e[s], h);
        } else {
            unpack(from.x[s], h);
#pragma unroll
            for (int j = 0; j < 8; ++j) h[j] = (h[j] - from.mean) * from.rstd;
        }
        // (what lies behind the row is no value: without x there it would count as -mean, and a group that is marked as no number is so in its padding)
        const int64_t left = f.cols - (static_cast<int64_t>(s) * W * 64 + lane) * 8;
        if (left < 8)
#pragma unroll
            for (int j = 0; j < 8; ++j) h[j] = j < left ? h[j] : 0.f;
    };
    for (; row - team < f.rows; row += step) {  // (the workgroup's teams go round together, one without a row along with the others)
        Row next;
        fetch(AHEAD ? next : now, AHEAD ? row + step : row);
        float sums[2] = {0.f, 0.f};
#pragma unroll
        for (int s = 0; s < S; ++s) {
            float g[8], h[8];
            take(now, s, g, h);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                dw[s][j] = __builtin_fmaf(g[j], h[j], dw[s][j]);
                db[s][j] += g[j];
                g[j] *= w[s][j];
                sums[0] += g[j];
                sums[1] = __builtin_fmaf(g[j], h[j], sums[1]);
            }
        }
        row_sum<W>(sums, scratch[team]);
        const float level = sums[0] * inverse, along = sums[1] * inverse;
#pragma unroll
        for (int s = 0; s < S; ++s) {
            const int64_t at = (static_cast<int64_t>(s) * W * 64 + lane) * 8, left = row < f.rows ? f.cols - at : 0;
            float g[8], h[8], add[8] = {};
            take(now, s, g, h);
            if (f.dsum != nullptr) unpack(now.ds[s], add);
#pragma unroll
            for (int j = 0; j < 8; ++j) add[j] += now.rstd * (g[j] * w[s][j] - level - h[j] * along);
            store_row(static_cast<T *>(f.dx) + row * f.dx_stride + at, left, pack<T>(add));
        }
        if constexpr (AHEAD) now = next;
    }
    if (f.partial == nullptr) return;
    if constexpr (teams_of<W>() > 1) {  // the teams' shares, in a fixed order
        __shared__ float share[teams_of<W>()][S * W * 512];
        const int wave = threadIdx.x / 64, waves = blockDim.x / 64;
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            if (which != 0) __syncthreads();
#pragma unroll
            for (int s = 0; s < S; ++s)
#pragma unroll
                for (int j = 0; j < 8; ++j) share[team][(s * 8 + j) * W * 64 + lane] = which == 0 ? dw[s][j] : db[s][j];
            __syncthreads();
            for (int piece = wave; piece < 2 * S * W; piece += waves) {  // four of the eight columns of 64 lanes' octets
                const int s = piece / (2 * W), l = piece / 2 % W * 64 + threadIdx.x % 64, j0 = piece % 2 * 4;
                float t[4] = {};
                for (int v = 0; v < teams; ++v)
#pragma unroll
                    for (int j = 0; j < 4; ++j) t[j] += share[v][(s * 8 + j0 + j) * W * 64 + l];
                const int64_t col = (static_cast<int64_t>(s) * W * 64 + l) * 8 + j0;
                float *to = f.partial + (blockIdx.x * static_cast<int64_t>(2) + which) * f.cols + col;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (col + j < f.cols) to[j] = t[j];
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

// Columns of the partial sums added up, in a fixed order: 32 columns per workgroup, 32 lanes of parts for each.
__global__ __launch_bounds__(1024) void k_layernorm_join(const float *partial, int parts, int64_t cols, float *dweight, float *dbias, int accumulate) {
    __shared__ float share[32][33];
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 32 + threadIdx.x % 32;  // column of the [2][cols] sums
    const int lane = threadIdx.x / 32;
    float t = 0.f;
    if (i < 2 * cols) {
#pragma unroll 8
        for (int p = lane; p < parts; p += 32) t += partial[static_cast<int64_t>(p) * 2 * cols + i];
    }
    share[lane][threadIdx.x % 32] = t;
    __syncthreads();
    if (lane != 0 || i >= 2 * cols) return;
    t = 0.f;
#pragma unroll
    for (int k = 0; k < 32; ++k) t += share[k][threadIdx.x];
    float *to = i < cols ? dweight : dbias;
    if (to == nullptr) return;
    to += i < cols ? i : i - cols;
    *to = accumulate != 0 ? *to + t : t;
}

// Wavefronts to a row and octets per lane that hold a row: f is called with W and S as types.  Two octets per lane leave room in the registers for the row
// behind and the weight's gradient.
template <int N> using Int = std::integral_constant<int, N>;
template <typename F> void with_shape(int64_t cols, F &&f) {
    if (cols <= 512) return f(Int<1>(), Int<1>());
    if (cols <= 1024) return f(Int<1>(), Int<2>());
    if (cols <= 2048) return f(Int<2>(), Int<2>());
    if (cols <= 4096) return f(Int<4>(), Int<2>());
    if (cols <= 8192) return f(Int<8>(), Int<2>());
    if (cols <= 16384) return f(Int<16>(), Int<2>());
    return f(Int<16>(), Int<4>());
}

// Wavefronts and workgroups of a launch: as many rows to a workgroup as it has teams for, but fewer where that would leave compute units without one.
struct Launch {
    int waves, groups;
};
Launch launch_of(int64_t rows, int waves_per_row, int groups_per_unit) {
    int teams = waves_per_row < WAVES ? WAVES / waves_per_row : 1;
    while (teams > 1 && rows < static_cast<int64_t>(COMPUTE_UNITS) * teams) teams /= 2;
    const int64_t groups = (rows + teams - 1) / teams, most = static_cast<int64_t>(COMPUTE_UNITS) * groups_per_unit;
    return Launch{teams * waves_per_row, static_cast<int>(groups < most ? groups : most)};
}
// Of the backward pass: as many partial sums as workgroups.
Launch backward_launch(int64_t rows, int waves_per_row) { return launch_of(rows, waves_per_row, 1); }
int64_t parts_at_most(int64_t rows) { return rows < COMPUTE_UNITS ? rows : COMPUTE_UNITS; }

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
    with_type(dt, [&](auto *null) {
        using T = std::remove_pointer_t<decltype(null)>;
        with_shape(cols, [&](auto waves, auto slots) {
            constexpr int W = decltype(waves)::value, S = decltype(slots)::value;
            const Launch l = launch_of(rows, W, 2);
            hipLaunchKernelGGL((k_layernorm_forward<T, W, S>), dim3(static_cast<unsigned>(l.groups)), dim3(static_cast<unsigned>(l.waves * 64)), 0,
                               static_cast<hipStream_t>(hip_stream), f);
        });
    });
    return launched();
}

size_t adatopk_layernorm_backward_workspace_bytes(int64_t rows, int64_t cols) {
    if (!shape_ok(rows, cols) || cols > MAX_COLS) return 0;
    return align_up(static_cast<size_t>(parts_at_most(rows)) * 2 * static_cast<size_t>(cols) * sizeof(float), 256);
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
    int parts = 0;
    float *partial = weights ? static_cast<float *>(workspace) : nullptr;
    if (rows > 0) {
        const Backward f{dy,        x,        weight,      dsum,      mean, rstd, dx,
                         partial,   dy_stride, x_stride,   dsum_stride, dx_stride, rows, cols, weight_dt != dt, act8_of(const_cast<void *>(act8), rows, cols)};
        with_type(dt, [&](auto *null) {
            using T = std::remove_pointer_t<decltype(null)>;
            with_shape(cols, [&](auto waves, auto slots) {
                constexpr int W = decltype(waves)::value, S = decltype(slots)::value;
                const Launch l = backward_launch(rows, W);
                parts = l.groups;
                const auto kernel = act8 != nullptr ? k_layernorm_backward<T, W, S, true> : k_layernorm_backward<T, W, S, false>;
                hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(l.groups)), dim3(static_cast<unsigned>(l.waves * 64)), 0, st, f);
            });
        });
    }
    if (weights)  // (no rows: the sums are zero)
        hipLaunchKernelGGL(k_layernorm_join, dim3(static_cast<unsigned>((2 * cols + 31) / 32)), dim3(1024), 0, st, partial, parts, cols,
                           dweight, dbias, accumulate);
    return launched();
}

}  // extern "C"
