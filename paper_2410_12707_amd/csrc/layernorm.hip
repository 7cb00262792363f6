// Layer norm over the rows of a matrix, forward and backward, with the residual addition before it and the normalised rows kept in 8 bits.
//
//   forward   s = x + residual, rounded to the type (the next block reads it);  mean = sum s / n;  rstd = 1 / sqrt(sum (s - mean)^2 / n + eps);
//             h = (s - mean) * rstd;  y = weight * h + bias
//   backward  g = dy * weight;  dx = rstd * (g - sum g / n - h * (sum g h) / n) + dsum;  dweight = sum over rows dy * h;  dbias = sum over rows dy
//             with h from the kept 8-bit rows, or from x, mean and rstd
//
// A row is read once and held in registers between the sums and their use (rows of more than 8192 elements are read again by the backward pass).  All sums
// are in 32 bits, the mean's in 64, and in a fixed order.  Memory bounds both passes on many rows; on few, the launch and the latency of load, sums and store.
#include <hip/hip_runtime.h>

#ifdef ADATOPK_MEASURE_BUILD
#include "adatopk_measure.h"
#endif
#include "norm.h"

namespace {

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
// A workgroup's teams take a row each, and rows come round in steps of the grid: weight and bias stay in registers, and the next row is on its way while this
// one is summed up.  The squares are summed of what the mean leaves, not of the values: nothing cancels.  16384 x 1600 bf16 with the residual, the sum and
// 8-bit rows: 51 us, 4.6 TB/s; from x to y alone 21.8 us, 4.8 TB/s; 32768 x 768 fp32 32 us, 6.3 TB/s; 512 x 768 fp32 3.9 us.
template <typename T, int L, int S> __global__ __launch_bounds__(threads_of(L)) void k_layernorm_forward(Forward f) {
    constexpr bool HELD = held(S);
    __shared__ double scratch[threads_of(L) / L][L > 64 ? L / 64 : 1];
    __shared__ float squares[threads_of(L) / L][L > 64 ? L / 64 : 1];
    const int lane = threadIdx.x % L, team = threadIdx.x / L;
    const int64_t teams = blockDim.x / L, step = gridDim.x * teams;
    const double inverse = 1.0 / static_cast<double>(f.cols);
    int64_t row = blockIdx.x * teams + team;
    auto place = [&](int s) {  // (rows that are not held: what is derived from it is not kept from row to row either)
        int l = lane;
        if constexpr (!HELD) asm volatile("" : "+v"(l));
        return (static_cast<int64_t>(s) * L + l) * 8;
    };
    Raw<T> x[S], r[S];
    auto fetch = [&](int64_t of) {
#pragma unroll
        for (int s = 0; s < S; ++s) {
            const int64_t at = place(s), left = of < f.rows ? f.cols - at : 0;
            x[s] = fetch_row(static_cast<const T *>(f.x) + of * f.x_stride + at, left, at > 0);
            if (f.residual != nullptr) r[s] = fetch_row(static_cast<const T *>(f.residual) + of * f.residual_stride + at, left, at > 0);
        }
    };
    float w[HELD ? S : 1][8], b[HELD ? S : 1][8];
    auto weights = [&](int s, int to) {
        load_weight<T>(f.weight, f.wide_weight, place(s), f.cols - place(s), 1.f, w[to]);
        load_weight<T>(f.bias, f.wide_weight, place(s), f.cols - place(s), 0.f, b[to]);
    };
    if constexpr (HELD) {
        fetch(row);
#pragma unroll
        for (int s = 0; s < S; ++s) weights(s, s);
    }
    for (; row - team < f.rows; row += step) {  // (the workgroup's teams go round together, one without a row along with the others)
        const bool there = row < f.rows;
        if constexpr (!HELD) fetch(row);
        float v[S][8];
        double sums[1] = {0.0};  // (64 bits: what is left of values that cancel is the mean)
#pragma unroll
        for (int s = 0; s < S; ++s) {
            const int64_t at = place(s), left = there ? f.cols - at : 0;
            unpack(settle(x[s], left, at > 0), v[s]);
            if (f.residual != nullptr) {
                float t[8];
                unpack(settle(r[s], left, at > 0), t);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[s][j] += t[j];
                const Raw<T> out = pack<T>(v[s]);
                if (f.sum != nullptr) store_row(static_cast<T *>(f.sum) + row * f.sum_stride + at, left, out);
                unpack(out, v[s]);
            }
            if constexpr (sizeof(T) == 2) {  // (eight values of 8 or 11 bits add up in 24 but for what lies 2^10 below the largest)
                sums[0] += ((v[s][0] + v[s][1]) + (v[s][2] + v[s][3])) + ((v[s][4] + v[s][5]) + (v[s][6] + v[s][7]));
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) sums[0] += v[s][j];
            }
        }
        if constexpr (HELD) fetch(row + step);
        team_sum<L>(sums, scratch[team]);
        const float mean = static_cast<float>(sums[0] * inverse);
        float square[1] = {0.f};
#pragma unroll
        for (int s = 0; s < S; ++s) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[s][j] = place(s) + j < f.cols ? v[s][j] - mean : 0.f;
                square[0] = __builtin_fmaf(v[s][j], v[s][j], square[0]);
            }
        }
        team_sum<L>(square, squares[team]);
        const float rstd = 1.f / __fsqrt_rn(square[0] * static_cast<float>(inverse) + f.eps);
        if (lane == 0 && there) {
            if (f.mean != nullptr) f.mean[row] = mean;
            if (f.rstd != nullptr) f.rstd[row] = rstd;
        }
#pragma unroll
        for (int s = 0; s < S; ++s) {
            const int64_t at = place(s), left = there ? f.cols - at : 0;
            const int k = HELD ? s : 0;
            if constexpr (!HELD) weights(s, 0);
            float y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[s][j] *= rstd;
                y[j] = __builtin_fmaf(v[s][j], w[k][j], b[k][j]);
            }
            store_row(static_cast<T *>(f.y) + row * f.y_stride + at, left, pack<T>(y));
            if (f.act8.q != nullptr && there) act8_put(f.act8, row, static_cast<int>(at / 8), v[s]);
        }
    }
}

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
        with_shape<false>(cols, [&](auto lanes, auto slots) {
            constexpr int L = decltype(lanes)::value, S = decltype(slots)::value;
            const Launch l = launch_of(rows, L, forward_groups_per_unit(S));
            hipLaunchKernelGGL((k_layernorm_forward<T, L, S>), dim3(static_cast<unsigned>(l.groups)), dim3(static_cast<unsigned>(l.threads)), 0,
                               static_cast<hipStream_t>(hip_stream), f);
        });
    });
    return launched();
}

size_t adatopk_layernorm_backward_workspace_bytes(int64_t rows, int64_t cols) {
    if (!shape_ok(rows, cols) || cols > MAX_COLS) return 0;
    return align_up(static_cast<size_t>(parts_at_most(rows, cols)) * 2 * static_cast<size_t>(cols) * sizeof(float), 256);
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
    launch_backward<true>(Backward{dy, x, weight, dsum, mean, rstd, dx, static_cast<float *>(weights ? workspace : nullptr), dweight, dbias, accumulate, 0, 0, rows,
                                   dy_stride, x_stride, dsum_stride, dx_stride, rows, cols, weight_dt != dt, act8_of(const_cast<void *>(act8), rows, cols)},
                          dt, static_cast<hipStream_t>(hip_stream));
    return launched();
}

#ifdef ADATOPK_MEASURE_BUILD
adatopk_status adatopk_measure_layernorm_cut(int64_t rows, int64_t cols, int32_t backward, int32_t *out) {
    if (!shape_ok(rows, cols) || cols > MAX_COLS || rows == 0 || cols == 0) return ADATOPK_EINVAL;
    const bool columns = backward != 0 && by_columns(rows, cols);
    const auto put = [&](auto lanes, auto slots) {
        const Launch l = columns         ? columns_launch(rows, lanes(), cols)
                         : backward != 0 ? launch_of(rows, lanes(), groups_per_unit(slots()))
                                         : launch_of(rows, lanes(), forward_groups_per_unit(slots()));
        out[0] = lanes();
        out[1] = slots();
        out[2] = l.groups * (l.threads / lanes());
        out[3] = columns ? strip_parts(rows) : 0;
    };
    if (backward != 0)
        with_shape<true>(cols, put);
    else
        with_shape<false>(cols, put);
    return ADATOPK_OK;
}
#endif

}  // extern "C"
