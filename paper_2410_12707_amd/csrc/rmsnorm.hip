// Root-mean-square norm over the rows of a matrix, forward and backward, with the residual addition before it, the divided rows kept in 8-bit whole numbers for
// the backward pass and the weighted ones put into 8-bit floating point for the product that reads them.
//
//   forward   s = x + residual, rounded to the type (the next block reads it);  rstd = 1 / sqrt(sum s^2 / n + eps);  h = s * rstd;  y = weight * h
//   backward  g = dy * weight;  dx = rstd * (g - h * (sum g h) / n) + dsum;  dweight = sum over rows dy * h: norm.h's
//
// A row is read once and held in registers between the sum and its use.  The forward pass's sum is in 64 bits and 1 / sqrt in two floats, and what goes into 8
// bits carries the sign of what its rounding to 32 left off: so the 8-bit numbers are those of the formulas, where a rounding before theirs would move one value in
// a million by a whole step of theirs.  On few rows the launch and the latency of load, sum and store
// bound it (512 x 768 fp32 4.5 us).  On many, from x to y alone, memory: 16384 x 2048 bf16 22.5 us, 6.0 TB/s, with residual and sum 42.6, 6.3.  Numbers in 8 bits
// are work for the vector unit, 70 instructions on an element with both forms: 16384 x 1600 with all five outputs 58 us, 4.6 TB/s, of 2048 68 us, 4.9.  (Forming what
// the roundings left off only in wavefronts with a value next to a border between two numbers takes a quarter of the instructions away, but ten registers more, and
// with them the fourth wavefront of a SIMD: 67 us, held to 128 registers with spills 64.  One octet to a lane 65.)
#include <hip/hip_runtime.h>

#ifdef ADATOPK_MEASURE_BUILD
#include "adatopk_measure.h"
#endif
#include "norm.h"

#include "fp8_form.h"

namespace {

struct Forward {
    const void *x, *residual, *weight;
    void *sum, *y;
    float *rstd;
    int64_t x_stride, residual_stride, sum_stride, y_stride;
    int64_t rows, cols;
    float eps;
    bool wide_weight;  // the weight in fp32 beside 16-bit rows
    Act8 act8;
    Fp8 fp8;
};

// h + low, a sum whose first part is its nearest float, rounded to odd: the float next to it towards zero, its last bit set.  Whatever is compared with it or
// rounds it to fewer bits does so as with the sum itself.
__device__ __forceinline__ float to_odd(float h, float low) {
    if (!(__builtin_fabsf(low) > 0.f)) return h;
    const uint32_t bits = __float_as_uint(h), towards = (bits ^ __float_as_uint(low)) >> 31;
    return __uint_as_float((bits - towards) | 1u);
}

template <typename T, int L, int S> __global__ __launch_bounds__(threads_of(L)) void k_rmsnorm_forward(Forward f) {
    constexpr bool HELD = held(S);
    __shared__ double scratch[threads_of(L) / L][L > 64 ? L / 64 : 1];
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
    float w[HELD ? S : 1][8];
    auto weights = [&](int s, int to) { load_weight<T>(f.weight, f.wide_weight, place(s), f.cols - place(s), 1.f, w[to]); };
    if constexpr (HELD) {
        fetch(row);
#pragma unroll
        for (int s = 0; s < S; ++s) weights(s, s);
    }
    for (; row - team < f.rows; row += step) {  // (the workgroup's teams go round together, one without a row along with the others)
        const bool there = row < f.rows;
        if constexpr (!HELD) fetch(row);
        float v[S][8];
        double sums[1] = {0.0};
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
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const double d = static_cast<double>(v[s][j]);
                sums[0] = __builtin_fma(d, d, sums[0]);
            }
        }
        if constexpr (HELD) fetch(row + step);
        team_sum<L>(sums, scratch[team]);
        const double square = __builtin_fma(sums[0], inverse, static_cast<double>(f.eps));
        double rstd = __builtin_amdgcn_rsq(square);  // to some 23 bits; a Newton step doubles them
        if (square > 0.0 && square < __builtin_inf()) rstd = rstd * __builtin_fma(-0.5 * square * rstd, rstd, 1.5);
        const float high = static_cast<float>(rstd), low = __builtin_fabsf(high) < __builtin_inff() ? static_cast<float>(rstd - static_cast<double>(high)) : 0.f;
        if (lane == 0 && there && f.rstd != nullptr) f.rstd[row] = high;
#pragma unroll
        for (int s = 0; s < S; ++s) {
            const int64_t at = place(s), left = there ? f.cols - at : 0;
            const int k = HELD ? s : 0;
            if constexpr (!HELD) weights(s, 0);
            float h[8], y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                h[j] = __builtin_fmaf(v[s][j], high, v[s][j] * low);
                y[j] = h[j] * w[k][j];
            }
            if (f.y != nullptr) store_row(static_cast<T *>(f.y) + row * f.y_stride + at, left, pack<T>(y));
            if ((f.act8.q == nullptr && f.fp8.q == nullptr) || !there) continue;
            float h_low[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) h_low[j] = __builtin_fmaf(v[s][j], low, __builtin_fmaf(v[s][j], high, -h[j]));
            if (f.act8.q != nullptr) {
                float t[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) t[j] = to_odd(h[j], h_low[j]);
                act8_put(f.act8, row, static_cast<int>(at / 8), t);
            }
            if (f.fp8.q != nullptr) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float rest = __builtin_fmaf(h_low[j], w[k][j], __builtin_fmaf(h[j], w[k][j], -y[j]));
                    const float sum = y[j] + rest;
                    y[j] = to_odd(sum, (y[j] - sum) + rest);
                }
                fp8_put(f.fp8, row, static_cast<int>(at / 8), y);
            }
        }
    }
}

// The teams of the layer norm, but none of eight lanes: sixteen share a scale.
template <typename F> void with_forward_shape(int64_t cols, F &&f) {
    if (cols <= 64) return f(Int<16>(), Int<1>());
    with_shape<false>(cols, f);
}

}  // namespace

extern "C" {

adatopk_status adatopk_rmsnorm_forward(const void *x, int64_t x_stride, const void *residual, int64_t residual_stride, const void *weight,
                                       adatopk_dtype weight_dt, int64_t rows, int64_t cols, adatopk_dtype dt, float eps, void *sum, int64_t sum_stride, void *y,
                                       int64_t y_stride, float *rstd, void *act8, void *fp8, void *hip_stream) {
    if (!dtype_ok(dt) || !(weight_dt == dt || weight_dt == ADATOPK_F32) || !shape_ok(rows, cols) || (fp8 != nullptr && !fp8_shape_ok(rows, cols)) || cols > MAX_COLS ||
        !(eps >= 0.f))
        return ADATOPK_EINVAL;
    if (rows == 0 || cols == 0) return ADATOPK_OK;
    if (!matrix_ok(x, x_stride, rows, cols, dt) || (y != nullptr ? !matrix_ok(y, y_stride, rows, cols, dt) : fp8 == nullptr) || !weights_ok(weight, weight_dt) ||
        (residual != nullptr && !matrix_ok(residual, residual_stride, rows, cols, dt)) || (sum != nullptr && residual == nullptr) ||
        (sum != nullptr && !matrix_ok(sum, sum_stride, rows, cols, dt)) || !pointer_ok_or_null(rstd, 4) || !pointer_ok_or_null(act8, 16) ||
        !pointer_ok_or_null(fp8, 16))
        return ADATOPK_EINVAL;
    const Forward f{x,        residual,   weight, sum,  y,    rstd, x_stride,         residual_stride,           sum_stride,
                    y_stride, rows,       cols,   eps,  weight_dt != dt, act8_of(act8, rows, cols), fp8_of(fp8, rows, cols)};
    with_type(dt, [&](auto *null) {
        using T = std::remove_pointer_t<decltype(null)>;
        with_forward_shape(cols, [&](auto lanes, auto slots) {
            constexpr int L = decltype(lanes)::value, S = decltype(slots)::value;
            const Launch l = launch_of(rows, L, forward_groups_per_unit(S));
            hipLaunchKernelGGL((k_rmsnorm_forward<T, L, S>), dim3(static_cast<unsigned>(l.groups)), dim3(static_cast<unsigned>(l.threads)), 0,
                               static_cast<hipStream_t>(hip_stream), f);
        });
    });
    return launched();
}

size_t adatopk_rmsnorm_backward_workspace_bytes(int64_t rows, int64_t cols) {
    if (!shape_ok(rows, cols) || cols > MAX_COLS) return 0;
    return align_up(static_cast<size_t>(parts_at_most(rows, cols)) * static_cast<size_t>(cols) * sizeof(float), 256);
}

adatopk_status adatopk_rmsnorm_backward(const void *dy, int64_t dy_stride, const void *x, int64_t x_stride, const void *act8, const float *rstd, const void *weight,
                                        adatopk_dtype weight_dt, const void *dsum, int64_t dsum_stride, int64_t rows, int64_t cols, adatopk_dtype dt, void *dx,
                                        int64_t dx_stride, float *dweight, int32_t accumulate, void *workspace, size_t workspace_bytes, void *hip_stream) {
    if (!dtype_ok(dt) || !(weight_dt == dt || weight_dt == ADATOPK_F32) || !shape_ok(rows, cols) || cols > MAX_COLS) return ADATOPK_EINVAL;
    if (cols == 0) return ADATOPK_OK;
    if (!pointer_ok_or_null(dweight, 4)) return ADATOPK_EINVAL;
    if (rows > 0 && (!matrix_ok(dy, dy_stride, rows, cols, dt) || !matrix_ok(dx, dx_stride, rows, cols, dt) || (x == nullptr) == (act8 == nullptr) ||
                     (x != nullptr && !matrix_ok(x, x_stride, rows, cols, dt)) || !pointer_ok_or_null(act8, 16) || !pointer_ok(rstd, 4) ||
                     !weights_ok(weight, weight_dt) || (dsum != nullptr && !matrix_ok(dsum, dsum_stride, rows, cols, dt)) ||
                     (dweight != nullptr && !pointer_ok(workspace, 256))))
        return ADATOPK_EINVAL;
    if (dweight != nullptr && rows > 0 && workspace_bytes < adatopk_rmsnorm_backward_workspace_bytes(rows, cols)) return ADATOPK_EWORKSPACE;
    launch_backward<false>(Backward{dy, x, weight, dsum, nullptr, rstd, dx, static_cast<float *>(dweight != nullptr ? workspace : nullptr), dweight, nullptr, accumulate,
                                    0, 0, rows, dy_stride, x_stride, dsum_stride, dx_stride, rows, cols, weight_dt != dt,
                                    act8_of(const_cast<void *>(act8), rows, cols)},
                           dt, static_cast<hipStream_t>(hip_stream));
    return launched();
}

}  // extern "C"
