// Activations kept in 8 bits (store, load) and GELU, which writes them in the forward pass and reads them in the backward pass.
//
// Every kernel here is one pass over its operands, one octet (eight consecutive elements of a row) per lane; memory bounds them all.  Four neighbouring lanes
// are a group: its largest value takes two moves between lanes, its exponent is written by the first.  With two or four octets per thread, or loads and
// stores past the caches, the larger sizes took 2 to 9 % longer; on few elements the launch is all there is (2.3 to 3.6 us).
//
// A copy of 1 GiB on the same card: 5.1 TB/s.
#include <hip/hip_runtime.h>

#include "stage_ops.h"

namespace {

using namespace adatopk_stage;

constexpr int NT = 256;  // threads per workgroup

// GELU(x) = x * Phi(x).  With a = |x|, Phi(-a) = exp(-a^2 / 2) * r(a), r(a) = erfcx(a / sqrt 2) / 2, and t = 1 / (1 + 0.21 a) maps a = 0 ... inf to
// (0, 1], where r = t * (polynomial of degree 8 in t) to 2e-8 of its value (a minimax fit in relative error).  So both tails keep their
// relative precision.  The square's rounding would cost a^2 / 2 units in the exponential; its low part is put back to first order.
struct Erf {
    // Phi(x), and the density's exponential exp(-x^2 / 2).  COARSE: for results that are rounded to 16 bits, degree 6 (1e-6) and the exponential as it
    // comes (7e-6 where it is 1e-38, less the larger it is).  The slope is then off by up to 6.2e-7 where it is 2.4e-7 otherwise; at x = -0.75, the number next to its
    // zero that the 8-bit form holds, by 8e-5 of its value, a third of fp16's rounding.
    template <bool COARSE> static __device__ __forceinline__ float phi(float x, float &expo) {
        const float a = __builtin_fabsf(x);
        constexpr float C = -0.72134752044448170f;  // -log2(e) / 2, and what its rounding left off
        constexpr float C_LOW = static_cast<float>(-0.72134752044448170368 - static_cast<double>(C));
        const float h = x * x, k = h * C;
        const float e = __builtin_amdgcn_exp2f(k);
        float r;
        if constexpr (COARSE) {
            const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(a, 0.36f, 1.f));
            r = 0.046782427f;
            r = __builtin_fmaf(r, t, -0.17882647f);
            r = __builtin_fmaf(r, t, 0.17967755f);
            r = __builtin_fmaf(r, t, 0.027426654f);
            r = __builtin_fmaf(r, t, 0.13940007f);
            r = __builtin_fmaf(r, t, 0.14183038f);
            r = __builtin_fmaf(r, t, 0.14370897f);
            r *= t;
            expo = e;
        } else {
            const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(a, 0.21f, 1.f));
            r = -0.0712955f;
            r = __builtin_fmaf(r, t, 0.28180775f);
            r = __builtin_fmaf(r, t, -0.32649943f);
            r = __builtin_fmaf(r, t, 0.3449933f);
            r = __builtin_fmaf(r, t, -0.09077693f);
            r = __builtin_fmaf(r, t, 0.12347385f);
            r = __builtin_fmaf(r, t, 0.06956933f);
            r = __builtin_fmaf(r, t, 0.085012496f);
            r = __builtin_fmaf(r, t, 0.08371515f);
            r *= t;
            const float low = __builtin_fmaf(__builtin_fmaf(x, x, -h), C, __builtin_fmaf(h, C_LOW, __builtin_fmaf(h, C, -k)));
            expo = k < -126.f ? 0.f : __builtin_fmaf(e, low * 0.69314718f, e);  // (also where x is infinite, and low no number)
        }
        const float q = r * expo;
        return x < 0.f ? q : 1.f - q;
    }
    static __device__ __forceinline__ float value(float x) {
        float e;
        return x * phi<false>(x, e);
    }
    template <bool COARSE> static __device__ __forceinline__ float slope(float x) {  // Phi(x) + x * exp(-x^2 / 2) / sqrt(2 pi)
        float e;
        const float p = phi<COARSE>(x, e);
        return __builtin_fmaf(x * e, 0.39894228f, p);
    }
};
// The form with the hyperbolic tangent: x / 2 * (1 + tanh u) = x * s, s = 1 / (1 + exp(-2 u)), u = sqrt(2 / pi) (x + 0.044715 x^3).
struct Tanh {
    static __device__ __forceinline__ float sigmoid(float x) {
        constexpr float A = -2.302208198f, B = -0.10294324f;  // -2 log2(e) sqrt(2 / pi), and that times 0.044715
        const float w = x * __builtin_fmaf(x * x, B, A);
        return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(w));
    }
    static __device__ __forceinline__ float value(float x) { return x * sigmoid(x); }
    template <bool> static __device__ __forceinline__ float slope(float x) {  // s + x s (1 - s) 2 u'
        constexpr float A = 1.5957691f, B = 0.21406445f;  // 2 sqrt(2 / pi), and that times 3 * 0.044715
        const float s = sigmoid(x), rise = x * __builtin_fmaf(x * x, B, A);
        const float d = s * (1.f - s);
        return d == 0.f ? s : __builtin_fmaf(rise, d, s);  // (rise may be infinite where d is none)
    }
};

struct Shape {
    uint32_t octets;   // of all rows, the 8-bit form's padding included: a multiple of four
    Divisor per_row;   // octets of one row
    int64_t cols;
    Shape(int64_t rows, const Act8 &a, int64_t c)
        : octets(static_cast<uint32_t>(rows * (a.pitch / 8))), per_row(static_cast<uint32_t>(a.pitch / 8)), cols(c) {}
};

// q = rint(x / step), step the power of two 2^(E - 133), by a multiplication that is exact.  32768 x 768 fp32: 25 us, 5.1 TB/s.
template <typename T> __global__ __launch_bounds__(NT) void k_act8_store(const T *x, int64_t stride, Shape s, Act8 a) {
    const uint32_t t = blockIdx.x * NT + threadIdx.x;
    if (t >= s.octets) return;
    const uint32_t row = s.per_row.quotient(t), octet = t - row * s.per_row.d;
    float v[8];
    unpack(load_row(x + row * stride + octet * static_cast<int64_t>(8), s.cols - octet * static_cast<int64_t>(8), octet > 0), v);
    act8_put(a, row, static_cast<int>(octet), v);
}

// q * step.  32768 x 768 to fp32: 21.8 us, 5.8 TB/s; 16384 x 6400 to bf16: 54 us, 5.9 TB/s.
template <typename T> __global__ __launch_bounds__(NT) void k_act8_load(Act8 a, Shape s, T *y, int64_t stride) {
    const uint32_t t = blockIdx.x * NT + threadIdx.x;
    if (t >= s.octets) return;
    const uint32_t row = s.per_row.quotient(t), octet = t - row * s.per_row.d;
    U2 d;
    uint32_t E;
    act8_get(a, row, static_cast<int>(octet), d, E);
    float v[8];
    values_of(d, E, v);
    store_row(y + row * stride + octet * static_cast<int64_t>(8), s.cols - octet * static_cast<int64_t>(8), pack<T>(v));
}

// The output, and what the backward pass and the next projection's weight gradient read, from one read of the input.  16384 x 6400 bf16 with both kept in 8
// bits: 108 us, 5.9 TB/s.
template <typename T, typename F>
__global__ __launch_bounds__(NT) void k_gelu_forward(const T *x, int64_t x_stride, Shape s, T *y, int64_t y_stride, Act8 of_x, Act8 of_y) {
    const uint32_t t = blockIdx.x * NT + threadIdx.x;
    if (t >= s.octets) return;
    const uint32_t row = s.per_row.quotient(t), octet = t - row * s.per_row.d;
    const int64_t at = octet * static_cast<int64_t>(8), left = s.cols - at;
    float v[8], g[8];
    unpack(load_row(x + row * x_stride + at, left, at > 0), v);
#pragma unroll
    for (int j = 0; j < 8; ++j) g[j] = F::value(v[j]);
    const Raw<T> out = pack<T>(g);
    store_row(y + row * y_stride + at, left, out);
    if (of_x.q != nullptr) act8_put(of_x, row, static_cast<int>(octet), v);
    if (of_y.q != nullptr) {
        unpack(out, g);  // what is kept is the rounded output, which the next projection reads
        act8_put(of_y, row, static_cast<int>(octet), g);
    }
}

// dx = dy * slope(x) from the 8-bit x.  8192 x 4096 fp32: 54 us, 5.6 TB/s.  For 16-bit types, where an element's bytes are few, the slope's arithmetic would
// take as long as they do; hence its coarser form.
template <typename T, typename F>
__global__ __launch_bounds__(NT) void k_gelu_backward(const T *dy, int64_t dy_stride, Act8 a, Shape s, T *dx, int64_t dx_stride) {
    const uint32_t t = blockIdx.x * NT + threadIdx.x;
    if (t >= s.octets) return;
    const uint32_t row = s.per_row.quotient(t), octet = t - row * s.per_row.d;
    const int64_t at = octet * static_cast<int64_t>(8), left = s.cols - at;
    U2 d;
    uint32_t E;
    act8_get(a, row, static_cast<int>(octet), d, E);
    float v[8], g[8];
    unpack(load_row(dy + row * dy_stride + at, left, at > 0), g);
    values_of(d, E, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) g[j] *= F::template slope<sizeof(T) == 2>(v[j]);
    store_row(dx + row * dx_stride + at, left, pack<T>(g));
}

// Rows without anything between them whose length is a multiple of the group are one long row to a kernel that goes by elements: no division.
struct Plan {
    Act8 a;
    int64_t rows, cols;
    Plan(void *act8, int64_t r, int64_t c, bool dense) : a(act8_of(act8, r, c)), rows(r), cols(c) {
        if (dense && c % GROUP == 0) {
            cols = r * c;
            rows = 1;
            a.pitch = cols;
        }
    }
    Shape shape() const { return Shape(rows, a, cols); }
    dim3 grid() const { return dim3(static_cast<unsigned>((static_cast<uint64_t>(rows) * (a.pitch / 8) + NT - 1) / NT)); }
};

}  // namespace

extern "C" {

adatopk_status adatopk_act8_store(const void *x, int64_t x_stride, int64_t rows, int64_t cols, adatopk_dtype dt, void *act8, void *hip_stream) {
    if (!dtype_ok(dt) || !shape_ok(rows, cols)) return ADATOPK_EINVAL;
    if (rows == 0 || cols == 0) return ADATOPK_OK;
    if (!matrix_ok(x, x_stride, rows, cols, dt) || !pointer_ok(act8, 16)) return ADATOPK_EINVAL;
    const Plan p(act8, rows, cols, rows == 1 || x_stride == cols);
    with_type(dt, [&](auto *null) {
        using T = std::remove_pointer_t<decltype(null)>;
        hipLaunchKernelGGL(k_act8_store<T>, p.grid(), dim3(NT), 0, static_cast<hipStream_t>(hip_stream), static_cast<const T *>(x), x_stride, p.shape(), p.a);
    });
    return launched();
}

adatopk_status adatopk_act8_load(const void *act8, int64_t rows, int64_t cols, adatopk_dtype dt, void *y, int64_t y_stride, void *hip_stream) {
    if (!dtype_ok(dt) || !shape_ok(rows, cols)) return ADATOPK_EINVAL;
    if (rows == 0 || cols == 0) return ADATOPK_OK;
    if (!matrix_ok(y, y_stride, rows, cols, dt) || !pointer_ok(act8, 16)) return ADATOPK_EINVAL;
    const Plan p(const_cast<void *>(act8), rows, cols, rows == 1 || y_stride == cols);
    with_type(dt, [&](auto *null) {
        using T = std::remove_pointer_t<decltype(null)>;
        hipLaunchKernelGGL(k_act8_load<T>, p.grid(), dim3(NT), 0, static_cast<hipStream_t>(hip_stream), p.a, p.shape(), static_cast<T *>(y), y_stride);
    });
    return launched();
}

adatopk_status adatopk_gelu_forward(const void *x, int64_t x_stride, int64_t rows, int64_t cols, adatopk_dtype dt, int32_t use_tanh, void *y,
                                    int64_t y_stride, void *act8_x, void *act8_y, void *hip_stream) {
    if (!dtype_ok(dt) || !shape_ok(rows, cols)) return ADATOPK_EINVAL;
    if (rows == 0 || cols == 0) return ADATOPK_OK;
    if (!matrix_ok(x, x_stride, rows, cols, dt) || !matrix_ok(y, y_stride, rows, cols, dt) || !pointer_ok_or_null(act8_x, 16) ||
        !pointer_ok_or_null(act8_y, 16))
        return ADATOPK_EINVAL;
    const bool dense = rows == 1 || (x_stride == cols && y_stride == cols);
    const Plan p(act8_x, rows, cols, dense), q(act8_y, rows, cols, dense);
    with_type(dt, [&](auto *null) {
        using T = std::remove_pointer_t<decltype(null)>;
        const auto kernel = use_tanh != 0 ? k_gelu_forward<T, Tanh> : k_gelu_forward<T, Erf>;
        hipLaunchKernelGGL(kernel, p.grid(), dim3(NT), 0, static_cast<hipStream_t>(hip_stream), static_cast<const T *>(x), x_stride, p.shape(),
                           static_cast<T *>(y), y_stride, p.a, q.a);
    });
    return launched();
}

adatopk_status adatopk_gelu_backward(const void *dy, int64_t dy_stride, const void *act8_x, int64_t rows, int64_t cols, adatopk_dtype dt,
                                     int32_t use_tanh, void *dx, int64_t dx_stride, void *hip_stream) {
    if (!dtype_ok(dt) || !shape_ok(rows, cols)) return ADATOPK_EINVAL;
    if (rows == 0 || cols == 0) return ADATOPK_OK;
    if (!matrix_ok(dy, dy_stride, rows, cols, dt) || !matrix_ok(dx, dx_stride, rows, cols, dt) || !pointer_ok(act8_x, 16)) return ADATOPK_EINVAL;
    const Plan p(const_cast<void *>(act8_x), rows, cols, rows == 1 || (dy_stride == cols && dx_stride == cols));
    with_type(dt, [&](auto *null) {
        using T = std::remove_pointer_t<decltype(null)>;
        const auto kernel = use_tanh != 0 ? k_gelu_backward<T, Tanh> : k_gelu_backward<T, Erf>;
        hipLaunchKernelGGL(kernel, p.grid(), dim3(NT), 0, static_cast<hipStream_t>(hip_stream), static_cast<const T *>(dy), dy_stride, p.a, p.shape(),
                           static_cast<T *>(dx), dx_stride);
    });
    return launched();
}

}  // extern "C"
