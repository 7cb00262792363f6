// Matrices in 8-bit floating point: activations and gradients put away with a scale for 128 elements of a row, weights with one for a tile of 128 x 128, as
// they are and transposed, and what is put away read back.
//
// Every kernel is one pass over its operands, octets of a row per lane; memory bounds them all, and on few elements the launch.  777 x 1001 fp16: store 2.7 us,
// load 2.8; 16384 x 1600 to bf16: load 14, 5.6 TB/s; weights of 6400 x 1600 bf16 both ways 11.5, 3.6 TB/s of 41 MB.
#include <hip/hip_runtime.h>

#include "fp8_form.h"

namespace {

using namespace adatopk_stage;

constexpr int NT = 256;  // threads per workgroup

struct Shape {
    uint32_t octets;  // of all rows, the padding included: a multiple of sixteen
    Divisor per_row;
    int64_t cols;
    Shape(int64_t rows, const Fp8 &a, int64_t c) : octets(static_cast<uint32_t>(rows * (a.pitch / 8))), per_row(static_cast<uint32_t>(a.pitch / 8)), cols(c) {}
};

template <typename T> __global__ __launch_bounds__(NT) void k_fp8_store(const T *x, int64_t stride, Shape s, Fp8 a) {
    const uint32_t t = blockIdx.x * NT + threadIdx.x;
    if (t >= s.octets) return;
    const uint32_t row = s.per_row.quotient(t), octet = t - row * s.per_row.d;
    float v[8];
    unpack(load_row(x + row * stride + octet * static_cast<int64_t>(8), s.cols - octet * static_cast<int64_t>(8), octet > 0), v);
    fp8_put(a, row, static_cast<int>(octet), v);
}

template <typename T> __global__ __launch_bounds__(NT) void k_fp8_load(Fp8 a, Shape s, T *y, int64_t stride) {
    const uint32_t t = blockIdx.x * NT + threadIdx.x;
    if (t >= s.octets) return;
    const uint32_t row = s.per_row.quotient(t), octet = t - row * s.per_row.d;
    const int64_t at = octet * static_cast<int64_t>(8);
    if (at >= s.cols) return;
    const U2 d = *reinterpret_cast<const U2 *>(a.q + row * a.pitch + at);
    float v[8];
    fp8_values(d, a.s[octet / BLOCK_OCTETS * a.scale_pitch + row], v);
    store_row(y + row * stride + at, s.cols - at, pack<T>(v));
}

// Bytes j of a, b, c and d side by side, for j = 0 ... 3.
__device__ __forceinline__ void transpose_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d, uint32_t (&out)[4]) {
    const uint32_t ab_low = __builtin_amdgcn_perm(b, a, 0x05010400u), ab_high = __builtin_amdgcn_perm(b, a, 0x07030602u);
    const uint32_t cd_low = __builtin_amdgcn_perm(d, c, 0x05010400u), cd_high = __builtin_amdgcn_perm(d, c, 0x07030602u);
    out[0] = __builtin_amdgcn_perm(cd_low, ab_low, 0x05040100u);
    out[1] = __builtin_amdgcn_perm(cd_low, ab_low, 0x07060302u);
    out[2] = __builtin_amdgcn_perm(cd_high, ab_high, 0x05040100u);
    out[3] = __builtin_amdgcn_perm(cd_high, ab_high, 0x07060302u);
}

// A workgroup takes a tile of 128 x 128, a thread eight rows of an octet: their largest magnitude is the workgroup's, and the transposed tile comes from the
// same registers, 8 x 8 numbers turned by byte permutes and put together to rows of 128 bytes in LDS, whose eights of bytes lie where no two of the lanes that
// store or read together meet in a bank.
template <typename T>
__global__ __launch_bounds__(NT) void k_fp8_store_weight(const T *w, int64_t stride, int64_t rows, int64_t cols, Fp8 straight, Fp8 across, int tiles_across) {
    __shared__ uint32_t most[NT / 64];
    __shared__ __attribute__((aligned(16))) U2 turned[128 * 16];
    const int64_t row0 = static_cast<int64_t>(blockIdx.x / tiles_across) * 128, col0 = static_cast<int64_t>(blockIdx.x % tiles_across) * 128;
    const int octet = threadIdx.x % 16, eight = threadIdx.x / 16;
    const int64_t at = col0 + octet * 8, first = row0 + eight * 8;
    Raw<T> raw[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) raw[i] = fetch_row(w + (first + i) * stride + at, first + i < rows ? cols - at : 0, at > 0);
    uint32_t m = 0;
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        raw[i] = settle(raw[i], first + i < rows ? cols - at : 0, at > 0);
        unpack(raw[i], v);
        const uint32_t k = largest_magnitude(v);
        m = m > k ? m : k;
    }
    m = max_of_sixteen(m);
#pragma unroll
    for (int lane = 16; lane < 64; lane *= 2) {
        const uint32_t o = static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), lane));
        m = m > o ? m : o;
    }
    if (threadIdx.x % 64 == 0) most[threadIdx.x / 64] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NT / 64; ++i) m = m > most[i] ? m : most[i];
    const uint32_t S = fp8_scale(m);
    U2 d[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        unpack(raw[i], v);
        d[i] = fp8_numbers(v, S);
        if (straight.q != nullptr && first + i < rows) *reinterpret_cast<U2 *>(straight.q + (first + i) * straight.pitch + at) = d[i];
    }
    if (straight.q != nullptr && threadIdx.x < 128 && row0 + threadIdx.x < rows) straight.s[blockIdx.x % tiles_across * straight.scale_pitch + row0 + threadIdx.x] = S;
    if (across.q == nullptr) return;
    if (threadIdx.x < 128 && col0 + threadIdx.x < cols) across.s[blockIdx.x / tiles_across * across.scale_pitch + col0 + threadIdx.x] = S;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t upper[4], lower[4];  // of columns 4 h ... 4 h + 3: rows 0 to 3, rows 4 to 7
        transpose_bytes(d[0][h], d[1][h], d[2][h], d[3][h], upper);
        transpose_bytes(d[4][h], d[5][h], d[6][h], d[7][h], lower);
#pragma unroll
        for (int j = 0; j < 4; ++j) turned[(octet * 8 + 4 * h + j) * 16 + (eight ^ octet)] = U2{upper[j], lower[j]};
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int col = static_cast<int>(threadIdx.x) / 8 + 32 * i, pair = threadIdx.x % 8, x = col / 8;
        if (col0 + col >= cols) break;
        // (exchanged where the column's octet is odd)
        const U2 one = turned[col * 16 + ((2 * pair) ^ x)], two = turned[col * 16 + ((2 * pair + 1) ^ x)];
        *reinterpret_cast<U4 *>(across.q + (col0 + col) * across.pitch + row0 + 16 * pair) = U4{one[0], one[1], two[0], two[1]};
    }
}

dim3 groups(const Shape &s) { return dim3((s.octets + NT - 1) / NT); }

}  // namespace

extern "C" {

size_t adatopk_fp8_bytes(int64_t rows, int64_t cols) { return fp8_shape_ok(rows, cols) ? adatopk_internal::fp8_bytes(rows, cols) : 0; }

adatopk_status adatopk_fp8_store(const void *x, int64_t x_stride, int64_t rows, int64_t cols, adatopk_dtype dt, void *fp8, void *hip_stream) {
    if (!dtype_ok(dt) || !fp8_shape_ok(rows, cols)) return ADATOPK_EINVAL;
    if (rows == 0 || cols == 0) return ADATOPK_OK;
    if (!matrix_ok(x, x_stride, rows, cols, dt) || !pointer_ok(fp8, 16)) return ADATOPK_EINVAL;
    const Fp8 a = fp8_of(fp8, rows, cols);
    const Shape s(rows, a, cols);
    with_type(dt, [&](auto *null) {
        using T = std::remove_pointer_t<decltype(null)>;
        hipLaunchKernelGGL(k_fp8_store<T>, groups(s), dim3(NT), 0, static_cast<hipStream_t>(hip_stream), static_cast<const T *>(x), x_stride, s, a);
    });
    return launched();
}

adatopk_status adatopk_fp8_store_weight(const void *w, int64_t w_stride, int64_t rows, int64_t cols, adatopk_dtype dt, void *fp8, void *fp8_transposed,
                                        void *hip_stream) {
    if (!dtype_ok(dt) || rows < 0 || cols < 0 || (fp8 != nullptr && !fp8_shape_ok(rows, cols)) || (fp8_transposed != nullptr && !fp8_shape_ok(cols, rows)))
        return ADATOPK_EINVAL;
    if (rows == 0 || cols == 0) return ADATOPK_OK;
    if (!matrix_ok(w, w_stride, rows, cols, dt) || !pointer_ok_or_null(fp8, 16) || !pointer_ok_or_null(fp8_transposed, 16) ||
        (fp8 == nullptr && fp8_transposed == nullptr))
        return ADATOPK_EINVAL;
    const Fp8 straight = fp8_of(fp8, rows, cols), across = fp8_of(fp8_transposed, cols, rows);
    const int64_t tiles_across = straight.pitch / adatopk_internal::FP8_BLOCK, tiles = tiles_across * (across.pitch / adatopk_internal::FP8_BLOCK);
    if (tiles > INT32_MAX) return ADATOPK_EINVAL;
    with_type(dt, [&](auto *null) {
        using T = std::remove_pointer_t<decltype(null)>;
        hipLaunchKernelGGL(k_fp8_store_weight<T>, dim3(static_cast<unsigned>(tiles)), dim3(NT), 0, static_cast<hipStream_t>(hip_stream), static_cast<const T *>(w),
                           w_stride, rows, cols, straight, across, static_cast<int>(tiles_across));
    });
    return launched();
}

adatopk_status adatopk_fp8_load(const void *fp8, int64_t rows, int64_t cols, adatopk_dtype dt, void *y, int64_t y_stride, void *hip_stream) {
    if (!dtype_ok(dt) || !fp8_shape_ok(rows, cols)) return ADATOPK_EINVAL;
    if (rows == 0 || cols == 0) return ADATOPK_OK;
    if (!matrix_ok(y, y_stride, rows, cols, dt) || !pointer_ok(fp8, 16)) return ADATOPK_EINVAL;
    const Fp8 a = fp8_of(const_cast<void *>(fp8), rows, cols);
    const Shape s(rows, a, cols);
    with_type(dt, [&](auto *null) {
        using T = std::remove_pointer_t<decltype(null)>;
        hipLaunchKernelGGL(k_fp8_load<T>, groups(s), dim3(NT), 0, static_cast<hipStream_t>(hip_stream), a, s, static_cast<T *>(y), y_stride);
    });
    return launched();
}

}  // extern "C"
