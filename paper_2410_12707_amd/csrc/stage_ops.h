// What the kernels of a stage's training step share (activations kept in 8 bits, GELU, layer norm, weight gradient): loads and stores of
// eight elements, the 8-bit form, sums over a wavefront, argument checks.  Internal to the library.
//
// All of them handle a row as octets, eight consecutive elements per lane: 16 bytes of a 16-bit type, 32 of fp32, 8 of the 8-bit form.  Four
// octets are a group of the 8-bit form, so a group is four neighbouring lanes and its largest magnitude two exchanges within a quad.
#ifndef ADATOPK_STAGE_OPS_H
#define ADATOPK_STAGE_OPS_H

#include <hip/hip_runtime.h>

#include <stddef.h>
#include <stdint.h>

#include <type_traits>

#include "act8_layout.h"
#include "adatopk.h"

namespace adatopk_stage {

using adatopk_internal::align_up;
using adatopk_internal::dtype_ok;
using adatopk_internal::elem_size;

struct Bf16 {
    uint16_t bits;
};
struct F16 {
    _Float16 value;
};

// ---- the 8-bit form's buffer
constexpr int GROUP = static_cast<int>(adatopk_internal::ACT8_GROUP);
struct Act8 {
    int8_t *q;
    uint8_t *e;
    int64_t pitch;  // numbers from one row to the next; pitch / 32 exponents
};
inline Act8 act8_of(void *buffer, int64_t rows, int64_t cols) {
    int8_t *q = static_cast<int8_t *>(buffer);
    return Act8{q, q == nullptr ? nullptr : reinterpret_cast<uint8_t *>(q) + adatopk_internal::act8_exponents_at(rows, cols), adatopk_internal::act8_pitch(cols)};
}
inline bool shape_ok(int64_t rows, int64_t cols) { return adatopk_internal::act8_shape_ok(rows, cols); }
inline bool pointer_ok(const void *p, size_t alignment) { return p != nullptr && reinterpret_cast<uintptr_t>(p) % alignment == 0; }
inline bool pointer_ok_or_null(const void *p, size_t alignment) { return reinterpret_cast<uintptr_t>(p) % alignment == 0; }

#if defined(__HIPCC__)
// ---- octets.  The vector types ask for no more than the element's alignment: the memory system takes wide accesses at any address, so rows
// of any stride go the same way, and only the last octet of a row that is no multiple of eight is read and written by elements.
typedef uint32_t U4 __attribute__((ext_vector_type(4)));
typedef uint32_t U2 __attribute__((ext_vector_type(2)));
typedef uint32_t U4a2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t U4a4 __attribute__((ext_vector_type(4), aligned(4)));

__device__ __forceinline__ float bf16_to_f32(uint32_t bits) { return __uint_as_float(bits << 16); }
typedef __bf16 B2 __attribute__((ext_vector_type(2)));
typedef _Float16 H2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {  // to nearest, ties to even
    B2 v;
    v.x = static_cast<__bf16>(lo);
    v.y = static_cast<__bf16>(hi);
    return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    H2 v;
    v.x = static_cast<_Float16>(lo);
    v.y = static_cast<_Float16>(hi);
    return __builtin_bit_cast(uint32_t, v);
}

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(Bf16 v) { return bf16_to_f32(v.bits); }
__device__ __forceinline__ float to_f32(F16 v) { return static_cast<float>(v.value); }
__device__ __forceinline__ void from_f32(float x, float *p) { *p = x; }
__device__ __forceinline__ void from_f32(float x, Bf16 *p) { p->bits = static_cast<uint16_t>(pack_bf16(x, 0.f)); }
__device__ __forceinline__ void from_f32(float x, F16 *p) { p->value = static_cast<_Float16>(x); }

// What an octet holds between its load and its use: four dwords, or eight floats.
template <typename T> struct Raw {
    U4 w[sizeof(T) == 4 ? 2 : 1];
};
template <typename T> __device__ __forceinline__ Raw<T> load_octet(const T *p) {
    Raw<T> r;
    if constexpr (sizeof(T) == 4) {
        r.w[0] = *reinterpret_cast<const U4a4 *>(p);
        r.w[1] = *reinterpret_cast<const U4a4 *>(p + 4);
    } else {
        r.w[0] = *reinterpret_cast<const U4a2 *>(p);
    }
    return r;
}
typedef uint32_t U2a2 __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t U2a4 __attribute__((ext_vector_type(2), aligned(4)));
typedef uint32_t U1a2 __attribute__((aligned(2)));
// Elements [0, n), 0 < n < 8, zeros behind them: four, two and one at a time.
template <typename T> __device__ __forceinline__ Raw<T> load_some(const T *p, int n) {
    uint32_t d[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    const bool four = (n & 4) != 0;
    Raw<T> r;
    if constexpr (sizeof(T) == 4) {
        if (four) {
            const U4 v = *reinterpret_cast<const U4a4 *>(p);
#pragma unroll
            for (int j = 0; j < 4; ++j) d[j] = v[j];
        }
        if ((n & 2) != 0) {
            const U2 v = *reinterpret_cast<const U2a4 *>(p + (n & 4));
            d[four ? 4 : 0] = v[0];
            d[four ? 5 : 1] = v[1];
        }
        if ((n & 1) != 0) {
            const uint32_t v = reinterpret_cast<const uint32_t *>(p)[n & 6];
#pragma unroll
            for (int j = 0; j < 8; j += 2)
                if ((n & 6) == j) d[j] = v;
        }
        r.w[1] = U4{d[4], d[5], d[6], d[7]};
    } else {
        if (four) {
            const U2 v = *reinterpret_cast<const U2a2 *>(p);
            d[0] = v[0];
            d[1] = v[1];
        }
        if ((n & 2) != 0) d[four ? 2 : 0] = *reinterpret_cast<const U1a2 *>(p + (n & 4));
        if ((n & 1) != 0) {
            const uint32_t v = reinterpret_cast<const uint16_t *>(p)[n & 6];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if ((n & 6) == 2 * j) d[j] = v;
        }
    }
    r.w[0] = U4{d[0], d[1], d[2], d[3]};
    return r;
}
// An octet without its first m elements, 0 < m < 8, zeros behind the rest.
template <typename T> __device__ __forceinline__ Raw<T> without_first(const Raw<T> &r, int m) {
    constexpr int N = sizeof(T) == 4 ? 8 : 4;  // dwords
    uint32_t d[N + 4] = {};
#pragma unroll
    for (int j = 0; j < N; ++j) d[j] = r.w[j / 4][j % 4];
    const int words = sizeof(T) == 4 ? m : m / 2;
#pragma unroll
    for (int step = N / 2; step > 0; step /= 2)
#pragma unroll
        for (int j = 0; j < N; ++j) d[j] = (words & step) != 0 ? (j + step < N ? d[j + step] : 0u) : d[j];
    if constexpr (sizeof(T) == 2) {
        if ((m & 1) != 0)
#pragma unroll
            for (int j = 0; j < N; ++j) d[j] = d[j] >> 16 | d[j + 1] << 16;
    }
    Raw<T> out;
#pragma unroll
    for (int j = 0; j < N; ++j) out.w[j / 4][j % 4] = d[j];
    return out;
}
// Octet of a row of which `left` elements follow from p on (none: zeros).  A row's last octet, where it is not a whole one, is read along with what stands
// before it (`before`: the row has eight elements before p + left), so that all lanes go the same way; settle() puts it right, apart from the load, so
// that loads can be on their way while others are waited for.
template <typename T> __device__ __forceinline__ Raw<T> fetch_row(const T *p, int64_t left, bool before) {
    if (left > 0 && (left >= 8 || before)) return load_octet(left >= 8 ? p : p - (8 - left));
    if (left > 0) return load_some(p, static_cast<int>(left));
    return Raw<T>{};
}
template <typename T> __device__ __forceinline__ Raw<T> settle(const Raw<T> &r, int64_t left, bool before) {
    if (left >= 8 || left <= 0 || !before) return r;
    return without_first(r, 8 - static_cast<int>(left));
}
template <typename T> __device__ __forceinline__ Raw<T> load_row(const T *p, int64_t left, bool before) { return settle(fetch_row(p, left, before), left, before); }
template <typename T> __device__ __forceinline__ void unpack(const Raw<T> &r, float (&v)[8]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (sizeof(T) == 4) {
            v[j] = __uint_as_float(r.w[0][j]);
            v[j + 4] = __uint_as_float(r.w[1][j]);
        } else if constexpr (__is_same(T, Bf16)) {
            v[2 * j] = __uint_as_float(r.w[0][j] << 16);
            v[2 * j + 1] = __uint_as_float(r.w[0][j] & 0xFFFF0000u);
        } else {
            const uint32_t d = r.w[0][j];  // (a bit cast of the element itself takes the first one for each)
            const H2 h = __builtin_bit_cast(H2, d);
            v[2 * j] = static_cast<float>(h.x);
            v[2 * j + 1] = static_cast<float>(h.y);
        }
    }
}
// Rounds to the type, to nearest with ties to even.
template <typename T> __device__ __forceinline__ Raw<T> pack(const float (&v)[8]) {
    Raw<T> r;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (sizeof(T) == 4) {
            r.w[0][j] = __float_as_uint(v[j]);
            r.w[1][j] = __float_as_uint(v[j + 4]);
        } else if constexpr (__is_same(T, Bf16)) {
            r.w[0][j] = pack_bf16(v[2 * j], v[2 * j + 1]);
        } else {
            r.w[0][j] = pack_f16(v[2 * j], v[2 * j + 1]);
        }
    }
    return r;
}
// The first `left` of an octet's elements (all of them, or none).
template <typename T> __device__ __forceinline__ void store_row(T *p, int64_t left, const Raw<T> &r) {
    if (left >= 8) {
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<U4a4 *>(p) = r.w[0];
            *reinterpret_cast<U4a4 *>(p + 4) = r.w[1];
        } else {
            *reinterpret_cast<U4a2 *>(p) = r.w[0];
        }
        return;
    }
    if (left <= 0) return;
    const int n = static_cast<int>(left);
    const bool four = (n & 4) != 0;
    if constexpr (sizeof(T) == 4) {
        if (four) *reinterpret_cast<U4a4 *>(p) = r.w[0];
        if ((n & 2) != 0) *reinterpret_cast<U2a4 *>(p + (n & 4)) = four ? U2{r.w[1][0], r.w[1][1]} : U2{r.w[0][0], r.w[0][1]};
        if ((n & 1) != 0) {
            const uint32_t low = (n & 2) != 0 ? r.w[0][2] : r.w[0][0], high = (n & 2) != 0 ? r.w[1][2] : r.w[1][0];
            reinterpret_cast<uint32_t *>(p)[n & 6] = four ? high : low;
        }
    } else {
        if (four) *reinterpret_cast<U2a2 *>(p) = U2{r.w[0][0], r.w[0][1]};
        if ((n & 2) != 0) *reinterpret_cast<U1a2 *>(p + (n & 4)) = four ? r.w[0][2] : r.w[0][0];
        if ((n & 1) != 0) {
            const uint32_t low = (n & 2) != 0 ? r.w[0][1] : r.w[0][0], high = (n & 2) != 0 ? r.w[0][3] : r.w[0][2];
            reinterpret_cast<uint16_t *>(p)[n & 6] = static_cast<uint16_t>(four ? high : low);
        }
    }
}

// ---- the 8-bit form.  E: the exponent field of the group's largest magnitude, at least 7 so that the step 2^(E - 133) and its inverse are
// normal numbers; 255 where the group holds a NaN or an infinity.  x / step is exact (or far below a half), so a number is one rounding of the
// value, whatever the machine; clamping +-128 to +-127 keeps number * step finite in every type and the error within amax / 127.5
// (within 2^-127 where the step is held at 2^-126).
__device__ __forceinline__ uint32_t max_of_quad(uint32_t v) {
    // (quad_perm [1,0,3,2] and [2,3,0,1]: all four lanes take part, so callers keep whole quads active)
    uint32_t o = static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0xB1, 0xF, 0xF, false));
    v = v > o ? v : o;
    o = static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0x4E, 0xF, 0xF, false));
    return v > o ? v : o;
}
__device__ __forceinline__ uint32_t group_exponent(const float (&v)[8]) {
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t k = __float_as_uint(v[j]) & 0x7FFFFFFFu;
        m = m > k ? m : k;
    }
    const uint32_t e = max_of_quad(m) >> 23;
    return e > 7 ? e : 7;
}
__device__ __forceinline__ U2 numbers(const float (&v)[8], uint32_t E) {
    const float inverse = __uint_as_float((260u - E) << 23);
    uint32_t d[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t b[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float q = __builtin_rintf(v[4 * h + j] * inverse);
            q = __builtin_amdgcn_fmed3f(q, -127.f, 127.f);
            b[j] = static_cast<uint32_t>(static_cast<int32_t>(q));
        }
        d[h] = (b[0] & 0xFFu) | (b[1] & 0xFFu) << 8 | (b[2] & 0xFFu) << 16 | b[3] << 24;
    }
    return E == 255 ? U2{0, 0} : U2{d[0], d[1]};  // (a marked group's numbers say nothing, and a padding behind a row that is no number stays one of zeros)
}
__device__ __forceinline__ float step_of(uint32_t E) { return E == 255 ? __uint_as_float(0x7FC00000u) : __uint_as_float((E > 7 ? E - 6 : 1) << 23); }
__device__ __forceinline__ void values_of(U2 d, uint32_t E, float (&v)[8]) {
    const float step = step_of(E);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < 4; ++j) v[4 * h + j] = static_cast<float>(static_cast<int8_t>(d[h] >> (8 * j))) * step;
}
// Puts a lane's octet of a row away; all four lanes of a quad take part.  `octet`: its place in the row.  Octets behind the pitch are not stored.
__device__ __forceinline__ void act8_put(const Act8 &a, int64_t row, int octet, const float (&v)[8]) {
    const uint32_t E = group_exponent(v);
    const U2 d = numbers(v, E);
    const int64_t at = static_cast<int64_t>(octet) * 8;
    if (at < a.pitch) {
        *reinterpret_cast<U2 *>(a.q + row * a.pitch + at) = d;
        if ((octet & 3) == 0) a.e[row * (a.pitch / GROUP) + octet / 4] = static_cast<uint8_t>(E);
    }
}
__device__ __forceinline__ void act8_get(const Act8 &a, int64_t row, int octet, U2 &d, uint32_t &E) {
    const int64_t at = static_cast<int64_t>(octet) * 8;
    if (at < a.pitch) {
        d = *reinterpret_cast<const U2 *>(a.q + row * a.pitch + at);
        E = a.e[row * (a.pitch / GROUP) + octet / 4];
    } else {
        d = U2{0, 0};
        E = 7;
    }
}

// A value of another lane, zero where `rows` takes none; 64-bit ones in halves.
template <int CONTROL, int ROWS, bool ZERO> __device__ __forceinline__ float moved(float v) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CONTROL, ROWS, 0xF, ZERO));
}
template <int CONTROL, int ROWS, bool ZERO> __device__ __forceinline__ double moved(double v) {
    return __hiloint2double(__builtin_amdgcn_update_dpp(0, __double2hiint(v), CONTROL, ROWS, 0xF, ZERO),
                            __builtin_amdgcn_update_dpp(0, __double2loint(v), CONTROL, ROWS, 0xF, ZERO));
}
__device__ __forceinline__ float from_lane(float v, int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane)); }
__device__ __forceinline__ double from_lane(double v, int lane) {
    return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), lane), __builtin_amdgcn_readlane(__double2loint(v), lane));
}

// Sum over the 64 lanes, in a fixed order, as a scalar.  Moves within a row of 16 lanes and from row to row ride on the additions: a tenth of the
// latency of exchanges through LDS.
template <typename V> __device__ __forceinline__ V wave_sum(V v) {
    v += moved<0x111, 0xF, true>(v);  // row_shr 1, 2, 4, 8: a row's last lane has its sum
    v += moved<0x112, 0xF, true>(v);
    v += moved<0x114, 0xF, true>(v);
    v += moved<0x118, 0xF, true>(v);
    v += moved<0x142, 0xA, true>(v);  // row_bcast 15: into rows 1 and 3
    v += moved<0x143, 0xC, true>(v);  // row_bcast 31: into rows 2 and 3
    return from_lane(v, 63);
}

// Division of a 32-bit number by one that a launch fixes: one multiplication and a shift (Granlund and Montgomery's round-up form, n < 2^31).
struct Divisor {
    uint32_t d, multiplier, shift;
    explicit Divisor(uint32_t by) : d(by), multiplier(0), shift(0) {
        if (by <= 1) return;
        while ((static_cast<uint64_t>(1) << shift) < by) ++shift;
        --shift;
        multiplier = static_cast<uint32_t>(((static_cast<uint64_t>(1) << (32 + shift)) + by - 1) / by);
    }
    __device__ __forceinline__ uint32_t quotient(uint32_t n) const { return d <= 1 ? n : __umulhi(n, multiplier) >> shift; }
};
inline adatopk_status launched() { return hipGetLastError() == hipSuccess ? ADATOPK_OK : ADATOPK_ERUNTIME; }

// Rows of a dense matrix: `stride` elements from one to the next.
inline bool matrix_ok(const void *p, int64_t stride, int64_t rows, int64_t cols, adatopk_dtype dt) {
    return pointer_ok(p, static_cast<size_t>(elem_size(dt))) && (stride >= cols || rows <= 1) && stride >= 0;
}

// Calls f with a null pointer of the element type.
template <typename F> inline void with_type(adatopk_dtype dt, F &&f) {
    if (dt == ADATOPK_F32)
        f(static_cast<float *>(nullptr));
    else if (dt == ADATOPK_BF16)
        f(static_cast<Bf16 *>(nullptr));
    else
        f(static_cast<F16 *>(nullptr));
}
#endif  // __HIPCC__

}  // namespace adatopk_stage
#endif
