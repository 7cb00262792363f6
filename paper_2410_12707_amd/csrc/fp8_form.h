// The 8-bit floating-point form in the kernels: 128 consecutive elements of a row share a power of two.  Internal to the library.
//
// S: with m the block's largest magnitude, the smallest scale 2^(S - 127) that has m <= 448 * scale (448 = 1.75 * 2^8 is the largest number of four
// significand bits, exponents to 8), so nothing is clamped; at least 1, so that scale and inverse are normal numbers and x / scale is exact (or
// far below the smallest number's half); 255 for a block with a NaN or an infinity, whose numbers are all NaN.  The matrix instruction takes S as it is.
#ifndef ADATOPK_FP8_FORM_H
#define ADATOPK_FP8_FORM_H

#include "fp8_layout.h"
#include "stage_ops.h"

namespace adatopk_stage {

struct Fp8 {
    uint8_t *q, *s;
    int64_t pitch, scale_pitch;
};
inline Fp8 fp8_of(void *buffer, int64_t rows, int64_t cols) {
    uint8_t *q = static_cast<uint8_t *>(buffer);
    return Fp8{q, q == nullptr ? nullptr : q + adatopk_internal::fp8_scales_at(rows, cols), adatopk_internal::fp8_pitch(cols), adatopk_internal::fp8_scale_pitch(rows)};
}
inline bool fp8_shape_ok(int64_t rows, int64_t cols) { return adatopk_internal::fp8_shape_ok(rows, cols); }

#if defined(__HIPCC__)
constexpr int BLOCK_OCTETS = static_cast<int>(adatopk_internal::FP8_BLOCK / 8);

// The largest of sixteen neighbouring lanes' values, in each of them.  All sixteen take part.
__device__ __forceinline__ uint32_t max_of_sixteen(uint32_t v) {
    v = max_of_quad(v);
    uint32_t o = static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0x141, 0xF, 0xF, false));  // the other quad of eight lanes
    v = v > o ? v : o;
    o = static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0x140, 0xF, 0xF, false));  // the other half of sixteen
    return v > o ? v : o;
}
__device__ __forceinline__ uint32_t largest_magnitude(const float (&v)[8]) {
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t k = __float_as_uint(v[j]) & 0x7FFFFFFFu;
        m = m > k ? m : k;
    }
    return m;
}
// S of a block from the bits of its largest magnitude: adding 0x1FFFFF carries into the exponent where the significand is above 1.75.
__device__ __forceinline__ uint32_t fp8_scale(uint32_t most) {
    if (most >= 0x7F800000u) return 255;
    const uint32_t e = (most + 0x1FFFFFu) >> 23;
    return e > 9 ? e - 8 : 1;
}
// Eight numbers, to nearest with ties to even.
__device__ __forceinline__ U2 fp8_numbers(const float (&v)[8], uint32_t S) {
    if (S == 255) return U2{0x7F7F7F7Fu, 0x7F7F7F7Fu};
    const float inverse = __uint_as_float((254u - S) << 23);
    int d[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        d[h] = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h] * inverse, v[4 * h + 1] * inverse, 0, false);
        d[h] = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h + 2] * inverse, v[4 * h + 3] * inverse, d[h], true);
    }
    return U2{static_cast<uint32_t>(d[0]), static_cast<uint32_t>(d[1])};
}
__device__ __forceinline__ void fp8_values(U2 d, uint32_t S, float (&v)[8]) {
    typedef float F2 __attribute__((ext_vector_type(2)));
    const float scale = __uint_as_float((S < 254 ? S : 254) << 23);  // (a marked block's numbers are NaN)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const F2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(d[h]), false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(d[h]), true);
        v[4 * h] = lo.x * scale;
        v[4 * h + 1] = lo.y * scale;
        v[4 * h + 2] = hi.x * scale;
        v[4 * h + 3] = hi.y * scale;
    }
}
// Puts a lane's octet of a row away; all sixteen lanes of a block take part.  `octet`: its place in the row.  Octets behind the pitch are not stored.
__device__ __forceinline__ void fp8_put(const Fp8 &a, int64_t row, int octet, const float (&v)[8]) {
    const uint32_t S = fp8_scale(max_of_sixteen(largest_magnitude(v)));
    const U2 d = fp8_numbers(v, S);
    const int64_t at = static_cast<int64_t>(octet) * 8;
    if (at < a.pitch) {
        *reinterpret_cast<U2 *>(a.q + row * a.pitch + at) = d;
        if (octet % BLOCK_OCTETS == 0) a.s[octet / BLOCK_OCTETS * a.scale_pitch + row] = static_cast<uint8_t>(S);
    }
}
#endif  // __HIPCC__

}  // namespace adatopk_stage
#endif
