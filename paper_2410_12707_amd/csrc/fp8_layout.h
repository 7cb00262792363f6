// Byte arithmetic of a matrix in 8-bit floating point, shared by the host-only helpers and the kernels' launch code: numbers [rows][pitch], a row padded
// to whole blocks of 128, then from the next multiple of 256 bytes on the blocks' scales [pitch / 128][rows padded to 256].  Internal to the library.
//
// The scales of a block's column lie side by side: a product's tile takes those of its rows in one load, and the padding keeps that load inside the buffer.
#ifndef ADATOPK_FP8_LAYOUT_H
#define ADATOPK_FP8_LAYOUT_H

#include <stddef.h>
#include <stdint.h>

#include "wire_layout.h"

namespace adatopk_internal {

constexpr int64_t FP8_BLOCK = 128, FP8_ROWS = 256;
constexpr int64_t FP8_MAX_OCTETS = static_cast<int64_t>(1) << 31;  // the kernels count octets of elements in 32 bits: 16 Gi elements

inline int64_t fp8_pitch(int64_t cols) { return (cols + FP8_BLOCK - 1) / FP8_BLOCK * FP8_BLOCK; }
inline int64_t fp8_scale_pitch(int64_t rows) { return (rows + FP8_ROWS - 1) / FP8_ROWS * FP8_ROWS; }
inline bool fp8_shape_ok(int64_t rows, int64_t cols) {
    if (rows < 0 || cols < 0 || cols >= (static_cast<int64_t>(1) << 31) - FP8_BLOCK) return false;
    return cols == 0 || rows < FP8_MAX_OCTETS / (fp8_pitch(cols) / 8);
}
inline size_t fp8_scales_at(int64_t rows, int64_t cols) { return align_up(static_cast<size_t>(rows) * static_cast<size_t>(fp8_pitch(cols)), 256); }
inline size_t fp8_bytes(int64_t rows, int64_t cols) {
    if (rows == 0 || cols == 0) return 0;
    return fp8_scales_at(rows, cols) + static_cast<size_t>(fp8_pitch(cols) / FP8_BLOCK) * static_cast<size_t>(fp8_scale_pitch(rows));
}

}  // namespace adatopk_internal
#endif
