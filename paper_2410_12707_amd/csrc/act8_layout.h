// Byte arithmetic of an activation kept in 8 bits, shared by the host-only helpers and the kernels' launch code: numbers [rows][pitch], a row
// padded to whole groups, then from the next multiple of 256 bytes on the groups' exponents [rows][pitch / 32].  Internal to the library.
#ifndef ADATOPK_ACT8_LAYOUT_H
#define ADATOPK_ACT8_LAYOUT_H

#include <stddef.h>
#include <stdint.h>

#include "wire_layout.h"

namespace adatopk_internal {

constexpr int64_t ACT8_GROUP = 32;
constexpr int64_t ACT8_MAX_OCTETS = static_cast<int64_t>(1) << 31;  // the kernels count octets of elements in 32 bits: 16 Gi elements

inline int64_t act8_pitch(int64_t cols) { return (cols + ACT8_GROUP - 1) / ACT8_GROUP * ACT8_GROUP; }
inline bool act8_shape_ok(int64_t rows, int64_t cols) {
    if (rows < 0 || cols < 0 || cols >= (static_cast<int64_t>(1) << 31) - ACT8_GROUP) return false;
    return cols == 0 || rows < ACT8_MAX_OCTETS / (act8_pitch(cols) / 8);
}
inline size_t act8_exponents_at(int64_t rows, int64_t cols) { return align_up(static_cast<size_t>(rows) * static_cast<size_t>(act8_pitch(cols)), 256); }

}  // namespace adatopk_internal
#endif
