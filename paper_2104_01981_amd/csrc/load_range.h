// What a load of an operand's tile may reach (products.h).
//
// A lane's bytes are read if their offset lies below `end` - `from`, where `end` is the size in the buffer's descriptor, from the tile's first
// row or column on, and `from` the offset that all lanes have in common; the others get zeros.  The difference is one of 32 bits: with
// `from` beyond `end` it could come round to nearly 2^32, and every lane would read.  So `from` is never larger than `end`.
#pragma once

#include "host_device.h"

namespace ecrm {

constexpr uint32_t kOutside = 0x7FFFFFFFu;       // an offset behind any operand's end

// Rows along K, `stride` bytes apart, `width` bytes of each: the operand has `count`, the tile up to `tile` from `first` on.
ECRM_HD uint32_t rows_end(uint32_t count, uint32_t first, uint32_t tile, uint32_t stride, uint32_t width)
{
    const uint32_t left = count > first ? count - first : 0u, rows = left < tile ? left : tile;
    return rows ? (rows - 1u) * stride + width : 0u;
}
// `at`: bytes of K before the load's, fewer than `width`.  Of no rows at all (the later half of kGate's columns, behind the last) nothing is read.
ECRM_HD uint32_t rows_from(uint32_t end, uint32_t at) { return end ? at : 0u; }

// Rows across K, `width` bytes of each from the tile's first column on (0: the tile lies behind the last), `rows` of K, with `from` = 0.
ECRM_HD uint32_t columns_end(uint32_t rows, uint32_t stride, uint32_t width) { return width ? (rows - 1u) * stride + width : 0u; }

}  // namespace ecrm
