// Arithmetic of what a stage of a product's loads may reach of an operand, the same on host and device (k_gemm.h).
#pragma once
#include <cstdint>

namespace kimad {

// Bytes from a stage's first element on, beyond which loads give zeros.  Along K: `lines` rows of `count` elements of K.  Across: `lines` rows of K of `count` elements, in
// whole words, for a load gives whole words (half of the last one may be beyond the array, never of another page).
constexpr uint32_t stage_bytes(bool across, uint32_t lines, uint32_t count, uint32_t ld_bytes) {
    const uint32_t line = across ? (2 * count + 3) & ~3u : 2 * count;
    return ((lines - 1) * ld_bytes + line) & (lines == 0 || line == 0 ? 0u : ~0u);
}
// Elements from row to row as the loads take them, of an operand whose rows begin at 16-byte addresses.  A row alone may be given with any distance to the next: an odd one would
// put the row behind it, which is none, into the last word of this one.
constexpr uint64_t pitch_of(uint64_t cols) { return (cols + 7) / 8 * 8; }
constexpr uint64_t stage_ld(uint64_t rows, uint64_t cols, uint64_t ld) { return rows > 1 ? ld : pitch_of(cols); }

}  // namespace kimad
