// Ranges of buffer descriptors: what a load may touch.  Plain arithmetic, for the device and for the tests on the host.
#pragma once

#include <cstdint>

namespace freemi {

// The descriptor's range for `bytes` bytes from its base on; loads behind it give zeros.  A base at or past the end has none: a number
// below zero would be a range of 4 GB.  By halves: the scalar unit has no order of 64-bit numbers, and the K loops make ranges.
constexpr uint32_t range_bytes(int64_t bytes) {
    const int32_t high = static_cast<int32_t>(bytes >> 32);
    const uint32_t low = static_cast<uint32_t>(bytes), most = 0x7fffffff;
    const uint32_t range = high > 0 || low > most ? most : low;
    return high < 0 ? 0 : range;
}

// The weight rows of [gate | up], N rows each, that a wavefront of eight loads for a tile whose first hidden value is n0: wavefronts 0 to 3
// the gate rows n0 + 8 wave + 32 j + 0 .. 7, 4 to 7 the up rows likewise.  The range ends with the wavefront's own matrix, so hidden values
// past N have zeros for both; where N - n0 is 8 or 16 the last wavefronts have no row at all.
struct RowRange {
    int32_t first, count;
};
constexpr RowRange gated_rows(int wave, int32_t N, int32_t n0) {
    const int32_t end = wave < 4 ? N : 2 * N, first = end - N + n0 + (wave & 3) * 8;
    return first < end ? RowRange{first, end - first} : RowRange{end, 0};
}

}  // namespace freemi
