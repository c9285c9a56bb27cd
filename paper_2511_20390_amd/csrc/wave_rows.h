// Which row a lane of a wavefront has where wavefronts have blocks of 32 rows.  Plain arithmetic, for the device and for the tests on the host.
#pragma once

#include <cstdint>

namespace freemi {

// Rows of a (sample, key head) are below 2^28 (blocks of 32 below 2^23, and 32 more for the last one), so no block of the last workgroup has a number
// that 32 bits do not hold: a wavefront past the last block has rows past the last row, and no other mark.
constexpr int32_t kBlockRows = 32;
constexpr int32_t wave_block(int32_t group, int32_t waves, int32_t wave) { return group * waves + wave; }
constexpr int32_t lane_row(int32_t block, int32_t lane) { return block * kBlockRows + lane; }

}  // namespace freemi
