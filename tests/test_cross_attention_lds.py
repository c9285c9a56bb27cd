"""The LDS of cross attention's launches holds every byte that their kernels read: column operands come in blocks of 32, so heads of 65 to 80 values are read up to
the 96th.  Compiled for the host alone, from the library's own header."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = r"""
#include <cstdio>
#include "cross_attn.h"
using namespace freemi;
// behind the last byte of a tile of 64 rows of `chunks` chunks of 16 bytes that is read by columns, from the formulas of the layout
template <int DP>
int columns_end() {
    using TL = Tile<bf16_t, DP>;
    int end = 0;
    for (int row = 0; row < 64; ++row)
        for (int c = 0; c < (DP + 31) / 32 * 4; ++c) end = TL::at(row, c) + 16 > end ? TL::at(row, c) + 16 : end;
    return end;
}
template <int DP, int NW>
int holds(const char* what, int tiles, size_t lds, size_t most) {
    using Ring = PairRing<DP, NW>;
    const size_t read = static_cast<size_t>(tiles - 1) * Ring::kTileBytes + Ring::kSecond + columns_end<DP>();
    if (read <= lds && lds <= most) return 0;
    std::printf("heads of %d, %s: %d tiles, %zu bytes of LDS of at most %zu, read up to %zu\n", DP, what, tiles, lds, most, read);
    return 1;
}
template <int DP>
int check() {
    // (128 bytes of masks; two workgroups to a compute unit where tiles pass through)
    int bad = holds<DP, kPassWaves>("pass through", kPassTiles<DP>, ring_bytes<DP, kPassWaves>(kPassTiles<DP>), 80 * 1024 - 128);
    for (int tiles = 1; tiles <= tiles_that_fit(DP); ++tiles) bad += holds<DP, kRingWaves>("stay", tiles, ring_bytes<DP, kRingWaves>(tiles), 160 * 1024 - 128);
    return bad;
}
int main() { return check<32>() + check<64>() + check<80>() + check<96>() + check<128>(); }
"""


def test_columns_are_inside(tmp_path):
    src, exe = tmp_path / "lds.hip", tmp_path / "lds"
    src.write_text(PROGRAM)
    subprocess.run(["hipcc", "-std=c++17", "--offload-arch=gfx950", "--offload-host-only", "-I" + os.path.join(ROOT, "paper_2511_20390_amd", "csrc"), str(src), "-o",
                    str(exe)], check=True)
    done = subprocess.run([str(exe)], timeout=60, capture_output=True, text=True)
    assert done.returncode == 0, done.stdout


def test_launches_take_their_size_from_there():
    csrc = os.path.join(ROOT, "paper_2511_20390_amd", "csrc")
    for name in ("cross_attn.hip", "cross_attn_grad.hip"):
        text = open(os.path.join(csrc, name)).read()
        assert "ring_bytes<DP, kPassWaves>(kPassTiles<DP>)" in text and "kPassTiles<DP> *" not in text, name
