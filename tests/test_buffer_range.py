"""What the loads of the gated feed-forward block's weights may touch: every row a tile needs, and no byte outside of its own matrix,
whatever is left of the hidden values in the last tile.  Host only: the library's own header, compiled here."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = r"""
#include <cstdio>
#include <initializer_list>
#include "buffer_range.h"
using namespace freemi;
int main() {
    if (range_bytes(-1) || range_bytes(-16) || range_bytes(-(1ll << 40)) || range_bytes(0)) return 1;
    if (range_bytes(16) != 16 || range_bytes(0x7fffffff) != 0x7fffffff || range_bytes(1ll << 40) != 0x7fffffff) return 2;
    for (int N = 8; N <= 2048; N += 8)
        for (int cols : {64, 128})                              // hidden values of a tile: 128 or 256 rows of [gate | up]
            for (int n0 = 0; n0 < (N + 63) / 64 * 64; n0 += cols)
                for (int wave = 0; wave < 8; ++wave) {
                    const RowRange r = gated_rows(wave, N, n0);
                    const int begin = wave < 4 ? 0 : N, end = begin + N;
                    if (r.count < 0 || r.first < begin || r.first + r.count > end) {
                        std::printf("N %d n0 %d wave %d: rows %d + %d of %d .. %d\n", N, n0, wave, r.first, r.count, begin, end);
                        return 3;
                    }
                    for (int j = 0; j < cols / 32; ++j)
                        for (int i = 0; i < 8; ++i) {           // row 32 j + i behind the first: read where the range holds it
                            const int hidden = n0 + 32 * j + 8 * (wave & 3) + i;
                            const bool read = 32 * j + i < r.count;
                            if (read != (hidden < N) || (read && r.first + 32 * j + i != begin + hidden)) {
                                std::printf("N %d n0 %d wave %d: hidden value %d\n", N, n0, wave, hidden);
                                return 4;
                            }
                        }
                }
    // the largest matrices: no overflow
    const RowRange r = gated_rows(7, 1 << 20, (1 << 20) - 64);
    return r.first == (2 << 20) - 64 + 24 && r.count == 40 ? 0 : 5;
}
"""


def test_gated_rows(tmp_path):
    src, exe = tmp_path / "range.cpp", tmp_path / "range"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-I" + os.path.join(ROOT, "paper_2511_20390_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    done = subprocess.run([str(exe)], timeout=60, capture_output=True, text=True)
    assert done.returncode == 0, done.stdout


def test_descriptors_take_their_range_from_there():
    """The arithmetic that is tested is the one that is compiled."""
    csrc = os.path.join(ROOT, "paper_2511_20390_amd", "csrc")
    text = lambda name: open(os.path.join(csrc, name)).read()
    assert "range_bytes(bytes)" in text("gemm_dma.h").split("make_rsrc", 1)[1].split("}\n", 1)[0]
    assert "gated_rows(wave, a.N, n0)" in text("ffn_mfma.hip")
