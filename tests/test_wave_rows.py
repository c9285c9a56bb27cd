"""The rows of cross attention's wavefronts: each row of a (sample, key head) has one lane, and a lane without a row is past the last one, whatever the number of
rows.  Host only: the library's own header, compiled here."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = r"""
#include <cstdio>
#include <initializer_list>
#include "wave_rows.h"
using namespace freemi;
int main() {
    const long long most = 32 * ((1ll << 23) - 1);                // what the checks of sizes allow
    for (long long about : {64ll, 4096ll, 1ll << 26, 1ll << 27, most})
        for (long long rows = about - 300; rows <= about + 300 && rows <= most; ++rows) {
            if (rows < 1) continue;
            for (int waves : {4, 8}) {
                const long long blocks = (rows + 31) / 32, groups = (blocks + waves - 1) / waves;
                long long next = (groups - 1) * waves * 32;       // the last workgroup's rows, one after the other
                for (int wave = 0; wave < waves; ++wave)
                    for (int lane = 0; lane < 32; ++lane, ++next) {
                        const int32_t row = lane_row(wave_block(static_cast<int32_t>(groups - 1), waves, wave), lane);
                        if (row != next || (row < rows) != (next < rows)) {
                            std::printf("%lld rows, %d wavefronts: wavefront %d, lane %d has row %d\n", rows, waves, wave, lane, row);
                            return 1;
                        }
                    }
            }
        }
    return 0;
}
"""


def test_rows_of_the_last_workgroup(tmp_path):
    src, exe = tmp_path / "rows.cpp", tmp_path / "rows"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-I" + os.path.join(ROOT, "paper_2511_20390_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    done = subprocess.run([str(exe)], timeout=60, capture_output=True, text=True)
    assert done.returncode == 0, done.stdout


def test_results_are_stored_by_these_rows():
    """A wavefront's block is its own number from there, also where it has none of the rows."""
    text = open(os.path.join(ROOT, "paper_2511_20390_amd", "csrc", "cross_attn.hip")).read()
    ring = text.split("void cross_ring_kernel", 1)[1].split("\n}\n", 1)[0]
    assert "const int r = lane_row(block, l32);" in ring.split("const auto finish", 1)[1]
    tail = ring.split("} else {", 1)[1]
    assert "const int block = wave_block(chunk, NW, wave);" in tail and "finish(block, any);" in tail
