"""Arithmetic of the tile engine (csrc/lmkan_tile.h), compiled for the host."""
import os
import subprocess

from paper_2509_07103_amd import build

PROGRAM = r"""
#include <stdio.h>
#include "lmkan_tile.h"
using namespace lmkan;

// every lane of every load of a tile of N rows: its own line where that exists, else the last bytes of the last one
template <int N>
static int wrong(int64_t last)
{
    int bad = 0;
    for (int r0 = 0; r0 < N; r0 += 8)
        for (int lane = 0; lane < 64; ++lane) {
            const int64_t own = (int64_t)r0 * kLine + lane * 16, end = last * kLine + kLine - 16;
            bad += panel_offset<N>((int)last, r0, lane) != (own < end ? own : end);
        }
    return bad;
}

int main()
{
    int bad = 0;
    const int64_t around[] = {0, 1, 62, 63, 64, 127, 128, 255, 256, 1000, (1 << 24) - 1, 1 << 24, (1 << 26) - 1};
    for (const int64_t last : around) bad += wrong<64>(last) + wrong<128>(last) + wrong<256>(last);
    // a panel of 2^32 bytes and a few lines more
    for (int64_t last = (1 << 25) - 300; last < (1 << 25) + 300; ++last) {
        const int now = wrong<64>(last) + wrong<128>(last) + wrong<256>(last);
        if (now && !bad) printf("first wrong: last row %ld, %d lanes\n", (long)last, now);
        bad += now;
    }
    printf("%d wrong\n", bad);
    return bad != 0;
}
"""


def test_lines_of_a_panel_of_more_than_4_gib(tmp_path):
    source, program = tmp_path / "panel.hip", tmp_path / "panel"
    source.write_text(PROGRAM)
    subprocess.run([build.HIPCC, "--offload-arch=gfx950", "-O1", "-std=c++17", "-I", build.CSRC, "-o", str(program), str(source)],
                   check=True, capture_output=True)
    got = subprocess.run([str(program)], capture_output=True, text=True)
    assert got.returncode == 0, got.stdout
