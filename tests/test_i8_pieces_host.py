"""Where the kernel for 8-bit products of any size reads a row (csrc/i8_pieces.hiph), compiled for the host: every piece of
every row of 1 to 300 columns, and of some up to the largest, is read within the row."""
import os
import subprocess

import paper_2403_17017_amd as S

DRIVER = r"""
#include "i8_pieces.hiph"
#include <cstdio>
#include <initializer_list>

int main()
{
    long bad = 0, seen = 0;
    const auto row = [&](uint32_t columns) {
        for (uint32_t k0 = 0; k0 < columns; k0 += 128) {
            uint32_t kept = 0;
            for (uint32_t col = 0; col < 128; col += 16, ++seen) {
                const seer::RowPiece p = seer::row_piece(k0, col, columns);
                // at least a column and at most 16, all of them the row's
                if (p.have < 1 || p.have > 16 || (uint64_t)p.from + p.have > columns) ++bad;
                // what is kept is where it belongs, and the row is covered
                if (p.keep > 0 && (p.from != k0 + col || p.keep > p.have)) ++bad;
                kept += p.keep > 0 ? p.keep : 0;
            }
            if (kept != (columns - k0 < 128 ? columns - k0 : 128)) ++bad;
        }
    };
    for (uint32_t columns = 1; columns <= 300; ++columns) row(columns);
    for (uint32_t columns : {4095u, 4111u, 131071u}) row(columns);
    std::printf("%ld of %ld\n", bad, seen);
    return bad != 0;
}
"""


def test_every_piece_is_read_within_its_row(tmp_path):
    (tmp_path / "driver.cpp").write_text(DRIVER)
    csrc = os.path.join(os.path.dirname(os.path.abspath(S.__file__)), "csrc")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-x", "c++", "-I", csrc, "-o", str(tmp_path / "driver"), str(tmp_path / "driver.cpp")])
    out = subprocess.run([str(tmp_path / "driver")], capture_output=True, text=True, timeout=120)
    assert out.returncode == 0, out.stdout
