"""What the attention kernels' copies to LDS reach, from the same header that the
kernels take it from (no GPU needed)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# For every head width: the last byte of a key that an unchecked copy reads.  A
# key's row is copied in 16-byte chunks, in an order that permutes the whole row.
PROGRAM = r"""
#include <cstdio>
#include "kv_view.h"
int main() {
  for (int D = 8; D <= 128; D += 8) {
    const int slices = brisk::head_slices(D), row = brisk::lds_row_bytes(slices);
    const int end = brisk::head_fills_row(D, slices) ? row / 16 * 16 : 2 * D;
    std::printf("%d %d %d %d\n", D, slices, row, end);
  }
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs a host compiler")
def test_copies_end_with_the_head(tmp_path):
    (tmp_path / "layout.cpp").write_text(PROGRAM)
    exe = str(tmp_path / "layout")
    subprocess.run(["g++", "-std=c++17", "-I", os.path.join(ROOT, "paper_2609_33390_amd", "csrc"), str(tmp_path / "layout.cpp"),
                    "-o", exe], check=True)
    rows = [tuple(map(int, line.split())) for line in subprocess.run([exe], check=True, capture_output=True,
                                                                     text=True).stdout.splitlines()]
    assert [r[0] for r in rows] == list(range(8, 129, 8))
    for D, slices, row, end in rows:
        assert 32 * (slices - 1) < D <= 32 * slices or (slices == 2 and D <= 64)
        assert 2 * D <= row
        assert end == 2 * D, f"a copy of a {D}-wide key reads {end - 2 * D} bytes past it"
