"""CPU checks of the 8-bit layer's rows in LDS: the header that the kernel and its launch share, compiled
for the host.  Whatever ids a caller passes, the rows that a block takes at a time fit its LDS."""

import os
import shutil
import subprocess

import pytest

from paper_2203_14685_amd import build as b

PROGRAM = r"""
#include <cstdio>
#include "layer_int8_rows.hpp"
using namespace hetumoe;
int main() {
  long held = 0, more = 0;
  for (int S = 1; S <= 64; ++S)
    for (int k = 1; k <= 8; ++k)
      for (int by_choice = 0; by_choice < 2; ++by_choice)
        for (int K = 16; K <= kInt8HeldK + 512; K += 16)
          for (int z = 1; z <= 8; ++z) {
            if (!layer_int8_held(S, k, by_choice, K, z)) continue;
            ++held;
            const int bytes = layer_int8_row_bytes(K, z), rows = layer_int8_held_rows(bytes);
            // all of K in the blocks' ranges, all choices of one expert in some number of passes
            if (S * k > 64 || K > kInt8HeldK || bytes * z < K || rows < 1 || rows > kInt8HeldRows || rows * bytes > kInt8HeldBytes) {
              std::printf("S=%d k=%d K=%d z=%d: %d rows of %d bytes\n", S, k, K, z, rows, bytes);
              return 1;
            }
            // rows that a block would hold if only S bounded them, with every id the same
            const int named = S * k < kInt8HeldRows ? S * k : kInt8HeldRows;
            more += named * bytes > kInt8HeldBytes;
          }
  std::printf("%ld %ld\n", held, more);
  // calls whose rows are as many as fit: more choices than that take further passes
  return layer_int8_held(1, 2, true, 8192, 1) && layer_int8_held_rows(layer_int8_row_bytes(8192, 1)) == 1 &&
         layer_int8_held(1, 8, true, 4096, 1) && layer_int8_held_rows(layer_int8_row_bytes(4096, 1)) == 3 &&
         layer_int8_held(2, 2, true, 6144, 1) && layer_int8_held_rows(layer_int8_row_bytes(6144, 1)) == 2 &&
         !layer_int8_held(4, 1, true, 4096, 1) && !layer_int8_held(1, 1, true, 8208, 1) ? 0 : 2;
}
"""


def test_rows_of_a_pass_fit_their_room(tmp_path):
    cc = shutil.which("g++") or shutil.which("clang++") or b.hipcc()
    src, exe = tmp_path / "rows.cpp", tmp_path / "rows"
    src.write_text(PROGRAM)
    subprocess.run([cc, "-std=c++17", "-O2", "-I", b.CSRC, str(src), "-o", str(exe)], check=True)
    res = subprocess.run([str(exe)], capture_output=True, text=True)
    assert res.returncode == 0, res.stdout
    held, more = map(int, res.stdout.split())
    assert held > 100_000 and more > 1000  # repeated ids do exceed the room that S rows need


@pytest.mark.parametrize("name", ["layer_int8.hip"])
def test_kernel_and_launch_share_the_rule(name):
    """Both take the rows of a pass from the header, neither from a number of its own."""
    with open(os.path.join(b.CSRC, name)) as f:
        text = f.read()
    assert text.count("layer_int8_held_rows(") == 2 and "layer_int8_held(" in text
    assert "constexpr int kInt8HeldRows" not in text
