"""How the eviction cuts long caches, on the CPU: over the lengths that the call
accepts the slices tile the rows, and no 32-bit sum overflows (the compiler
evaluates the formulas, and refuses a constant whose evaluation overflows).
Caches of that size fit no GPU's memory; nothing is allocated here."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

import paper_2503_10571_amd as radar
from paper_2503_10571_amd import _build

PROGRAM = r"""
#include "evict_slices.h"
using namespace radar_impl;

// the slices of every sequence of a call with t rows hold its rows, each once
constexpr bool tiles(int64_t t, int64_t len) {
  if (slice_rows_of(t) > INT32_MAX) return false;
  const int rows = (int)slice_rows_of(t), n = (int)((t + rows - 1) / rows);
  if (n > kSlices || rows % kStep != 0) return false;
  if (slices_of((int)len, rows) > n || slices_of((int)len, rows) < 1) return false;
  int64_t at = 0;
  for (int s = 0; s < n; ++s) {
    const int begin = s * rows, end = slice_end((int)len, begin, rows);
    if (begin >= len) {
      if (s < slices_of((int)len, rows)) return false;
      continue;
    }
    if (s >= slices_of((int)len, rows) || begin != at || end <= begin) return false;
    // a step's last row and the next step's first, as a workgroup counts them
    const int last = begin + (end - begin - 1) / kStep * kStep;
    if (last + kStep - 1 < begin || last + kStep < begin) return false;
    at = end;
  }
  return at == len;
}
constexpr bool tiles_up_to(int64_t t) {
  return tiles(t, t) && tiles(t, t - 1) && tiles(t, 1) && tiles(t, t / 2) && tiles(t, t / 3 + 1);
}
static_assert(tiles_up_to(kMostRows) && tiles_up_to(kMostRows - 1), "");
static_assert(tiles_up_to(((int64_t)1 << 31) - (1 << 18)) && tiles_up_to(((int64_t)1 << 31) - (1 << 18) + 1), "");
static_assert(tiles_up_to(((int64_t)1 << 31) - (1 << 26)) && tiles_up_to(((int64_t)1 << 31) - (1 << 26) + 1), "");
static_assert(tiles_up_to((int64_t)1 << 30) && tiles_up_to(65600) && tiles_up_to(262145), "");
static_assert(tiles_up_to(kStep + 1) && tiles_up_to(2 * kStep), "");
// a launch of the move
static_assert(kMostChunks * kMoveThreads < ((int64_t)1 << 32), "");
static_assert(move_chunks(kMostRows, 512) > kMostChunks && move_chunks(kMostRows, 128) <= kMostChunks, "");
int main() { return 0; }
"""


def test_slices_tile_every_length(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    src = tmp_path / "slices.cpp"
    src.write_text(PROGRAM)
    r = subprocess.run([cxx, "-std=c++17", "-fconstexpr-ops-limit=100000000", "-I", _build.CSRC, "-fsyntax-only",
                        str(src)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr


def test_a_move_of_more_than_a_launch_is_refused():
    if not os.path.exists(radar.LIB_PATH):
        _build.build_library()
    cap = (1 << 31) - 1
    cfg = radar.Config(1, 1, 1, 128, 64, 16, 16, cap, torch.float32)
    most = ((1 << 32) - 1) // 1024 * (1 << 17) // 512               # rows of 512 bytes
    assert radar.evict_workspace_bytes(cfg, most + 100, most, 0) > 0
    assert radar.evict_workspace_bytes(cfg, most + 100, most + 1, 0) == 0
    p = ctypes.c_void_p(0x1000)
    assert radar.lib().radar_evict(ctypes.byref(cfg.c_struct()), p, p, p, most + 100, None, most + 1, 0, None,
                                   None, p, 1 << 62, None) == 3
    # rows of 128 bytes: every accepted t
    cfg = radar.Config(1, 1, 1, 64, 64, 16, 16, cap, torch.bfloat16)
    assert radar.evict_workspace_bytes(cfg, cap - (1 << 14), 1 << 30, 1 << 29) > 0
