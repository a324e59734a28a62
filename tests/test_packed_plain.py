"""Pins of the packed cache's plain 64-bit form by values worked out by hand, and of the
stored form's layout (compiled from the library's header on the host)."""
import os
import shutil
import subprocess

import numpy as np
import pytest

from tests import packed_plain as pp

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_stored_values_by_hand():
    # largest 6: scale 1, so entries go to the grid itself, ties to the even code
    x = np.array([6, -6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -5, 0.2, 0.3, 4.9, 5.1, 0, -0.26])
    want = [6, -6, 0, 1, 1, 2, 2, 4, 4, -4, 0, 0.5, 4, 6, 0, -0.5]
    assert pp.stored(x).tolist() == want
    # largest 6.4: 6.4 / 6 = 1.0667 is nearer to 1.125 than to 1; 6.4 / 1.125 = 5.69 -> 6
    assert pp.stored(np.r_[6.4, np.zeros(15)])[0] == 6.75
    # largest 6.375: 1.0625 lies halfway; the even mantissa is 1's, and 6.375 saturates at 6
    assert pp.stored(np.r_[6.375, np.zeros(15)])[0] == 6.0
    # the scale saturates at 10240, and vanishes below half of 2^-17
    assert pp.stored(np.r_[1e9, np.zeros(15)])[0] == 61440.0
    assert pp.stored(np.r_[6 * 2.0 ** -18, np.zeros(15)])[0] == 0.0  # a tie: to even, zero
    assert pp.stored(np.r_[6.1 * 2.0 ** -18, np.zeros(15)])[0] == 3 * 2.0 ** -17
    # a NaN or infinity takes its whole row, and no other
    y = pp.stored(np.stack([np.r_[np.ones(31), np.inf], np.ones(32)]))
    assert np.isnan(y[0]).all() and np.isfinite(y[1]).all()


def test_bounds_and_selection_by_hand():
    k = np.zeros((130, 1, 16))
    k[3, 0, 0], k[70, 0, 0], k[129, 0, 1] = 127.0, 128.0, -1.0
    hi, lo, u = pp.bounds(k)
    assert u[0].tolist() == [1.0, 2.0, 2.0 ** -6]
    assert hi[0, :, 0].tolist() == [127, 64, 0] and lo[0, 2, 1] == -64
    q = np.zeros((1, 2, 16))
    q[0, 0, 0], q[0, 1, 0] = 1.0, -2.0  # up 1, down -2: scores 127 P_0 and 128 P_0
    assert pp.select(q, [129], k, 2)[0, 0].tolist() == [1, 2]
    assert pp.select(q, [129], k, 5)[0, 0].tolist() == [0, 1, 2, -1, -1]
    assert pp.select(np.zeros((1, 2, 16)), [129], k, 2)[0, 0].tolist() == [0, 2]  # ties
    assert pp.select(q, [-1], k, 2)[0, 0].tolist() == [-1, -1]


def test_attention_by_hand():
    k = np.zeros((3, 1, 16))
    v = np.zeros((3, 1, 16))
    v[:, 0, 0] = [1.0, 2.0, 6.0]
    q = np.ones((4, 1, 16))
    out = pp.attention(q, [-1, 0, 1, 2], k, v)[0]
    assert out[:, 0, 0].tolist() == [0.0, 1.0, 1.5, 3.0]
    out = pp.attention(q, [2] * 4, k, v, np.array([[[-1]], [[0]], [[1]], [[0]]]))[0]
    assert out[:, 0, 0].tolist() == [0.0, 3.0, 0.0, 3.0]


HOST = r"""
#include <cstdio>
#include "packed.cuh"
using namespace kvr;
int main() {
  for (int dh = 64; dh <= 128; dh += 64) {
    const int cb = pack_code_bytes(dh), hb = pack_half_bytes(dh);
    if (pack_block_bytes(dh) != 2 * hb) return 1;
    std::vector<int> k(hb, 0), v(hb, 0);  // bytes taken
    for (int key = 0; key < 64; ++key) {
      for (int e = 0; e < dh; e += 4) {
        const int a = pack_k_code(dh, key, e);
        if (a < 0 || a + 2 > cb || a % 2) return 2;
        ++k[a], ++k[a + 1];
        // the two keys of a word, as the kernels write them in one store
        if (key % 4 < 2 && (a % 4 || pack_k_code(dh, key + 2, e) != a + 2)) return 3;
      }
      for (int db = 0; db < dh / 16; ++db) {
        const int a = pack_k_scale(dh, key, db), b = pack_v_scale(dh, key, db);
        if (a < cb || a >= hb || b < cb || b >= hb) return 4;
        ++k[a], ++v[b];
      }
    }
    for (int k4 = 0; k4 < 16; ++k4)
      for (int e = 0; e < dh; ++e) {
        const int a = pack_v_code(k4, e);
        if (a < 0 || a + 2 > cb || a % 2) return 5;
        ++v[a], ++v[a + 1];
      }
    for (int i = 0; i < hb; ++i)
      if (k[i] != 1 || v[i] != 1) return 6;  // every byte once
  }
  std::vector<int> keys(16, 0);
  for (int g = 0; g < 8; ++g) ++keys[pack_key_of(g)], ++keys[pack_key_of(g) + 2];
  for (int x : keys)
    if (x != 1) return 7;
  PackedView big{nullptr, nullptr, nullptr, 1 << 14, 8, 128};  // 2^20 positions, 32 layers
  if ((size_t)big.block(31, 7, (1 << 14) - 1) != (size_t)((32ull << 17) - 1) * 9216) return 8;
  puts("ok");
  return 0;
}
"""


def test_layout_takes_every_byte_once(tmp_path):
    from paper_2609_17983_gb300 import build
    if not (shutil.which("nvcc") or os.path.exists("/usr/local/cuda/bin/nvcc")):
        pytest.skip("no nvcc")
    src = tmp_path / "layout.cu"
    src.write_text(HOST)
    exe = tmp_path / "layout"
    r = subprocess.run([build.nvcc(), *build.ARCH, "-std=c++17", "--expt-relaxed-constexpr", "-I",
                        build.CSRC, "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.returncode
