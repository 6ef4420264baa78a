"""Whether strided tensors share a byte (csrc/overlap.h), on the host: against all bytes of small
layouts, and for the layouts that real programs slice."""
import os
import shutil
import subprocess

import pytest

pytestmark = pytest.mark.cpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_23743_amd", "csrc")

PROGRAM = r"""
#include <cstdio>
#include <random>
#include <set>
#include "overlap.h"

using sva::RowSet;
using sva::rows_meet;

std::set<int64_t> bytes(const RowSet& r) {
  std::set<int64_t> s;
  for (int64_t a = 0; a < r.size[0]; ++a)
    for (int64_t b = 0; b < r.size[1]; ++b)
      for (int64_t c = 0; c < r.size[2]; ++c)
        for (int64_t e = 0; e < r.row; ++e) s.insert((int64_t)r.at + a * r.stride[0] + b * r.stride[1] + c * r.stride[2] + e);
  return s;
}

int main() {
  std::mt19937 rng(5);
  long bad = 0, met = 0;
  for (int rep = 0; rep < 40000; ++rep) {
    RowSet x, y;
    const int kind = rng() % 3;                  // strides of their own, the same, or nested ones
    for (RowSet* r : {&x, &y}) {
      r->at = 1000 + rng() % 60;
      r->row = 1 + rng() % 5;
      for (int i = 0; i < 3; ++i) {
        r->size[i] = 1 + rng() % 4;
        r->stride[i] = rng() % 30;
      }
      if (kind == 2) {
        r->stride[2] = 6 + rng() % 3;
        r->stride[1] = 4 * r->stride[2] + rng() % 3;
        r->stride[0] = 4 * r->stride[1] + rng() % 3;
      }
    }
    if (kind == 1)
      for (int i = 0; i < 3; ++i) y.stride[(i + 1) % 3] = x.stride[i];
    const std::set<int64_t> bx = bytes(x);
    bool want = false;
    for (int64_t e : bytes(y)) want = want || bx.count(e);
    bad += rows_meet(x, y) != want;
    met += want;
  }
  printf("%ld %ld ", bad, met);
  // slices of a projection [B, N, 3, H, D], with as many key heads or fewer: apart, and one head further not
  const int64_t B = 3, N = 63240, H = 32, D = 256;       // (bytes of a head's row)
  for (int64_t kv : {H, H / 4}) {
    const int64_t all = H + 2 * kv;
    const RowSet q = {1 << 20, (int64_t)D, {B, H, N}, {N * all * D, D, all * D}};
    const RowSet k = {(uint64_t)((1 << 20) + H * D), (int64_t)D, {B, kv, N}, {N * all * D, D, all * D}};
    RowSet v = k;
    v.at += kv * D;
    printf("%d%d%d", rows_meet(q, k), rows_meet(q, v), rows_meet(k, v));
    v.at += D;                                           // its last head is the next token's first of q
    printf("%d%d", rows_meet(q, v), rows_meet(k, v));
    v.at -= 2 * D;
    printf("%d%d ", rows_meet(k, v), rows_meet(v, q));
  }
  // entries packed one after the other, queries and then keys of other numbers and pitches
  const int64_t M = 512, kv = 8, entry = (N * H + M * kv) * D;
  RowSet q = {1 << 20, D, {B, H, N}, {entry, D, H * D}}, k = {(uint64_t)((1 << 20) + N * H * D), D, {B, kv, M}, {entry, M * D, D}};
  printf("%d", rows_meet(q, k));
  k.at -= D;
  printf("%d", rows_meet(q, k));
  // moved by one token and by one head
  RowSet o = q;
  o.at += H * D;
  printf("%d", rows_meet(q, o));
  o.at = q.at + 16;
  printf("%d", rows_meet(q, o));
  // a cache's rows around it: heads of 128 in pitches of 160 elements
  RowSet w = {1 << 20, D, {B, H, N}, {N * H * 320, 320, H * 320}}, gap = w;
  gap.at += D;
  gap.row = 64;
  printf("%d", rows_meet(w, gap));
  gap.row = 65;
  printf("%d\n", rows_meet(w, gap));
  return 0;
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_rows_that_share_a_byte(tmp_path):
    src, exe = tmp_path / "overlap.cpp", tmp_path / "overlap"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Werror", "-I", CSRC, "-o", str(exe), str(src)], check=True)
    bad, met, *layouts = subprocess.run([str(exe)], check=True, capture_output=True, text=True, timeout=60).stdout.split()
    assert int(bad) == 0 and 10000 < int(met) < 39000
    # v one head on meets the next token's q and not k, one head back k and not q
    assert layouts == ["0001010", "0001010", "011101"]
