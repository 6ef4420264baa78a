"""The division of cached keys among workgroups (csrc/cache_attn_plan.h), on the
host: every unit of every segment goes to exactly one workgroup, the one that owner()
names, no workgroup has none, and the parts of divided segments lie in slots of their
own, where the join looks for them; for ragged, empty and single entries, and for
segments that are not divided."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_23743_amd", "csrc")

PROGRAM = r"""
#include <cstdio>
#include <random>
#include <set>
#include <vector>
#include "cache_attn_plan.h"

using namespace sva::cattn;

int main() {
  std::mt19937 rng(7);
  long bad = 0;
  for (int rep = 0; rep < 3000; ++rep) {
    const int B = 1 + rng() % (rep % 10 == 0 ? 200 : 6), kv = 1 + rng() % 5, G = 1 + rng() % 9, T = 1 + rng() % 70;
    const int rows = 16 << (rng() % 3), max_len = 1 + rng() % 5000, grid = 1 + rng() % 300;
    const bool drafts = rng() % 2, whole = rng() % 8 == 0;
    std::vector<Entry> e(B);
    std::vector<int64_t> base(B + 1, 0);
    int begin = whole ? -1 : 0;
    for (int pass = 0; pass < 2; ++pass) {           // units first, then with what beginning a segment takes
      std::mt19937 same(rep);
      for (int b = 0; b < B; ++b) {
        const int len = same() % 4 == 0 ? (int)(same() % 3) - 1 : (int)(same() % (max_len + 50));
        const int cnt = same() % 4 == 0 ? (int)(same() % (T + 3)) - 1 : T;
        const Entry x = e[b] = entry_of(len, cnt, max_len, T, G, rows, drafts, begin);
        bad += x.len < 0 || x.len > max_len || x.cnt < 0 || x.cnt > T || x.units < 1;
        bad += (int64_t)x.cached_units * kUnit < x.len || (int64_t)x.tiles * rows < (int64_t)x.cnt * G;
        if (drafts) bad += (int64_t)(x.units - x.cached_units) * kUnit < x.cnt;
        base[b + 1] = base[b] + entry_work(x, kv);
      }
      if (!whole && pass == 0) begin = begin_of(base[B], grid);
    }
    const int64_t W = base[B];
    if (W == 0) continue;
    const int n = (int)(grid < W ? grid : W);
    // runs as the kernels take them: every unit once, at its owner, none empty
    std::set<std::vector<int>> units;
    std::set<int64_t> wrote, read;
    int64_t at = 0;
    for (int i = 0; i < n; ++i) {
      int64_t x = run_of(i, n, W);
      const int64_t end = run_of(i + 1, n, W);
      bad += x != at;
      at = end;
      int took = 0, b = 0;
      while (x < end) {
        while (x >= base[b + 1]) ++b;
        const Piece p = piece_at(e[b], x - base[b], end - x);
        bad += p.seg < 0 || p.seg >= e[b].tiles * kv || base[b] + p.next <= x || base[b] + p.next > base[b + 1];
        bad += p.u0 < 0 || p.u1 > e[b].units || p.u0 > p.u1;
        for (int u = p.u0; u < p.u1; ++u, ++took) {
          bad += !units.insert({b, p.seg, u}).second;
          if (!whole) bad += owner(base[b] + place_of(e[b], p.seg, u), n, W) != i;
        }
        if (p.u0 < p.u1 && p.u1 - p.u0 < e[b].units) bad += !wrote.insert(2 * i + (p.u0 == 0 ? 1 : 0)).second;
        x = base[b] + p.next;
      }
      bad += took == 0;
    }
    bad += at != W;
    size_t all = 0;
    for (int b = 0; b < B; ++b) {
      all += (size_t)e[b].units * e[b].tiles * kv;
      for (int s = 0; s < e[b].tiles * kv && !whole; ++s) {
        const int i0 = owner(base[b] + place_of(e[b], s, 0), n, W);
        const int i1 = owner(base[b] + place_of(e[b], s, e[b].units - 1), n, W);
        if (i0 == i1) continue;
        for (int i = i0; i <= i1; ++i) bad += !read.insert(2 * i + (i == i0 ? 1 : 0)).second;
      }
    }
    bad += units.size() != all || wrote != read || (whole && !wrote.empty());
  }
  std::printf("%ld\n", bad);
  return bad != 0;
}
"""

pytestmark = pytest.mark.cpu


def test_every_unit_once_and_slots_agree(tmp_path):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    src = tmp_path / "plan.cpp"
    src.write_text(PROGRAM)
    exe = tmp_path / "plan"
    subprocess.run([hipcc, "-x", "c++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I", CSRC, "-I",
                    "/opt/rocm/include", str(src), "-o", str(exe)], check=True, capture_output=True, text=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.strip() == "0", r.stdout
