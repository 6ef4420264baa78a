"""The division of cached keys among workgroups (csrc/cache_attn_plan.h), on the
host: every unit of every segment goes to exactly one workgroup, runs differ by at
most one unit, owner() names the workgroup whose run holds a unit, and no two parts
of divided segments share a slot; for ragged, empty and single entries."""
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
    const bool drafts = rng() % 2;
    std::vector<Entry> e(B);
    int64_t U = 0;
    for (auto& x : e) {
      const int len = rng() % 4 == 0 ? (int)(rng() % 3) - 1 : (int)(rng() % (max_len + 50));
      const int cnt = rng() % 4 == 0 ? (int)(rng() % (T + 3)) - 1 : T;
      x = entry_of(len, cnt, max_len, T, G, rows, drafts, true);
      bad += x.len < 0 || x.len > max_len || x.cnt < 0 || x.cnt > T || x.units < 1;
      bad += (int64_t)x.cached_units * kUnit < x.len || (int64_t)x.tiles * rows < (int64_t)x.cnt * G;
      if (drafts) bad += (int64_t)(x.units - x.cached_units) * kUnit < x.cnt;
      U += entry_work(x, kv);
    }
    const Entry whole = entry_of(max_len, T, max_len, T, G, rows, drafts, false);
    bad += entry_work(whole, kv) != (int64_t)whole.tiles * kv;     // undivided: a place for each segment
    if (U == 0) continue;
    const int n = (int)(grid < U ? grid : U);
    int64_t at = 0, least = U, most = 0;
    for (int i = 0; i < n; ++i) {
      const int64_t x0 = first_unit(i, n, U), x1 = first_unit(i + 1, n, U);
      bad += x0 != at || x1 <= x0;
      at = x1;
      least = x1 - x0 < least ? x1 - x0 : least;
      most = x1 - x0 > most ? x1 - x0 : most;
      for (int64_t x = x0; x < x1; x += 1 + (x1 - x0) / 7) bad += owner(x, n, U) != i;
      bad += owner(x1 - 1, n, U) != i;
    }
    bad += at != U || most - least > 1;
    // slots as the kernel takes them against those that the join reads
    std::set<int64_t> wrote, read;
    for (int i = 0; i < n; ++i) {
      int64_t x = first_unit(i, n, U);
      const int64_t end = first_unit(i + 1, n, U);
      while (x < end) {
        int64_t base = 0;
        int b = 0;
        while (x >= base + entry_work(e[b], kv)) base += entry_work(e[b++], kv);
        const int64_t seg = (x - base) / e[b].units, u0 = x - base - seg * e[b].units;
        const int64_t u1 = e[b].units < u0 + (end - x) ? e[b].units : u0 + (end - x);
        if (u1 - u0 < e[b].units) bad += !wrote.insert(2 * i + (u0 == 0 ? 1 : 0)).second;
        x += u1 - u0;
      }
    }
    int64_t base = 0;
    for (int b = 0; b < B; ++b)
      for (int64_t s = 0; s < (int64_t)e[b].tiles * kv; ++s, base += e[b].units) {
        const int i0 = owner(base, n, U), i1 = owner(base + e[b].units - 1, n, U);
        if (i0 == i1) continue;
        for (int i = i0; i <= i1; ++i) bad += !read.insert(2 * i + (i == i0 ? 1 : 0)).second;
      }
    bad += base != U || wrote != read;
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
