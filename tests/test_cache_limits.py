"""Limits of the cache and rotary entry points: scales, and tensors of more tokens than one launch
holds workgroups for; without a GPU."""
import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2606_23743_amd import _lib
from paper_2606_23743_amd._lib import Cache, CacheQuery, Heads

pytestmark = pytest.mark.cpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_23743_amd", "csrc")
A, MB = 1 << 30, 1 << 24
LOG2E = 1.4426950408889634


@pytest.fixture(scope="module")
def lib():
    return _lib.load()


def _cache(fmt):
    return Cache(fmt, 4, 2, 64, 64, A, A + MB, A + 2 * MB, A + 2 * MB)


# A scale is used as float32 and in base 2: one that becomes zero there turns the logits of masked keys into
# 0 * -inf, one that becomes infinite all others.
BAD_SCALES = [5e-324, 1e-300, 1e-46, 2.0 ** -127 / LOG2E, 3.4e38 / LOG2E * 1.01, 1e39, 1.7e308]
GOOD_SCALES = [-1.0, 0.0, -1e300, 2.0 ** -126 / LOG2E * 1.000001, 1e-30, 0.125, 1.0, 1e30,
               3.4e38 / LOG2E * 0.999]


@pytest.mark.parametrize("fmt", [0, 1, 2])
def test_softmax_scales_that_float32_does_not_hold_are_refused(lib, fmt):
    heads = lambda at, h: Heads(at, h, h * 3 * 64, 3 * 64, 64)  # noqa: E731
    need = ctypes.c_size_t()

    def query(scale):
        return CacheQuery(2, 4, 3, 32, scale, 0)

    assert lib.sva_cache_attention_workspace(_cache(fmt), query(0.0), need) == _lib.SVA_OK
    for scale in BAD_SCALES:
        assert lib.sva_cache_attention_workspace(_cache(fmt), query(scale), need) == _lib.SVA_ERR_INVALID_ARG, scale
        # the call itself: with these addresses it must not come to a launch
        assert lib.sva_cache_attention(_cache(fmt), query(scale), heads(A + 4 * MB, 4), A, A, heads(A + 6 * MB, 2),
                                       heads(A + 7 * MB, 2), A, 9, A, A + 8 * MB, need.value, heads(A + 5 * MB, 4), A,
                                       None) == _lib.SVA_ERR_INVALID_ARG, scale
    for scale in GOOD_SCALES:
        assert lib.sva_cache_attention_workspace(_cache(fmt), query(scale), need) == _lib.SVA_OK, scale


SLICES = r"""
#include <cstdio>
#include "cache_args.h"

int main() {
  long bad = 0;
  for (int threads : {64, 256, 1024}) {
    const int64_t most = UINT32_MAX / threads;
    for (int64_t groups : {(int64_t)1, (int64_t)2, most - 1, most, most + 1, 2 * most, 2 * most + 1, (int64_t)INT32_MAX}) {
      if (groups > INT32_MAX) continue;
      int64_t at = 0;
      int calls = 0;
      sva::launch_slices(groups, threads, [&](int first, unsigned n) {
        bad += first != at || n == 0 || (int64_t)n * threads >= (int64_t)1 << 32;
        at += n;
        ++calls;
      });
      bad += at != groups || calls != (groups + most - 1) / most;
    }
  }
  std::printf("%ld\n", bad);
  return bad != 0;
}
"""


def test_launches_hold_fewer_than_2_to_the_32_threads(tmp_path):
    """Every workgroup once, in launches that the runtime takes (a launch of 2^32 threads or more is an error)."""
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    (tmp_path / "slices.cpp").write_text(SLICES)
    subprocess.run([hipcc, "-x", "c++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I", CSRC, "-I",
                    "/opt/rocm/include", str(tmp_path / "slices.cpp"), "-o", str(tmp_path / "slices")], check=True,
                   capture_output=True, text=True)
    r = subprocess.run([str(tmp_path / "slices")], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0 and r.stdout.strip() == "0", r.stdout
