"""Which tiles a dense product takes, asked on the host: the plan that the launches follow, compiled without a GPU."""
import os
import subprocess

import pytest

from paper_2603_21090_amd import build

ASK = r"""
#include "linear.h"
#include <cstdio>
#include <cstdlib>
using namespace stgn::dense;
template <class T>
static void ask(const char* name, long m, long n, long k, bool l, bool r) {
  const Plan p = plan_of<T>(m, n, k, l, r);
  printf("%s %ld %ld %ld %d %d %d %d %d %d\n", name, m, n, k, (int)l, (int)r, p.bm, p.bn, p.splits, p.k_per);
}
int main() {
  const long out[] = {1, 8, 64, 200, 1024, 4096, 4104, 65536}, sum[] = {0, 1, 63, 64, 128, 4096, 100000};
  for (long m : out)
    for (long n : out)
      for (long k : sum)
        for (int o = 0; o < 4; ++o) {
          ask<float>("f32", m, n, k, o & 1, o & 2);
          ask<__bf16>("bf16", m, n, k, o & 1, o & 2);
          ask<_Float16>("f16", m, n, k, o & 1, o & 2);
        }
  return 0;
}
"""


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    """type, m, n, k, whether k runs along the operands' rows, and the plan: tile, splits, k a split"""
    at = tmp_path_factory.mktemp("plans")
    (at / "ask.hip").write_text(ASK)
    subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "-O1", "--offload-host-only", "--offload-arch=gfx950", "-std=c++17", "-I", build.CSRC, "-I",
                    os.path.join(build.ROOT, "include"), str(at / "ask.hip"), "-o", str(at / "ask")], check=True, capture_output=True)
    lines = subprocess.run([str(at / "ask")], check=True, capture_output=True, text=True).stdout.splitlines()
    return [(f[0], *map(int, f[1:])) for f in map(str.split, lines)]


def test_large_tiles_have_whole_tiles_to_sum(plans):
    """The kernel of 256 x 256 outputs reads whole tiles of 64 of k unasked, the first one at once: never for sums of nothing (dW without
    rows, whose operands may be null) or of a part of a tile, nor where a row per k is not whole pieces or an operand has a type of 32 bits."""
    large = [p for p in plans if p[6] == 256]
    assert large
    for t, m, n, k, l_rows, r_rows, bm, bn, splits, k_per in large:
        assert t != "f32" and bn == 256 and splits == 1 and k > 0 and k % 64 == 0, (t, m, n, k)
        assert (l_rows or n % 8 == 0) and (r_rows or m % 8 == 0), (t, m, n, k)
    assert any(p[3] == 0 and p[1] >= 4096 and p[2] >= 4096 for p in plans)


def test_splits_cover_the_sum_once(plans):
    for t, m, n, k, _, _, bm, bn, splits, k_per in plans:
        assert splits >= 1 and k_per >= 1 and (splits - 1) * k_per < max(k, 1) <= splits * k_per, (t, m, n, k)
