"""Which kernel the product of operands in 8 bits takes, asked on the host: the plan that the launches follow, compiled without a GPU."""
import os
import subprocess

import pytest

from paper_2603_21090_amd import build

ASK = r"""
#include "linear_i8.h"
#include <cstdio>
using namespace stgn::dense8;
int main() {
  const long rows[] = {1, 16, 17, 64, 65, 100, 200, 512, 1000, 1531, 2048, 4096, 5000, 8192, 40000, 1000000}, cols[] = {1, 64, 200, 777, 1024, 4096, 5000, 8192, 65536},
             sum[] = {1, 15, 16, 63, 64, 100, 128, 256, 368, 512, 1000, 1024, 1027, 2000, 2048, 4096, 4112, 8192, 131071};
  for (long m : rows)
    for (long n : cols)
      for (long k : sum)
        for (int rows = 0; rows < 3; ++rows) {                // whole pieces; whole ones but for where they lie; rows that 16 bytes do not align
          if (rows < 2 && k % 16) continue;
          stgn::Linear8Args f{};
          f.rows = (int)m; f.d_out = (int)n; f.d_in = (int)k; f.ld_x = rows == 2 ? k / 16 * 16 + 17 : k; f.ld_w = k;
          f.x = reinterpret_cast<const int8_t*>(rows == 1 ? 8 : 16);
          const Plan p = plan_of(m, n, k, whole_pieces(f), !whole_rows(f));
          printf("%ld %ld %ld %d %d %d %d %d %d %zu %d\n", m, n, k, rows, (int)p.kind, p.splits, p.k_per, p.mb, p.nb, part_bytes(f), p.aligned);
        }
  return 0;
}
"""
FRAGMENTS, SMALL, SMALL2, DIRECT, LARGE = range(5)
WHOLE, ELSEWHERE, UNALIGNED = range(3)


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    """m, n, k, how the rows lie, and the plan: kernel, splits, k a split, blocks; bytes of the workspace; k of operands that are laid out again"""
    at = tmp_path_factory.mktemp("plans")
    (at / "ask.hip").write_text(ASK)
    subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "-O1", "--offload-host-only", "--offload-arch=gfx950", "-std=c++17", "-I", build.CSRC, "-I",
                    os.path.join(build.ROOT, "include"), str(at / "ask.hip"), "-o", str(at / "ask")], check=True, capture_output=True)
    return [tuple(map(int, line.split())) for line in subprocess.run([str(at / "ask")], check=True, capture_output=True, text=True).stdout.splitlines()]


def test_every_kernel_is_reached(plans):
    assert {p[4] for p in plans if p[3] == WHOLE} == {FRAGMENTS, SMALL, SMALL2, DIRECT, LARGE}
    assert {p[4] for p in plans if p[10]} == {DIRECT, LARGE}
    assert {p[7:9] for p in plans if p[4] == FRAGMENTS} == {(1, 1), (2, 1), (2, 2), (2, 4), (4, 4)}


def test_tiles_that_go_into_lds_directly_are_whole_pieces(plans):
    """The direct kernels read 16 aligned bytes a lane, the one of 256 x 256 whole tiles of 64 bytes of k: never a part of one."""
    for m, n, k, rows, kind, splits, k_per, _, _, _, aligned in plans:
        if aligned:
            assert rows == UNALIGNED and k > 16 and aligned % 64 == 0 and k <= aligned < k + 64 and kind in (DIRECT, LARGE), (m, n, k)
        if kind in (DIRECT, LARGE):
            assert (rows == WHOLE or aligned) and (aligned or k) % 16 == 0 and k_per % 128 == 0, (m, n, k)
        if kind in (DIRECT, LARGE):
            assert n >= 8, (m, n, k)                          # their epilogue goes by eights
        if kind == LARGE:
            assert (aligned or k) % 64 == 0 and splits == 1, (m, n, k)


def test_splits_cover_the_sum_once_and_fit_the_workspace(plans):
    for m, n, k, _, kind, splits, k_per, mb, nb, size, aligned in plans:
        assert splits >= 1 and (splits - 1) * k_per < (aligned or k) <= splits * k_per, (m, n, k)
        assert size >= (splits * m * n * 4 if splits > 1 else 0) + (m + n) * aligned, (m, n, k)
        assert splits == 1 or kind in (SMALL2, DIRECT), (m, n, k)
        if kind == FRAGMENTS:
            assert -(-m // (16 * mb)) * -(-n // (16 * nb)) <= 256, (m, n, k)
