"""The kernel that each size of the GPU tests of the 8-bit product is meant for, asked of the plan on the host."""
import os
import subprocess

import pytest

import linear_i8_sizes as sizes
from paper_2603_21090_amd import build

ASK = r"""
#include "linear_i8.h"
#include <cstdio>
#include <cstdlib>
using namespace stgn::dense8;
int main(int count, char** v) {
  for (int i = 1; i + 2 < count; i += 3) {
    stgn::Linear8Args f{};
    f.rows = atoi(v[i]); f.d_in = atoi(v[i + 1]); f.d_out = atoi(v[i + 2]);
    for (int start = 0; start < 2; ++start)                   // at a multiple of 16 bytes; 8 behind one
      for (int apart = 0; apart < 3; ++apart) {               // rows side by side; 16 bytes apart; 19
        f.ld_w = f.d_in;
        f.ld_x = f.d_in + (apart == 0 ? 0 : apart == 1 ? 16 : 19);
        f.x = reinterpret_cast<const int8_t*>(16 + 8 * start);
        f.w = reinterpret_cast<const int8_t*>(16);
        const Plan p = plan_of(f.rows, f.d_out, f.d_in, whole_pieces(f), !whole_rows(f));
        printf("%d %d %d %d %d %d %d %d\n", f.rows, f.d_in, f.d_out, start, apart, (int)p.kind, p.splits, p.aligned);
      }
  }
  return 0;
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    """(size, how x starts, how far apart its rows lie) -> (kernel, split or not, laid out again or not)"""
    at = tmp_path_factory.mktemp("kinds")
    (at / "ask.hip").write_text(ASK)
    subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "-O1", "--offload-host-only", "--offload-arch=gfx950", "-std=c++17", "-I", build.CSRC, "-I",
                    os.path.join(build.ROOT, "include"), str(at / "ask.hip"), "-o", str(at / "ask")], check=True, capture_output=True)
    every = {**sizes.FAR, **sizes.ANYWHERE, **sizes.OVER, **sizes.KINDS}
    out = subprocess.run([str(at / "ask"), *(str(n) for s in every for n in s)], check=True, capture_output=True, text=True).stdout
    return {(v[:3], v[3], v[4]): (v[5], v[6] > 1, v[7] > 0) for v in (tuple(map(int, line.split())) for line in out.splitlines())}


@pytest.mark.parametrize("table", ["FAR", "ANYWHERE", "OVER", "KINDS"])
def test_sizes_take_the_kernel_they_are_for(plan, table):
    for size, want in getattr(sizes, table).items():
        assert plan[size, 0, 0] == want, size


def test_operands_that_are_no_whole_pieces_are_never_loaded_directly_as_they_are(plan):
    """Whole pieces elsewhere than at a multiple of 16 bytes go through registers; rows that no 16 bytes align are laid out again for the same kernel."""
    for size, (kind, split, _) in sizes.ANYWHERE.items():
        assert plan[size, 0, 1] == (kind, split, False), size
        for start, apart in ((1, 0), (1, 1)):
            assert plan[size, start, apart] == (sizes.SMALL, False, False), size
        for start in (0, 1):
            assert plan[size, start, 2] == (kind, split, True), size
