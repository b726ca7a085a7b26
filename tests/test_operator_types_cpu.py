"""What the operators' kernels say about addresses, asked of the compiler: no GPU is needed."""
import os
import subprocess

import pytest

from paper_2603_21090_amd import build


@pytest.mark.parametrize("name", ["u32_any", "u32x2_any", "u32x4_any"])
def test_words_that_lie_anywhere(name, tmp_path):
    """Rows of 8-bit numbers start at any byte: the types that global memory is read and written through promise no alignment, and are as long as their words."""
    words = {"u32_any": 1, "u32x2_any": 2, "u32x4_any": 4}[name]
    at = tmp_path / "ask.hip"
    at.write_text(f'#include "tile_ops.h"\nstruct After {{ char first; stgn::{name} word; }};\n'
                  f"static_assert(alignof(After) == 1, \"alignment\");\nstatic_assert(sizeof(After) == {4 * words} + 1, \"size\");\n")
    r = subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "-fsyntax-only", "--offload-host-only", "--offload-arch=gfx950", "-std=c++17", "-I", build.CSRC, str(at)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
