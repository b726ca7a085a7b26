"""The norm and matrices in 8 bits where a workgroup has many rows, where outputs lie apart, and at magnitudes whose products 32 bits do not hold
(bounds: block_refs, computed on the GPU in 64 bits)."""
import ctypes as C

import pytest
import torch

import block_refs as refs
from operator_refs import within
from paper_2603_21090_amd import binding

pytestmark = pytest.mark.gpu
ALL = [torch.float32, torch.bfloat16, torch.float16]
TYPES = [torch.float32, torch.bfloat16]                       # the sizes of element that kernels are made for


def make(rows, width, dt, seed=0):
    g = torch.Generator(device="cuda").manual_seed(1000 * rows + width + seed)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    return n(rows, width).to(dt), n(rows, width).to(dt), (1 + n(width) / 4).to(dt), n(rows, width).to(dt), n(rows, width).to(dt)


def near(got, want, name):
    within(got, tuple(t.cpu() for t in want), name)


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("sizes", [(1e30, 1e10), (2.0 ** 120, 2.0 ** 100), (1e-30, 1e-10), (2.0 ** -100, 2.0 ** -60)], ids=str)
@pytest.mark.parametrize("width", [200, 5000, 16384, 16389, 40001])
def test_gradients_of_large_and_small_numbers(width, sizes, dt):
    """dy h overflows or vanishes in 32 bits; neither dy h r nor anything else that the formulas have does."""
    _, h, gain, dy, _ = make(200, width, dt)
    h, dy = (h.double() * sizes[0]).to(dt), (dy.double() * sizes[1]).to(dt)
    for got, want, name in zip(binding.rms_norm_grad(dy, h, gain, eps=0.0), refs.rms_norm_grad(dy, h, gain, None, 0.0), ("dx", "dgain")):
        near(got, want, name)
