"""The 8-bit product's kernels that load tiles into LDS directly: rows far apart, operands that start anywhere, y over the residual (bounds: block_refs, computed on the
GPU in 64 bits; which kernel a size takes: test_linear_i8_kinds_cpu)."""
import pytest
import torch

import block_refs as refs
import linear_i8_sizes as sizes
from operator_refs import within
from paper_2603_21090_amd import binding

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16]


def make(rows, d_in, d_out, dt):
    g = torch.Generator(device="cuda").manual_seed(1000 * rows + 10 * d_in + d_out)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    i = lambda *s: torch.randint(-127, 128, s, generator=g, dtype=torch.int8, device="cuda")  # noqa: E731
    return i(rows, d_in), n(rows).abs() / 100, i(d_out, d_in), n(d_out).abs() / 100 * d_in ** -0.5, n(d_out).to(dt), n(rows, d_out).to(dt)


def near(got, want):
    within(got, tuple(t.cpu() for t in want), "y")


def apart(t, ld, at=0):
    """t as rows `ld` bytes apart that start `at` bytes behind a multiple of 16, 127 beside them where that is little."""
    rows, width = t.shape
    buffer = torch.empty(rows * ld + at, dtype=torch.int8, device="cuda")
    if buffer.numel() < 1 << 28:
        buffer.fill_(127)
    view = buffer[at:].view(rows, ld)[:, :width]
    view.copy_(t)
    assert view.data_ptr() % 16 == at % 16
    return view


@pytest.mark.parametrize("size", sizes.FAR, ids=str)
def test_rows_up_to_2_to_the_23_bytes_apart(size):
    """A tile's last row lies 2^30 bytes from its first but for a hundredth (2^31 in tiles of 256): the largest offsets that the plan allows."""
    x, xs, w, ws, b, _ = make(*size, torch.float32)
    far = lambda t: apart(t, (1 << 23) - 16) if t.shape[0] <= 1504 else t  # noqa: E731
    got = binding.linear_i8(far(x), xs, far(w), ws, bias=b)
    near(got, refs.linear_i8(x, xs, w, ws, b, "none", None, torch.float32))
    assert torch.equal(got, binding.linear_i8(x, xs, w, ws, bias=b))


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("more", [16, 19])
@pytest.mark.parametrize("at", [0, 1, 8])
@pytest.mark.parametrize("size", sizes.ANYWHERE, ids=str)
def test_operands_that_start_anywhere(size, at, more, dt):
    """Either operand, whichever kernel that makes; the residual is only read."""
    x, xs, w, ws, b, r = make(*size, dt)
    before = r.clone()
    want = binding.linear_i8(x, xs, w, ws, bias=b, activation="silu", residual=r)
    near(want, refs.linear_i8(x, xs, w, ws, b, "silu", r, dt))
    ld = size[1] + more
    for X, W in ((apart(x, ld, at), w), (x, apart(w, ld, at)), (apart(x, ld, at), apart(w, ld, at))):
        got = binding.linear_i8(X, xs, W, ws, bias=b, activation="silu", residual=r)
        near(got, refs.linear_i8(x, xs, w, ws, b, "silu", r, dt))
    assert torch.equal(r, before)


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("size", sizes.OVER, ids=str)
def test_y_over_the_residual(size, dt):
    x, xs, w, ws, b, r = make(*size, dt)
    want = binding.linear_i8(x, xs, w, ws, bias=b, activation="gelu", residual=r)
    near(want, refs.linear_i8(x, xs, w, ws, b, "gelu", r, dt))
    rows, d_in, d_out = size
    args = binding._PACK_LINEAR_I8.pack(binding._dtype_code(r), binding.ACTIVATIONS["gelu"], rows, d_in, d_out, 0, d_in, d_in, d_out, d_out, x.data_ptr(), w.data_ptr(),
                                        xs.data_ptr(), ws.data_ptr(), b.data_ptr(), r.data_ptr(), r.data_ptr())
    L = binding.load_library()
    binding._run_operator(L.stgn_linear_quantized_workspace, L.stgn_linear_quantized, args, None, r.device)
    assert torch.equal(r, want)
