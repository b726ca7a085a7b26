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


# more rows than a launch has lanes for, for every number of lanes and pieces that hold a row: a workgroup has two rows and more, the next one on its way
LONG = [(20000, 40), (20000, 200), (5000, 500), (5000, 1000), (4500, 2000), (2100, 4000), (2100, 4099), (1100, 8191), (600, 16380), (600, 32763)]


def check_eight(q, scale, y):
    """q and scale of y's rows in 64 bits, y having been within 6 u of them in 32: half a step and what 12 u of 127 make."""
    top = y.abs().amax(1, keepdim=True)
    assert ((q.double() - 127 * y / top).abs() <= 0.5 + 127 * 14 * refs.U).all()
    assert ((scale.double() - top[:, 0] / 127).abs() <= 8 * refs.U * top[:, 0] / 127).all()


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("size", LONG, ids=str)
def test_workgroups_walk_down_the_rows(size, dt):
    x, res, gain, *_ = make(*size, dt)
    near(binding.rms_norm(x, gain), refs.rms_norm(x, None, gain)[0], "y")
    y, h = binding.rms_norm(x, gain, residual=res)
    want = refs.rms_norm(x, res, gain)
    near(y, want[0], "y of the sum")
    near(h, want[1], "h")
    for residual, wide in ((None, refs.rms_norm(x, None, gain)[0]), (res, want[0])):
        got = binding.rms_norm_i8(x, gain, residual=residual, keep_y=True)
        near(got[-1], wide, "y beside q")
        check_eight(got[0], got[1], wide[0])
    q, scale = binding.quantize(x)
    want_q, want_scale = refs.eight(x.float())
    assert torch.equal(q, want_q) and torch.equal(scale, want_scale)


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("size", LONG, ids=str)
def test_gradients_of_workgroups_with_many_rows(size, dt):
    _, h, gain, dy, dh = make(*size, dt)
    want = refs.rms_norm_grad(dy, h, gain, dh)
    dx, dgain = binding.rms_norm_grad(dy, h, gain, dh=dh)
    near(dx, want[0], "dx")
    near(dgain, want[1], "dgain")
    assert torch.equal(binding.rms_norm_grad(dy, h, gain, dh=dh, need_gain=False)[0], dx)


@pytest.mark.parametrize("dt", TYPES, ids=str)
def test_launches_of_as_many_workgroups_as_there_are(dt):
    """The norm with a residual and the gradient without the gain's have a workgroup for sixteen rows, 2^20 at most: the last rows are a second round.  One
    number a row: y = g sign(h) with eps = 0; with eps = 3 and h = +-1 r is a half, dx = r (g dy - r^2 g dy) + dh = 3/8 g dy + dh, which no step rounds."""
    rows = (1 << 24) + 37
    at = torch.arange(rows, device="cuda")[:, None]
    sign = torch.where(at % 3 == 0, -1, 1).to(dt)
    x, res = sign * (at % 4 + 1).to(dt), sign * (at % 5).to(dt)
    g = torch.full((1,), 0.5, dtype=dt, device="cuda")
    y, h = binding.rms_norm(x, g, residual=res, eps=0.0)
    assert torch.equal(h, x + res) and torch.equal(y, 0.5 * sign)
    dy, dh = (at % 7 - 3).to(dt), (at % 2).to(dt)
    dx, none = binding.rms_norm_grad(dy, sign, g, dh=dh, eps=3.0, need_gain=False)
    assert none is None and torch.equal(dx, 0.375 * (0.5 * dy) + dh)


def call(entry, args, space=None):
    lib = binding.load_library()
    n = 0 if space is None else space.numel()
    rc = getattr(lib, entry)(C.byref(args), None if n == 0 else space.data_ptr(), n, torch.cuda.current_stream().cuda_stream)
    assert rc == 0, lib.stgn_last_error(None)


def beside(rows, width, at, more):
    """Rows of bytes `more` longer than their width that start `at` bytes in, all 99: (the buffer, its rows, those of the width)."""
    ld = width + more
    buffer = torch.full((rows * ld + at + 64,), 99, dtype=torch.int8, device="cuda")
    return buffer, buffer[at:at + rows * ld].view(rows, ld), ld


@pytest.mark.parametrize("dt", ALL, ids=str)
@pytest.mark.parametrize("at,more", [(0, 16), (1, 3), (2, 1), (3, 6)])
@pytest.mark.parametrize("width", [1, 5, 13, 200, 1027, 5000, 40001])
def test_8_bit_rows_that_lie_apart_and_start_anywhere(width, at, more, dt):
    """The norm's q and that of a matrix's rows, at every start of four bytes; what lies between rows stays as it was."""
    x, res, gain, *_ = make(9, width, dt)
    for norm in (True, False):
        want = binding.rms_norm_i8(x, gain, residual=res) if norm else binding.quantize(x)
        buffer, rows, ld = beside(9, width, at, more)
        scale = torch.empty(9, device="cuda")
        if norm:
            call("stgn_rms_norm", binding.RmsNormArgs(dtype=ALL.index(dt), rows=9, width=width, eps=refs.EPS, ld_x=width, ld_residual=width, ld_q=ld, x=x.data_ptr(),
                                                      residual=res.data_ptr(), gain=gain.data_ptr(), q=rows.data_ptr(), scale=scale.data_ptr()))
        else:
            call("stgn_quantize", binding.QuantizeArgs(dtype=ALL.index(dt), rows=9, width=width, ld_x=width, ld_q=ld, x=x.data_ptr(), q=rows.data_ptr(), scale=scale.data_ptr()))
        assert torch.equal(rows[:, :width], want[0]) and torch.equal(scale, want[1])
        rows[:, :width] = 99
        assert (buffer == 99).all()


@pytest.mark.parametrize("dt", ALL, ids=str)
@pytest.mark.parametrize("at,more", [(0, 16), (1, 3)])
@pytest.mark.parametrize("size", [(7, 70), (129, 5), (1000, 65), (1025, 64), (2050, 70)], ids=str)
def test_8_bit_columns_that_lie_apart_and_start_anywhere(size, at, more, dt):
    """The same of a matrix's columns, in one kernel and in two."""
    x, *_ = make(*size, dt)
    rows, width = size
    want = binding.quantize(x, columns=True)
    buffer, lines, ld = beside(width, rows, at, more)
    scale = torch.empty(width, device="cuda")
    args = binding.QuantizeArgs(dtype=ALL.index(dt), columns=1, rows=rows, width=width, ld_x=width, ld_q=ld, x=x.data_ptr(), q=lines.data_ptr(), scale=scale.data_ptr())
    n = C.c_size_t(0)
    assert binding.load_library().stgn_quantize_workspace(C.byref(args), C.byref(n)) == 0
    call("stgn_quantize", args, torch.empty(n.value, dtype=torch.uint8, device="cuda") if n.value else None)
    assert torch.equal(lines[:, :rows], want[0]) and torch.equal(scale, want[1])
    lines[:, :rows] = 99
    assert (buffer == 99).all()


@pytest.mark.parametrize("dt", ALL, ids=str)
@pytest.mark.parametrize("width", [13, 1027, 40001])
def test_the_sum_is_not_handed_out_where_it_is_not_asked_for(width, dt):
    """A residual and no h: y, or y's numbers in 8 bits, as beside h."""
    x, res, gain, *_ = make(9, width, dt)
    y, scale, q = torch.empty_like(x), torch.empty(9, device="cuda"), torch.empty(9, width, dtype=torch.int8, device="cuda")
    same = dict(dtype=ALL.index(dt), rows=9, width=width, eps=refs.EPS, ld_x=width, ld_residual=width, ld_y=width, ld_q=width, x=x.data_ptr(), residual=res.data_ptr(),
                gain=gain.data_ptr())
    call("stgn_rms_norm", binding.RmsNormArgs(**same, y=y.data_ptr()))
    assert torch.equal(y, binding.rms_norm(x, gain, residual=res)[0])
    call("stgn_rms_norm", binding.RmsNormArgs(**same, q=q.data_ptr(), scale=scale.data_ptr()))
    want = binding.rms_norm_i8(x, gain, residual=res)
    assert torch.equal(q, want[0]) and torch.equal(scale, want[1])
