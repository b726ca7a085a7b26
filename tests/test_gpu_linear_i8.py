"""The dense product of operands in 8 bits against 64 bits (bounds: block_refs)."""
import ctypes as C

import pytest
import torch

import block_refs as refs
from operator_refs import within
from paper_2603_21090_amd import binding

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]
# rows, d_in, d_out: single numbers, rows and columns, sums shorter than 16 bytes and that end with a part of them, both sides of every tile
# and number of rows that has a kernel of its own, sums long enough to be split
SIZES = [(1, 1, 1), (1, 100, 1), (3, 7, 5), (1, 4096, 96), (5, 333, 129), (16, 64, 64), (17, 128, 16), (31, 129, 33), (33, 1000, 47), (64, 64, 64), (65, 63, 127),
         (200, 200, 100), (17, 31, 1), (129, 1, 65), (300, 257, 140), (2, 2000, 257), (16, 1027, 64), (1000, 40, 3), (700, 130, 257), (9, 640, 1030),
         (4, 8200, 40), (70, 20000, 33), (128, 4096, 128), (257, 384, 300)]


def make(rows, d_in, d_out, dt, seed=0):
    g = torch.Generator().manual_seed(1000 * rows + 10 * d_in + d_out + seed)
    n = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    i = lambda *s: torch.randint(-127, 128, s, generator=g, dtype=torch.int8)  # noqa: E731
    xs, ws = n(rows).abs() / 100, n(d_out).abs() / 100 * d_in ** -0.5
    return i(rows, d_in), xs, i(d_out, d_in), ws, n(d_out).to(dt), n(rows, d_out).to(dt)


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("name,bias,residual", [("none", False, False), ("relu", True, False), ("gelu", True, True), ("silu", False, True)])
def test_forward(size, dt, name, bias, residual):
    x, xs, w, ws, b, r = make(*size, dt)
    b, r = b if bias else None, r if residual else None
    got = binding.linear_i8(x.cuda(), xs.cuda(), w.cuda(), ws.cuda(), bias=b if b is None else b.cuda(), activation=name,
                            residual=r if r is None else r.cuda(), dtype=dt)
    assert got.dtype == dt
    within(got, refs.linear_i8(x, xs, w, ws, b, name, r, dt), "y")


@pytest.mark.parametrize("size", SIZES + [(4100, 256, 4104), (3970, 320, 4360), (4000, 100, 1030), (20000, 70, 200)], ids=str)
def test_sums_are_exact(size):
    """Scales of one, no epilogue: fp32 holds the sums as they are where they stay below 2^24."""
    x, _, w, *_ = make(*size, torch.float32)
    most = min(127, int((2 ** 24 / size[1]) ** 0.5))
    x, w = x.clamp(-most, most).cuda(), w.clamp(-most, most).cuda()
    y = binding.linear_i8(x, torch.ones(size[0], device="cuda"), w, torch.ones(size[2], device="cuda"), dtype=torch.float32)
    assert torch.equal(y.double(), x.double() @ w.double().t())


@pytest.mark.parametrize("size", [(3, 131071, 17), (70, 131071, 65), (300, 131071, 257)], ids=str)
def test_the_largest_sums(size):
    """All numbers -128: 2,147,467,264 a sum, the largest that 32 bits hold."""
    x = torch.full(size[:2], -128, dtype=torch.int8, device="cuda")
    w = torch.full((size[2], size[1]), -128, dtype=torch.int8, device="cuda")
    one = torch.ones(max(size), device="cuda")
    for by, want in ((w, 131071.0 * 16384), (-1 - w, -131071.0 * 128 * 127)):
        y = binding.linear_i8(x, one[:size[0]], by, one[:size[2]], dtype=torch.float32)
        assert (y == torch.tensor(want).float().item()).all()


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("size", [(9, 77, 45), (90, 77, 45), (40, 1000, 300), (300, 2051, 129), (2060, 384, 4100)], ids=str)
def test_rows_that_lie_apart_and_start_anywhere(size, dt):
    """Columns of wider matrices that start one byte or element in, beside numbers that would show."""
    x, xs, w, ws, b, r = make(*size, dt)

    def inside(t, fill):
        wide = torch.full((t.shape[0], t.shape[1] + 9), fill, dtype=t.dtype, device="cuda")
        wide[:, 1:1 + t.shape[1]] = t.cuda()
        return wide[:, 1:1 + t.shape[1]]
    got = binding.linear_i8(inside(x, 127), xs.cuda(), inside(w, 127), ws.cuda(), bias=b.cuda(), activation="silu", residual=inside(r, float("nan")))
    within(got, refs.linear_i8(x, xs, w, ws, b, "silu", r, dt), "y")


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("size", [(3, 2000, 65), (90, 77, 45), (300, 500, 200), (2100, 256, 4104)], ids=str)
def test_y_in_the_residuals_place(size, dt):
    """Residual and y are the same columns of a wider matrix, the others stay as they were."""
    rows, d_in, d_out = size
    x, xs, w, ws, b, r = make(*size, dt)
    m = torch.full((rows, d_out + 4), 7.0, dtype=dt, device="cuda")
    m[:, 1:1 + d_out] = r.cuda()
    X, XS, W, WS, B = (t.cuda() for t in (x, xs, w, ws, b))
    p = m.data_ptr() + m.element_size()
    a = binding.LinearI8Args(dtype=TYPES.index(dt), activation=1, rows=rows, d_in=d_in, d_out=d_out, ld_x=d_in, ld_w=d_in, ld_residual=d_out + 4, ld_y=d_out + 4,
                             x=X.data_ptr(), w=W.data_ptr(), x_scale=XS.data_ptr(), w_scale=WS.data_ptr(), bias=B.data_ptr(), residual=p, y=p)
    lib, n = binding.load_library(), C.c_size_t(0)
    assert lib.stgn_linear_quantized_workspace(C.byref(a), C.byref(n)) == 0
    space = torch.empty(n.value, dtype=torch.uint8, device="cuda")
    assert lib.stgn_linear_quantized(C.byref(a), space.data_ptr() if n.value else None, n.value, torch.cuda.current_stream().cuda_stream) == 0, lib.stgn_last_error(None)
    within(m[:, 1:1 + d_out], refs.linear_i8(x, xs, w, ws, b, "relu", r, dt), "y")
    for c in (0, d_out + 1, d_out + 2, d_out + 3):
        assert (m[:, c] == 7).all()


@pytest.mark.parametrize("dt", TYPES, ids=str)
def test_no_rows(dt):
    x, w = torch.empty(0, 20, dtype=torch.int8, device="cuda"), torch.ones(30, 20, dtype=torch.int8, device="cuda")
    assert binding.linear_i8(x, torch.empty(0, device="cuda"), w, torch.ones(30, device="cuda"), dtype=dt).shape == (0, 30)


@pytest.mark.parametrize("rows", [5, 40, 300])
def test_scales_that_are_no_numbers_stay_in_their_rows_and_columns(rows):
    x, xs, w, ws, *_ = make(rows, 200, 70, torch.float32)
    xs[3], ws[11] = float("nan"), float("inf")
    y = binding.linear_i8(x.cuda(), xs.cuda(), w.cuda(), ws.cuda(), dtype=torch.float32).cpu()
    assert y[3].isnan().all() and not y[:, 11].isfinite().any()
    y[3], y[:, 11] = 0.0, 0.0
    assert y.isfinite().all()


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("rows", [3, 40, 300])
def test_the_same_bits_again_on_another_stream_and_in_a_graph(rows, dt):
    x, xs, w, ws, b, r = (t.cuda() for t in make(rows, 3000, 200, dt))

    def step():
        return binding.linear_i8(x, xs, w, ws, bias=b, activation="gelu", residual=r)
    first = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = step()
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(first, other)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = step()
    for turn in range(3):
        x.mul_(-1 if turn else 1)                             # new contents for every replay
        graph.replay()
        eager = step()
        torch.cuda.synchronize()
        assert torch.equal(kept, eager)


@pytest.mark.parametrize("size", [(5, 4096, 300), (200, 70, 40), (4096, 256, 4096)], ids=str)
def test_rows_past_32_bits(size):
    """x and w as columns of matrices so wide that their last rows lie past 2^31 bytes, y and the residual past 2^31 numbers."""
    rows, d_in, d_out = size
    dt = torch.bfloat16
    x, xs, w, ws, b, r = make(*size, dt)

    def far(t):
        ld = (1 << 31) // (t.shape[0] - 1) + t.shape[1] + 2
        buffer = torch.empty(t.shape[0] * ld, dtype=t.dtype, device="cuda").view(t.shape[0], ld)
        buffer[:, 1:1 + t.shape[1]].copy_(t.cuda())
        return buffer[:, 1:1 + t.shape[1]]
    got = binding.linear_i8(far(x), xs.cuda(), far(w), ws.cuda(), bias=b.cuda(), residual=far(r))
    within(got, refs.linear_i8(x, xs, w, ws, b, "none", r, dt), "y")


# one size and more for each kernel and its edges: fragments of every shape; tiles of 64 x 64 in one sum and in several; 128 x 128 directly, with k that ends
# inside a tile, in one sum and in several; 256 x 256, whole and cut; outputs of few columns and a part of an eight; rows that no
# 16 bytes align laid out again for each of them
KINDS = [(16, 512, 4000), (33, 512, 2000), (100, 640, 1250), (60, 1500, 8100), (1000, 272, 1000), (500, 1027, 900), (300, 3001, 200), (2100, 4001, 2050), (2100, 1040, 2050),
         (200, 4112, 4096), (1500, 2048, 1530), (2000, 512, 4090), (3900, 1088, 4090), (4096, 1024, 4096), (25000, 704, 5), (60000, 1024, 5), (60000, 1024, 13), (60000, 1024, 69), (40000, 1024, 135),
         (4000, 1001, 1000), (8190, 1023, 2048), (1999, 2050, 2001), (20000, 33, 2000), (20000, 17, 2000), (20000, 17, 2003)]


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("size", KINDS, ids=str)
def test_every_kernel(size, dt):
    x, xs, w, ws, b, r = (t.cuda() for t in make(*size, dt))
    cpu = lambda t: tuple(v.cpu() for v in t)  # noqa: E731
    within(binding.linear_i8(x, xs, w, ws, bias=b, activation="gelu", residual=r), cpu(refs.linear_i8(x, xs, w, ws, b, "gelu", r, dt)), "y")
    within(binding.linear_i8(x, xs, w, ws, dtype=dt), cpu(refs.linear_i8(x, xs, w, ws, None, "none", None, dt)), "no epilogue")


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("size", [(33, 512, 2000), (300, 3001, 200), (2100, 1040, 2050), (200, 4112, 4096), (1500, 2048, 1530), (3900, 1088, 4090), (1999, 2050, 2001)], ids=str)
def test_y_over_the_residual(size, dt):
    """The C entry's y may be exactly the residual."""
    x, xs, w, ws, b, r = (t.cuda() for t in make(*size, dt))
    want = binding.linear_i8(x, xs, w, ws, bias=b, activation="gelu", residual=r)
    rows, d_in, d_out = size
    args = binding._PACK_LINEAR_I8.pack(binding._dtype_code(r), binding.ACTIVATIONS["gelu"], rows, d_in, d_out, 0, d_in, d_in, d_out, d_out, x.data_ptr(), w.data_ptr(),
                                        xs.data_ptr(), ws.data_ptr(), b.data_ptr(), r.data_ptr(), r.data_ptr())
    L = binding.load_library()
    binding._run_operator(L.stgn_linear_quantized_workspace, L.stgn_linear_quantized, args, None, r.device)
    assert torch.equal(r, want)


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("at", [0, 1, 8, 16])
def test_rows_that_start_anywhere(at, dt):
    """Whole pieces but for where the first row lies, or how far apart rows are; the residual is only read."""
    x, xs, w, ws, b, r = (t.cuda() for t in make(2100, 1040, 2050, dt))
    for ld in (1040 + 16, 1040 + 19):
        X = torch.empty(2100 * ld + 16, dtype=torch.int8, device="cuda")[at:at + 2100 * ld].view(2100, ld)[:, :1040]
        X.copy_(x)
        y = r.clone()
        got = binding.linear_i8(X, xs, w, ws, bias=b, activation="silu", residual=y)
        within(got, tuple(v.cpu() for v in refs.linear_i8(x, xs, w, ws, b, "silu", r, dt)), "y")
        assert torch.equal(y, r)


@pytest.mark.parametrize("size", [(260, 32784, 260), (1500, 2048, 1500)], ids=str)
def test_rows_in_whole_pieces_that_lie_far_apart(size):
    """Rows 2^23 - 16 bytes apart: a tile's last row lies 2^30 bytes and more from its first."""
    x, xs, w, ws, b, _ = (t.cuda() for t in make(*size, torch.float32))
    ld = (1 << 23) - 16
    X = torch.empty(size[0] * ld, dtype=torch.int8, device="cuda").view(size[0], ld)[:, :size[1]]
    X.copy_(x)
    W = torch.empty(260 * ld if size[2] == 260 else w.numel(), dtype=torch.int8, device="cuda").view(size[2], -1)[:, :size[1]]
    W.copy_(w)
    got = binding.linear_i8(X, xs, W, ws, bias=b)
    within(got, tuple(v.cpu() for v in refs.linear_i8(x, xs, w, ws, b, "none", None, torch.float32)), "y")
    assert torch.equal(got, binding.linear_i8(x, xs, w, ws, bias=b))
