"""The dense product with its epilogue and its gradients against 64 bits (bounds: operator_refs)."""
import pytest
import torch

import operator_refs as refs
from paper_2603_21090_amd import binding

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]
# rows, d_in, d_out: single numbers, single rows and columns, odd sizes on both sides of a tile, tails shorter than 16 bytes,
# sums long enough to be split, more than one tile each way
SIZES = [(1, 1, 1), (1, 100, 1), (3, 7, 5), (1, 4096, 96), (5, 333, 129), (64, 64, 64), (65, 63, 127), (200, 200, 100), (17, 31, 1),
         (129, 1, 65), (300, 257, 140), (2, 2000, 257), (16, 1027, 64), (1000, 40, 3), (700, 130, 257), (9, 640, 1030)]


def make(rows, d_in, d_out, dt, seed=0):
    g = torch.Generator().manual_seed(1000 * rows + 10 * d_in + d_out + seed)
    n = lambda *s: torch.randn(*s, generator=g).to(dt)  # noqa: E731
    return n(rows, d_in), (n(d_in, d_out).float() * d_in ** -0.5).to(dt), n(d_out), n(rows, d_out), n(rows, d_out)


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("name,bias,residual,keep", [("none", False, False, False), ("relu", True, False, True), ("gelu", True, True, True),
                                                     ("silu", False, True, False)])
def test_forward(size, dt, name, bias, residual, keep):
    x, w, b, r, _ = make(*size, dt)
    got = binding.linear(x.cuda(), w.cuda(), bias=b.cuda() if bias else None, activation=name, residual=r.cuda() if residual else None, keep_pre=keep)
    y, z = refs.linear(x, w, b if bias else None, name, r if residual else None)
    refs.within(got[0] if keep else got, y, "y")
    if keep:
        refs.within(got[1], z, "pre")


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("size", SIZES + [(5000, 24, 40), (3001, 33, 17)], ids=str)
@pytest.mark.parametrize("name", ["none", "relu", "gelu", "silu"])
def test_gradients(size, dt, name):
    x, w, b, z, dy = make(*size, dt)
    got = binding.linear_grad(dy.cuda(), x.cuda(), w.cuda(), activation=name, pre=z.cuda() if name != "none" else None)
    for g, want, what in zip(got, refs.linear_grad(dy, x, w, name, z), ("dx", "dw", "db")):
        refs.within(g, want, what)


@pytest.mark.parametrize("dt", TYPES, ids=str)
def test_only_the_gradients_asked_for(dt):
    x, w, b, z, dy = (t.cuda() for t in make(130, 70, 50, dt))
    full = binding.linear_grad(dy, x, w, activation="gelu", pre=z)
    for need in [(True, False, False), (False, True, False), (False, False, True), (True, False, True)]:
        got = binding.linear_grad(dy, x, w, activation="gelu", pre=z, need_x=need[0], need_w=need[1], bias=need[2])
        for g, f, n in zip(got, full, need):
            assert torch.equal(g, f) if n else g is None


@pytest.mark.parametrize("dt", TYPES, ids=str)
def test_rows_that_lie_apart_and_start_anywhere(dt):
    """Columns of wider matrices that start one element in: no row is aligned, and the numbers beside them are NaN."""
    x, w, b, r, dy = make(90, 77, 45, dt)

    def inside(t):
        wide = torch.full((t.shape[0], t.shape[1] + 9), float("nan"), dtype=dt, device="cuda")
        wide[:, 1:1 + t.shape[1]] = t.cuda()
        return wide[:, 1:1 + t.shape[1]]
    y, z = refs.linear(x, w, b, "silu", r)
    got = binding.linear(inside(x), inside(w), bias=b.cuda(), activation="silu", residual=inside(r), keep_pre=True)
    refs.within(got[0], y, "y")
    refs.within(got[1], z, "pre")
    for g, want, what in zip(binding.linear_grad(inside(dy), inside(x), inside(w), activation="silu", pre=inside(r)),
                             refs.linear_grad(dy, x, w, "silu", r), ("dx", "dw", "db")):
        refs.within(g, want, what)


@pytest.mark.parametrize("dt", TYPES, ids=str)
def test_no_rows(dt):
    x, w = torch.empty(0, 20, dtype=dt, device="cuda"), torch.ones(20, 30, dtype=dt, device="cuda")
    y, z = binding.linear(x, w, keep_pre=True)
    assert y.shape == z.shape == (0, 30)
    dx, dw, db = binding.linear_grad(y, x, w)
    assert dx.shape == (0, 20) and not dw.any() and not db.any()


def test_infinities_and_nan_stay_in_their_rows():
    x, w, *_ = make(70, 40, 33, torch.float32)
    x[3, 5], x[40, 0] = float("inf"), float("nan")
    y = binding.linear(x.cuda(), w.cuda(), activation="relu").cpu()
    rows = torch.ones(70, dtype=torch.bool)
    rows[3] = rows[40] = False
    refs.within(y[rows], tuple(t for t in refs.linear(x[rows], w, None, "relu", None)[0]), "y")
    assert not torch.isfinite(y[3]).all()


@pytest.mark.parametrize("dt", TYPES, ids=str)
def test_the_same_bits_again_on_another_stream_and_in_a_graph(dt):
    x, w, b, z, dy = (t.cuda() for t in make(300, 500, 200, dt))

    def step():
        y, pre = binding.linear(x, w, bias=b, activation="gelu", residual=z, keep_pre=True)
        return (y, pre) + binding.linear_grad(dy, x, w, activation="gelu", pre=pre)
    first = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = step()
    torch.cuda.current_stream().wait_stream(side)
    for a, c in zip(first, other):
        assert torch.equal(a, c)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = step()
    for turn in range(3):
        x.mul_(-1 if turn else 1)                             # new contents for every replay
        graph.replay()
        eager = step()
        torch.cuda.synchronize()
        for a, c in zip(kept, eager):
            assert torch.equal(a, c)


# products of many tiles: 256 x 256 (16-bit types, whole tiles of k; edges in both directions), 128 rows by 128, 112, 96 and 64 columns
LARGE = [(4100, 64, 4104), (3970, 192, 4360), (4000, 100, 1030), (33000, 20, 112), (33000, 33, 96), (33000, 20, 40), (20000, 70, 200)]


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("size", LARGE, ids=str)
def test_forward_of_many_tiles(size, dt):
    x, w, b, r, _ = make(*size, dt)
    y, z = refs.linear(x, w, b, "gelu", r)
    got = binding.linear(x.cuda(), w.cuda(), bias=b.cuda(), activation="gelu", residual=r.cuda(), keep_pre=True)
    refs.within(got[0], y, "y")
    refs.within(got[1], z, "pre")
    refs.within(binding.linear(x.cuda(), w.cuda()), refs.linear(x, w, None, "none", None)[0], "no epilogue")


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("size", [(4100, 4099, 64), (128, 4104, 4112), (192, 4360, 3976), (20000, 372, 200), (17000, 300, 420), (4000, 1030, 100)], ids=str)
def test_gradients_of_many_tiles(size, dt):
    """dx with an odd width, dW from whole tiles of k, long sums cut for 128-row tiles."""
    x, w, b, z, dy = make(*size, dt)
    got = binding.linear_grad(dy.cuda(), x.cuda(), w.cuda(), activation="relu", pre=z.cuda())
    for g, want, what in zip(got, refs.linear_grad(dy, x, w, "relu", z), ("dx", "dw", "db")):
        refs.within(g, want, what)


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("size", [(90, 77, 45), (3, 2000, 65), (4200, 128, 4104)], ids=str)
def test_columns_of_one_matrix(size, dt):
    """x, pre, residual and y (in the residual's place) as columns of one matrix: the columns between them stay as they were."""
    import ctypes as C
    rows, d_in, d_out = size
    x, w, b, r, _ = make(*size, dt)
    ld, at = d_in + 2 * d_out + 5, (1, d_in + 3, d_in + d_out + 4)
    m = torch.full((rows, ld), 7.0, dtype=dt, device="cuda")
    m[:, at[0]:at[0] + d_in], m[:, at[2]:at[2] + d_out] = x.cuda(), r.cuda()
    w, b = w.cuda(), b.cuda()
    p = [m.data_ptr() + c * m.element_size() for c in at]
    a = binding.LinearArgs(dtype=TYPES.index(dt), activation=3, rows=rows, d_in=d_in, d_out=d_out, ld_x=ld, ld_w=d_out, ld_residual=ld, ld_y=ld, ld_pre=ld,
                           x=p[0], w=w.data_ptr(), bias=b.data_ptr(), residual=p[2], y=p[2], pre=p[1])
    lib, n = binding.load_library(), C.c_size_t(0)
    assert lib.stgn_linear_workspace(C.byref(a), C.byref(n), None) == 0
    ws = torch.empty(n.value, dtype=torch.uint8, device="cuda")
    assert lib.stgn_linear(C.byref(a), ws.data_ptr() if n.value else None, n.value, torch.cuda.current_stream().cuda_stream) == 0, lib.stgn_last_error(None)
    y, z = refs.linear(x, w.cpu(), b.cpu(), "silu", r)
    refs.within(m[:, at[2]:at[2] + d_out], y, "y")
    refs.within(m[:, at[1]:at[1] + d_out], z, "pre")
    assert torch.equal(m[:, at[0]:at[0] + d_in].cpu(), x)
    for c in (0, at[0] + d_in, at[0] + d_in + 1, at[1] + d_out):
        assert (m[:, c] == 7).all()


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("d_in,d_out", [(4096, 4096), (4104, 4160), (6000, 200)])
@pytest.mark.parametrize("name", ["none", "gelu"])
def test_no_rows_of_wide_layers(name, d_in, d_out, dt):
    """Outputs of many tiles from sums of nothing: zeros, and no operand is read (empty tensors have no address)."""
    x, w = torch.empty(0, d_in, dtype=dt, device="cuda"), torch.ones(d_in, d_out, dtype=dt, device="cuda")
    z = torch.empty(0, d_out, dtype=dt, device="cuda")
    dx, dw, db = binding.linear_grad(z, x, w, activation=name, pre=z if name != "none" else None)
    assert dx.shape == (0, d_in) and dw.shape == w.shape and not dw.any() and db.shape == (d_out,) and not db.any()
    assert binding.linear(x, w, activation=name).shape == (0, d_out)


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("size", [(200, 70, 40), (4096, 64, 4096), (40000, 72, 200)], ids=str)
def test_rows_past_32_bits(size, dt):
    """x and dy as columns of matrices so wide that their last rows lie past 2^31 numbers."""
    rows, d_in, d_out = size
    x, w, b, _, dy = make(*size, dt)
    ld = (1 << 31) // (rows - 1) + d_in + d_out + 2
    buffer = torch.empty(rows * ld, dtype=dt, device="cuda").view(rows, ld)
    X, DY = buffer[:, 1:1 + d_in], buffer[:, 1 + d_in:1 + d_in + d_out]
    X.copy_(x.cuda())
    DY.copy_(dy.cuda())
    assert (rows - 1) * ld >= 1 << 31
    refs.within(binding.linear(X, w.cuda(), bias=b.cuda()), refs.linear(x, w, b, "none", None)[0], "y")
    for g, want, what in zip(binding.linear_grad(DY, X, w.cuda()), refs.linear_grad(dy, x, w, "none", None), ("dx", "dw", "db")):
        refs.within(g, want, what)
