"""The norm of rows, its gradient and matrices in 8 bits against 64 bits (bounds: block_refs)."""
import ctypes as C

import pytest
import torch

import block_refs as refs
from operator_refs import within
from paper_2603_21090_amd import binding

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]
# single numbers and rows; widths around every number of lanes and pieces that hold a row, in both sizes of an element; rows that end with a part
# of 16 bytes; rows longer than any number of lanes holds
SIZES = [(1, 1), (1, 4096), (2, 3), (17, 8), (300, 5), (33, 63), (65, 100), (129, 128), (40, 200), (7, 255), (9, 257), (5, 333), (70, 512), (3, 777), (2, 1024),
         (6, 1025), (3, 1500), (2, 2047), (3, 4099), (5, 8191), (2, 8192), (3, 16380), (2, 16389), (2, 32768), (3, 40001)]


def make(rows, width, dt, seed=0):
    g = torch.Generator().manual_seed(1000 * rows + width + seed)
    n = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    return n(rows, width).to(dt), n(rows, width).to(dt), (1 + n(width) / 4).to(dt), n(rows, width).to(dt), n(rows, width).to(dt)


def cuda(*tensors):
    return [None if t is None else t.cuda() for t in tensors]


def check_eight(q, scale, y32):
    """q and scale are those of the fp32 rows."""
    want_q, want_scale = refs.eight(y32.cpu())
    assert torch.equal(q.cpu(), want_q)
    assert torch.equal(scale.cpu().nan_to_num(-1), want_scale.nan_to_num(-1))


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_forward(size, dt):
    x, res, gain, *_ = make(*size, dt)
    X, R, G = cuda(x, res, gain)
    within(binding.rms_norm(X, G), refs.rms_norm(x, None, gain)[0], "y")
    y, h = binding.rms_norm(X, G, residual=R, eps=0.5)
    want = refs.rms_norm(x, res, gain, 0.5)
    within(y, want[0], "y of the sum")
    within(h, want[1], "h")


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_forward_in_8_bits(size, dt):
    """The same y beside it; q within half a step of 127 y / max |y|, whose fp32 values are 12 u apart at most; in fp32, where y is handed out as the
    kernel had it, q is exactly its rounding."""
    x, res, gain, *_ = make(*size, dt)
    X, R, G = cuda(x, res, gain)
    for residual, r in ((None, None), (R, res)):
        got = binding.rms_norm_i8(X, G, residual=residual, keep_y=True)
        q, scale, y = got[0], got[1], got[-1]
        plain = binding.rms_norm(X, G, residual=residual)
        assert torch.equal(y, plain if residual is None else plain[0])
        if residual is not None:
            assert torch.equal(got[2], plain[1])
        want = refs.rms_norm(x, r, gain)[0][0]
        top = want.abs().amax(1, keepdim=True)
        assert ((q.cpu().double() - 127 * want / top).abs() <= 0.5 + 127 * 14 * refs.U).all()
        assert ((scale.cpu().double() - top[:, 0] / 127).abs() <= 8 * refs.U * top[:, 0] / 127).all()
        if dt == torch.float32:
            check_eight(q, scale, y)
        again = binding.rms_norm_i8(X, G, residual=residual)                # without y
        assert torch.equal(again[0], q) and torch.equal(again[1], scale)


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("size", SIZES + [(3000, 40), (5000, 200), (2500, 1030), (200, 16400)], ids=str)
def test_gradients(size, dt):
    _, h, gain, dy, dh = make(*size, dt)
    H, G, DY, DH = cuda(h, gain, dy, dh)
    for got, want, name in zip(binding.rms_norm_grad(DY, H, G), refs.rms_norm_grad(dy, h, gain, None), ("dx", "dgain")):
        within(got, want, name)
    for got, want, name in zip(binding.rms_norm_grad(DY, H, G, dh=DH, eps=0.5), refs.rms_norm_grad(dy, h, gain, dh, 0.5), ("dx with dh", "dgain")):
        within(got, want, name)


def test_gradients_against_differences():
    """The loss sum(dy y) at h +- step: central differences are off by step^2 / 6 of the third derivative, and by the outputs' roundings over the
    step (both in 64 bits here: the plain form's loss at points that the fp32 gradient is evaluated at)."""
    _, h, gain, dy, _ = make(3, 37, torch.float32)
    dx, dg = (t.cpu().double() for t in binding.rms_norm_grad(*cuda(dy, h, gain)))

    def loss(h, gain):
        return (dy.double() * h / torch.sqrt((h * h).mean(1, keepdim=True) + refs.EPS) * gain).sum()
    step = 1e-5
    for i in range(0, h.numel(), 7):
        at = torch.zeros(h.numel(), dtype=torch.float64)
        at[i] = step
        at = at.view_as(h)
        diff = (loss(h.double() + at, gain.double()) - loss(h.double() - at, gain.double())) / (2 * step)
        assert abs(diff - dx.view(-1)[i]) <= 1e-6 * (1 + abs(diff))
    for j in range(0, 37, 5):
        at = torch.zeros(37, dtype=torch.float64)
        at[j] = step
        diff = (loss(h.double(), gain.double() + at) - loss(h.double(), gain.double() - at)) / (2 * step)
        assert abs(diff - dg[j]) <= 1e-6 * (1 + abs(diff))


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("width", [40, 1030, 5000, 40001])
def test_only_the_gradients_asked_for(width, dt):
    _, h, gain, dy, dh = cuda(*make(130, width, dt))
    dx, dg = binding.rms_norm_grad(dy, h, gain, dh=dh)
    assert torch.equal(binding.rms_norm_grad(dy, h, gain, dh=dh, need_gain=False)[0], dx)
    assert torch.equal(binding.rms_norm_grad(dy, h, gain, dh=dh, need_x=False)[1], dg)
    assert binding.rms_norm_grad(dy, h, gain, need_x=False, need_gain=False) == (None, None)


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("size", [s for s in SIZES if s[0] * s[1] < 50000] + [(1000, 70), (2, 40001)], ids=str)
def test_rows_in_8_bits(size, dt):
    x, *_ = make(*size, dt)
    x[0, 0] = 0.0
    check_eight(*binding.quantize(x.cuda()), x.float())


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("size", [(1, 1), (1, 300), (300, 1), (3, 7), (127, 65), (128, 64), (129, 63), (1000, 257), (1023, 65), (1024, 200), (1025, 64), (4096, 96), (33, 5000), (2050, 770)], ids=str)
def test_columns_in_8_bits(size, dt):
    x, *_ = make(*size, dt)
    q, scale = binding.quantize(x.cuda(), columns=True)
    assert q.shape == (size[1], size[0])
    check_eight(q, scale, x.float().t())


@pytest.mark.parametrize("columns", [False, True])
def test_halves_go_to_the_even_neighbour(columns):
    """Quotients that are whole and a half, of maxima whose 127th is no fp32 number."""
    tops = torch.tensor([127.0, 254.0, 3 * 127.0, 127 / 1024.0, 127 * 2.0 ** 100, 127 * 2.0 ** -130, 1.0, 3.0])
    k = torch.arange(-126, 126).float() + 0.5
    x = torch.cat([tops[:6, None], tops[:6, None] / 127 * k], 1)
    check = torch.round(k)
    q, scale = binding.quantize((x.t().contiguous() if columns else x).cuda(), columns=columns)
    assert (q.cpu()[:, 0] == 127).all()
    assert torch.equal(q.cpu()[:, 1:].float(), check.expand(6, -1))
    g = torch.Generator().manual_seed(3)
    y = torch.randn(2000, 64, generator=g)
    y = y * (2.0 ** torch.randint(-140, 120, (2000, 1), generator=g))
    check_eight(*binding.quantize((y.t().contiguous() if columns else y).cuda(), columns=columns), y)


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("width", [40, 600, 5000, 40001])
def test_rows_of_zeros_infinities_and_nan(width, dt):
    """Zeros have scale 0; a row with an infinity or a NaN has scale NaN, zeros in q, and is no other row's concern."""
    x, _, gain, *_ = make(6, width, dt)
    x[1], x[2, 7], x[3, width - 1], x[4, 0] = 0.0, float("inf"), float("nan"), -float("inf")
    X, G = cuda(x, gain)
    for q, scale in (binding.quantize(X), binding.rms_norm_i8(X, G)):
        q, scale = q.cpu(), scale.cpu()
        assert scale[1] == 0 and not q[1:5].any() and scale[2:5].isnan().all()
        assert scale[[0, 5]].isfinite().all() and (q[[0, 5]].abs().amax(1) == 127).all()
    q, scale = binding.quantize(X.t().contiguous(), columns=True)
    check_eight(q, scale, x.float())
    y = binding.rms_norm(X, G)
    rows = [0, 1, 5]
    within(y[rows], refs.rms_norm(x[rows], None, gain)[0], "y")
    assert not y[1].any() and not binding.rms_norm(X[1:2], G, eps=0.0).any()
    assert y[3].isnan().all() and y[2, 7].isnan() and y[4, 0].isnan()


@pytest.mark.parametrize("bits", [0x7F800001, 0x7FBFFFFF, 0x7FFFFFFF, -0x3FFFF9, -1, 0x7F800000, -0x800000], ids=hex)
def test_every_kind_of_nan_gives_zeros(bits):
    """NaN of any payload, quiet and signalling, and the infinities: the row's or column's numbers are zeros, its scale NaN."""
    x = torch.ones(3, 300)
    x.view(torch.int32)[1, 37] = bits
    assert not x[1, 37].isfinite()
    for q, scale in (binding.quantize(x.cuda()), binding.rms_norm_i8(x.cuda(), torch.ones(300, device="cuda")), binding.quantize(x.t().contiguous().cuda(), columns=True)):
        assert not q[1].any() and scale[1].isnan() and (q[[0, 2]] == 127).all()


def test_large_and_small_numbers():
    """Squares that fp32 could not hold."""
    _, h, gain, dy, _ = make(4, 300, torch.float32)
    for size in (1e-30, 1e30, 2.0 ** 120):
        x = h * size
        within(binding.rms_norm(*cuda(x, gain), eps=0.0), refs.rms_norm(x, None, gain, 0.0)[0], "y")
        want = refs.rms_norm_grad(dy, x, gain, None, 0.0)
        got = binding.rms_norm_grad(*cuda(dy, x, gain), eps=0.0)
        within(got[0], want[0], "dx")
        within(got[1], want[1], "dgain")


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("width", [77, 1027, 4099, 40001])
def test_rows_that_lie_apart_and_start_anywhere(width, dt):
    """Columns of wider matrices that start one element in: no row is aligned, and the numbers beside them are NaN."""
    x, res, gain, dy, dh = make(9, width, dt)

    def inside(t):
        wide = torch.full((t.shape[0], t.shape[1] + 9), float("nan"), dtype=dt, device="cuda")
        wide[:, 1:1 + t.shape[1]] = t.cuda()
        return wide[:, 1:1 + t.shape[1]]
    G = gain.cuda()
    y, h = binding.rms_norm(inside(x), G, residual=inside(res))
    want = refs.rms_norm(x, res, gain)
    within(y, want[0], "y")
    within(h, want[1], "h")
    assert torch.equal(binding.rms_norm_i8(inside(x), G)[0], binding.rms_norm_i8(x.cuda(), G)[0])
    check_eight(*binding.quantize(inside(x)), x.float())
    check_eight(*binding.quantize(inside(x), columns=True), x.float().t())
    for got, want, name in zip(binding.rms_norm_grad(inside(dy), inside(x), G, dh=inside(dh)), refs.rms_norm_grad(dy, x, gain, dh), ("dx", "dgain")):
        within(got, want, name)


@pytest.mark.parametrize("dt", TYPES, ids=str)
def test_no_rows(dt):
    x, g = torch.empty(0, 20, dtype=dt, device="cuda"), torch.ones(20, dtype=dt, device="cuda")
    y, h = binding.rms_norm(x, g, residual=x)
    assert y.shape == h.shape == (0, 20)
    dx, dg = binding.rms_norm_grad(x, x, g)
    assert dx.shape == (0, 20) and dg.shape == (20,) and not dg.any()
    wide = torch.empty(0, 40001, dtype=dt, device="cuda")
    assert not binding.rms_norm_grad(wide, wide, torch.ones(40001, dtype=dt, device="cuda"))[1].any()
    q, scale = binding.quantize(x)
    assert q.shape == (0, 20) and scale.shape == (0,)
    q, scale = binding.quantize(x, columns=True)
    assert q.shape == (20, 0) and scale.shape == (20,) and not scale.any()


def norm_call(dt, rows, width, ld, **where):
    lib = binding.load_library()
    a = binding.RmsNormArgs(dtype=TYPES.index(dt), rows=rows, width=width, eps=refs.EPS, **{f"ld_{n}": ld for n in ("x", "residual", "h", "y", "q")}, **where)
    assert lib.stgn_rms_norm(C.byref(a), None, 0, torch.cuda.current_stream().cuda_stream) == 0, lib.stgn_last_error(None)


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("width", [13, 77, 1027, 4099, 8191, 40001])
def test_outputs_in_the_inputs_places(width, dt):
    """h over the residual and y over x, and the other way round; rows that end with a part of 16 bytes, beside columns that stay as they were."""
    x, res, gain, *_ = make(9, width, dt)
    G, ld = gain.cuda(), 2 * width + 5
    want = refs.rms_norm(x, res, gain)
    for h_over_x in (False, True):
        m = torch.full((9, ld), 7.0, dtype=dt, device="cuda")
        m[:, 1:1 + width], m[:, width + 3:2 * width + 3] = x.cuda(), res.cuda()
        p = [m.data_ptr() + c * m.element_size() for c in (1, width + 3)]
        norm_call(dt, 9, width, ld, x=p[0], residual=p[1], gain=G.data_ptr(), h=p[0 if h_over_x else 1], y=p[1 if h_over_x else 0])
        y, h = m[:, 1:1 + width], m[:, width + 3:2 * width + 3]
        if h_over_x:
            y, h = h, y
        within(y, want[0], "y")
        within(h, want[1], "h")
        for c in (0, width + 1, width + 2, 2 * width + 3, 2 * width + 4):
            assert (m[:, c] == 7).all()


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("width", [200, 4096])
def test_the_same_bits_again_on_another_stream_and_in_a_graph(width, dt):
    x, res, gain, dy, dh = cuda(*make(700, width, dt))

    def step():
        y, h = binding.rms_norm(x, gain, residual=res)
        return (y, h) + binding.rms_norm_i8(x, gain, residual=res) + binding.quantize(x) + binding.quantize(x, columns=True) + binding.rms_norm_grad(dy, h, gain, dh=dh)
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


@pytest.mark.parametrize("dt", TYPES, ids=str)
def test_more_rows_than_a_launch_has_workgroups_for(dt):
    """Rows of one number: y = g sign(h) but for eps; the last ones belong to a workgroup's second round."""
    rows = (1 << 24) + 37
    x = torch.randint(1, 5, (rows, 1), device="cuda").to(dt) * torch.where(torch.arange(rows, device="cuda") % 3 == 0, -1, 1).to(dt)[:, None]
    g = torch.full((1,), 0.5, dtype=dt, device="cuda")
    assert torch.equal(binding.rms_norm(x, g, eps=0.0), 0.5 * torch.sign(x))
    q, scale = binding.quantize(x)
    assert torch.equal(q, (127 * torch.sign(x.float())).to(torch.int8)) and torch.equal(scale, (x.double().abs()[:, 0] / 127).float())


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("width", [70, 5000])
def test_rows_past_32_bits(width, dt):
    """Rows of a matrix so wide that the last ones lie past 2^31 numbers."""
    rows = 200
    x, _, gain, dy, _ = make(rows, width, dt)
    ld = (1 << 31) // (rows - 1) + 2 * width + 2
    buffer = torch.empty(rows * ld, dtype=dt, device="cuda").view(rows, ld)
    X, DY = buffer[:, 1:1 + width], buffer[:, 1 + width:1 + 2 * width]
    X.copy_(x.cuda())
    DY.copy_(dy.cuda())
    G = gain.cuda()
    within(binding.rms_norm(X, G), refs.rms_norm(x, None, gain)[0], "y")
    check_eight(*binding.quantize(X), x.float())
    check_eight(*binding.quantize(X, columns=True), x.float().t())
    for got, want, name in zip(binding.rms_norm_grad(DY, X, G), refs.rms_norm_grad(dy, x, gain, None), ("dx", "dgain")):
        within(got, want, name)
