"""Dropout against its definition: the generator's words computed by the CPU (block_refs), values in 64 bits."""
import ctypes as C

import pytest
import torch

import block_refs as refs
from operator_refs import within
from paper_2603_21090_amd import binding

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]
SIZES = [(1, 1), (1, 4096), (3, 7), (17, 8), (300, 5), (33, 63), (65, 100), (129, 128), (9, 257), (2, 40001), (1000, 200)]


def make(rows, width, dt, seed=0):
    g = torch.Generator().manual_seed(1000 * rows + width + seed)
    return torch.randn(rows, width, generator=g).to(dt), torch.randn(rows, width, generator=g).to(dt)


def rng_of(seed, step):
    as_int64 = lambda v: v - (1 << 64) if v >> 63 else v  # noqa: E731
    return torch.tensor([as_int64(seed), as_int64(step)], dtype=torch.int64, device="cuda")


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 1 / 3, 1 - 2.0 ** -16, 1.0])
def test_values_and_mask(size, p, dt):
    x, res = make(*size, dt)
    seed, step, site = 0x0123456789ABCDEF, 0xFEDCBA9876543210, 65535
    mask = refs.kept(*size, p, seed, step, site)
    rng = rng_of(seed, step)
    within(binding.dropout(x.cuda(), p, rng, site=site), refs.dropout(x, p, mask, None), "y")
    within(binding.dropout(x.cuda(), p, rng, site=site, residual=res.cuda()), refs.dropout(x, p, mask, res), "y and the residual")
    within(binding.dropout_grad(res.cuda(), p, rng, site=site), refs.dropout(res, p, mask, None), "dx")


def test_the_mean_and_the_share():
    """65,536 x 64 numbers of p = 0.1 (border 6,554): the share kept is within five standard deviations, sqrt(p (1 - p) / n) = 1.5e-4 each."""
    x = torch.ones(65536, 64, device="cuda")
    y = binding.dropout(x, 0.1, rng_of(1, 2))
    share = (y != 0).double().mean().item()
    assert abs(share - (1 - 6554 / 65536)) <= 5 * 1.5e-4
    assert y[y != 0].unique().tolist() == [torch.tensor(65536 / (65536 - 6554)).item()]


def test_seed_step_site_and_place_make_the_mask():
    x = torch.ones(50, 640, device="cuda")
    first = binding.dropout(x, 0.5, rng_of(5, 6), site=7)
    assert torch.equal(first, binding.dropout(x, 0.5, rng_of(5, 6), site=7))
    others = [binding.dropout(x, 0.5, rng_of(*r), site=s) for r, s in (((6, 6), 7), ((5, 7), 7), ((5, 6), 8), ((5 + (1 << 32), 6), 7), ((5, 6 + (1 << 32)), 7))]
    for y in others:
        assert 0.45 < (y == first).double().mean().item() < 0.55
    assert torch.equal(first[:20], binding.dropout(x[:20], 0.5, rng_of(5, 6), site=7))


def test_what_is_dropped_is_zero_whatever_it_holds():
    x = torch.full((40, 77), float("nan"), device="cuda")
    mask = refs.kept(40, 77, 0.5, 1, 1, 0)
    y = binding.dropout(x, 0.5, rng_of(1, 1)).cpu()
    assert (y[~mask] == 0).all() and y[mask].isnan().all()
    assert not binding.dropout(x, 1.0, rng_of(1, 1)).any()


@pytest.mark.parametrize("dt", TYPES, ids=str)
@pytest.mark.parametrize("width", [5, 77, 1027])
def test_places_and_strides(width, dt):
    """Columns of wider matrices, and y in the place of x or of the residual, beside columns that stay as they were."""
    rows = 33
    x, res = make(rows, width, dt)
    mask = refs.kept(rows, width, 0.25, 3, 4, 9)
    want = refs.dropout(x, 0.25, mask, res)
    rng, lib = rng_of(3, 4), binding.load_library()
    for over in (0, 1):
        ld = 2 * width + 5
        m = torch.full((rows, ld), float("nan"), dtype=dt, device="cuda")
        m[:, 1:1 + width], m[:, width + 3:2 * width + 3] = x.cuda(), res.cuda()
        p = [m.data_ptr() + c * m.element_size() for c in (1, width + 3)]
        within(binding.dropout(m[:, 1:1 + width], 0.25, rng, site=9, residual=m[:, width + 3:2 * width + 3]), want, "apart")
        a = binding.DropoutArgs(dtype=TYPES.index(dt), rows=rows, width=width, site=9, p=0.25, ld_x=ld, ld_residual=ld, ld_y=ld, x=p[0], residual=p[1], y=p[over],
                                rng=rng.data_ptr())
        assert lib.stgn_dropout(C.byref(a), torch.cuda.current_stream().cuda_stream) == 0, lib.stgn_last_error(None)
        within(m[:, 1:1 + width] if over == 0 else m[:, width + 3:2 * width + 3], want, "in place")
        assert m[:, [0, width + 1, width + 2, 2 * width + 3, 2 * width + 4]].isnan().all()


def test_no_rows():
    x = torch.empty(0, 20, device="cuda")
    assert binding.dropout(x, 0.5, rng_of(1, 1), residual=x).shape == (0, 20)


@pytest.mark.parametrize("dt", TYPES, ids=str)
def test_a_captured_call_follows_the_step(dt):
    """Replays draw the mask of the step that the program wrote, as the same call outside the graph does."""
    x, res = (t.cuda() for t in make(300, 200, dt))
    rng = rng_of(11, 0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = binding.dropout(x, 0.1, rng, residual=res)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(other, binding.dropout(x, 0.1, rng, residual=res))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = binding.dropout(x, 0.1, rng, residual=res)
        dx = binding.dropout_grad(res, 0.1, rng)
        rng[1:2].add_(1)
    for step in range(4):
        want = binding.dropout(x, 0.1, rng_of(11, step), residual=res), binding.dropout_grad(res, 0.1, rng_of(11, step))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[0]) and torch.equal(dx, want[1])
    assert rng.tolist() == [11, 4]


@pytest.mark.parametrize("dt", TYPES, ids=str)
def test_more_numbers_than_a_launch_has_lanes_for(dt):
    """2^28 groups a launch: the last rows belong to the lanes' second round; their groups are past 2^28."""
    rows, width = (1 << 28) + 1000, 1
    x = torch.ones(rows, width, dtype=dt, device="cuda")
    y = binding.dropout(x, 0.5, rng_of(21, 22))
    for first in (0, (1 << 28) - 500, (1 << 28) + 500):
        mask = refs.kept(500, 1, 0.5, 21, 22, 0, first_row=first)
        assert torch.equal(y[first:first + 500].cpu(), torch.where(mask, 2.0, 0.0).to(dt))


def test_rows_past_32_bits():
    rows, width, dt = 200, 77, torch.bfloat16
    x, _ = make(rows, width, dt)
    ld = (1 << 31) // (rows - 1) + width + 2
    X = torch.empty(rows * ld, dtype=dt, device="cuda").view(rows, ld)[:, 1:1 + width]
    X.copy_(x.cuda())
    within(binding.dropout(X, 0.1, rng_of(1, 2), residual=X), refs.dropout(x, 0.1, refs.kept(rows, width, 0.1, 1, 2, 0), x), "y")
