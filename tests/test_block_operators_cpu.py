"""Refusals of the norm, the 8-bit operands, their product and dropout: every check runs on the host, before anything is enqueued, so bad calls can be
made without a GPU.  Pointers are made-up addresses that nothing follows.  And the plain forms themselves."""
import ctypes as C
import os

import numpy as np
import pytest
import torch

import block_refs as refs
from paper_2603_21090_amd import binding

INVALID, WORKSPACE = -1, -8
FAR = 1 << 40


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2603_21090_amd import build
        build.build_library()
    return binding.load_library()


def norm_args(**kw):
    base = dict(dtype=1, rows=100, width=64, eps=1e-6, ld_x=64, ld_residual=64, ld_h=64, ld_y=64, ld_q=64, ld_dy=64, ld_dh=64, x=1 << 20, residual=2 << 20,
                gain=3 << 20, h=4 << 20, y=5 << 20, q=6 << 20, scale=7 << 20, dy=8 << 20, dh=9 << 20, dx=10 << 20, dgain=11 << 20)
    base.update(kw)
    return binding.RmsNormArgs(**base)


def quantize_args(**kw):
    base = dict(dtype=1, columns=0, rows=100, width=64, ld_x=64, ld_q=100, x=1 << 20, q=2 << 20, scale=3 << 20)
    base.update(kw)
    return binding.QuantizeArgs(**base)


def product_args(**kw):
    base = dict(dtype=1, activation=0, rows=100, d_in=64, d_out=32, ld_x=64, ld_w=64, ld_residual=32, ld_y=32, x=1 << 20, w=2 << 20, x_scale=3 << 20,
                w_scale=4 << 20, bias=5 << 20, residual=6 << 20, y=7 << 20)
    base.update(kw)
    return binding.LinearI8Args(**base)


def dropout_args(**kw):
    base = dict(dtype=1, rows=100, width=64, site=0, p=0.5, ld_x=64, ld_residual=64, ld_y=64, x=1 << 20, residual=2 << 20, y=3 << 20, rng=4 << 20)
    base.update(kw)
    return binding.DropoutArgs(**base)


NORM = [dict(dtype=3), dict(reserved=1), dict(rows=(1 << 30) + 1), dict(width=0), dict(width=(1 << 24) + 1), dict(eps=-1e-9), dict(eps=float("nan")),
        dict(eps=float("inf")), dict(gain=None), dict(gain=(3 << 20) + 1), dict(ld_h=63), dict(ld_h=FAR + 1), dict(rows=1 << 24, ld_h=FAR)]


@pytest.mark.parametrize("bad", NORM + [dict(x=None), dict(y=None, q=None), dict(scale=None), dict(ld_x=63), dict(ld_residual=63), dict(ld_y=63), dict(ld_q=63),
                                        dict(x=(1 << 20) + 1), dict(residual=(2 << 20) + 1), dict(h=(4 << 20) + 1), dict(y=(5 << 20) + 1), dict(scale=(7 << 20) + 2),
                                        dict(h=5 << 20), dict(y=(1 << 20) + 2), dict(h=(2 << 20) + 128), dict(y=1 << 20, ld_y=65), dict(h=1 << 20, y=1 << 20),
                                        dict(q=1 << 20), dict(q=5 << 20), dict(q=3 << 20), dict(scale=6 << 20), dict(scale=4 << 20), dict(y=3 << 20), dict(h=3 << 20),
                                        dict(rows=1 << 24, ld_x=FAR), dict(rows=1 << 24, ld_y=FAR), dict(rows=1 << 24, ld_residual=FAR)], ids=str)
def test_rms_norm_refuses(lib, bad):
    assert lib.stgn_rms_norm(C.byref(norm_args(**bad)), None, 0, None) == INVALID
    assert lib.stgn_last_error(None)


@pytest.mark.parametrize("bad", NORM + [dict(h=None), dict(dy=None), dict(ld_dy=63), dict(ld_dh=63), dict(dy=(8 << 20) + 1), dict(dx=(10 << 20) + 1),
                                        dict(dgain=(11 << 20) + 1), dict(dx=4 << 20), dict(dx=8 << 20), dict(dx=9 << 20), dict(dx=3 << 20), dict(dgain=3 << 20),
                                        dict(dgain=(10 << 20) + 12), dict(dgain=4 << 20), dict(rows=1 << 24, ld_dy=FAR), dict(rows=1 << 24, ld_dh=FAR)], ids=str)
def test_rms_norm_grad_refuses(lib, bad):
    assert lib.stgn_rms_norm_grad(C.byref(norm_args(**bad)), None, 0, None) == INVALID
    assert lib.stgn_last_error(None)


@pytest.mark.parametrize("bad", [dict(dtype=3), dict(columns=2), dict(rows=(1 << 30) + 1), dict(width=0), dict(width=(1 << 24) + 1), dict(x=None), dict(q=None),
                                 dict(scale=None), dict(x=(1 << 20) + 1), dict(scale=(3 << 20) + 2), dict(ld_x=63), dict(ld_q=63), dict(columns=1, ld_q=99),
                                 dict(q=1 << 20), dict(scale=1 << 20), dict(scale=2 << 20), dict(columns=1, rows=1 << 24, width=1 << 20, ld_x=1 << 20, ld_q=1 << 24),
                                 dict(rows=1 << 24, ld_x=FAR), dict(rows=1 << 30, ld_q=1 << 20)], ids=str)
def test_quantize_refuses(lib, bad):
    assert lib.stgn_quantize(C.byref(quantize_args(**bad)), None, 0, None) == INVALID
    assert lib.stgn_last_error(None)


@pytest.mark.parametrize("bad", [dict(dtype=3), dict(activation=4), dict(reserved=1), dict(rows=(1 << 30) + 1), dict(d_in=0), dict(d_in=131072, ld_x=1 << 18, ld_w=1 << 18),
                                 dict(d_out=0), dict(d_out=(1 << 24) + 1), dict(rows=1 << 29, d_out=1 << 20), dict(x=None), dict(w=None), dict(x_scale=None), dict(w_scale=None),
                                 dict(y=None), dict(ld_x=63), dict(ld_w=63), dict(ld_y=31), dict(ld_residual=31), dict(y=(7 << 20) + 1), dict(bias=(5 << 20) + 1),
                                 dict(x_scale=(3 << 20) + 2), dict(w_scale=(4 << 20) + 1), dict(y=1 << 20), dict(y=2 << 20), dict(y=3 << 20), dict(y=4 << 20),
                                 dict(y=5 << 20), dict(y=(6 << 20) + 2), dict(y=6 << 20, ld_y=33), dict(rows=1 << 24, ld_x=FAR), dict(rows=1 << 24, ld_y=FAR)], ids=str)
def test_linear_i8_refuses(lib, bad):
    assert lib.stgn_linear_quantized(C.byref(product_args(**bad)), None, 0, None) == INVALID
    assert lib.stgn_last_error(None)


@pytest.mark.parametrize("bad", [dict(dtype=3), dict(rows=(1 << 30) + 1), dict(width=0), dict(width=(1 << 24) + 1), dict(site=65536), dict(p=-0.1), dict(p=1.1),
                                 dict(p=float("nan")), dict(x=None), dict(y=None), dict(rng=None), dict(rng=(4 << 20) + 4), dict(x=(1 << 20) + 1), dict(ld_x=63),
                                 dict(ld_residual=63), dict(ld_y=63), dict(y=(1 << 20) + 2), dict(y=1 << 20, ld_y=65), dict(y=4 << 20), dict(y=(2 << 20) + 128),
                                 dict(rows=1 << 24, ld_x=FAR), dict(rows=1 << 24, ld_y=FAR)], ids=str)
def test_dropout_refuses(lib, bad):
    assert lib.stgn_dropout(C.byref(dropout_args(**bad)), None) == INVALID
    assert lib.stgn_last_error(None)


@pytest.mark.parametrize("wide", [1, 20, 2048, 2049, 4096, 40001, 131071])
def test_no_rows(lib, wide):
    """Nothing is enqueued for a product, a norm or dropout of no rows, at any width."""
    n = C.c_size_t(7)
    args = product_args(rows=0, d_in=wide, ld_x=wide, ld_w=wide, d_out=wide, ld_y=wide, ld_residual=wide)
    assert lib.stgn_linear_quantized_workspace(C.byref(args), C.byref(n)) == 0 and n.value == 0
    assert lib.stgn_linear_quantized(C.byref(args), None, 0, None) == 0
    args = norm_args(rows=0, width=wide, **{f"ld_{m}": wide for m in ("x", "residual", "h", "y", "q", "dy", "dh")})
    assert lib.stgn_rms_norm_workspace(C.byref(args), C.byref(n), C.byref(n)) == 0
    assert lib.stgn_rms_norm(C.byref(args), None, 0, None) == 0
    args.dx = args.dgain = None
    assert lib.stgn_rms_norm_grad(C.byref(args), 1 << 30, n.value, None) == 0
    for columns in (0, 1):
        args = quantize_args(rows=0, columns=columns, width=wide, ld_x=wide, ld_q=wide)
        assert lib.stgn_quantize_workspace(C.byref(args), C.byref(n)) == 0 and n.value == 0
    args = quantize_args(rows=0, width=wide, ld_x=wide, ld_q=wide)
    assert lib.stgn_quantize(C.byref(args), None, 0, None) == 0
    assert lib.stgn_dropout(C.byref(dropout_args(rows=0, width=wide, ld_x=wide, ld_y=wide, ld_residual=wide)), None) == 0


def test_null_arguments_and_workspaces(lib):
    n, m = C.c_size_t(0), C.c_size_t(1)
    assert lib.stgn_dropout(None, None) == INVALID
    for op in ("rms_norm", "rms_norm_grad", "quantize", "linear_quantized"):
        assert getattr(lib, f"stgn_{op}")(None, None, 0, None) == INVALID
    assert lib.stgn_rms_norm_workspace(None, C.byref(n), C.byref(n)) == INVALID
    assert lib.stgn_quantize_workspace(None, C.byref(n)) == INVALID and lib.stgn_linear_quantized_workspace(None, C.byref(n)) == INVALID
    args = norm_args()
    assert lib.stgn_rms_norm_workspace(C.byref(args), None, None) == 0
    assert lib.stgn_rms_norm_workspace(C.byref(args), C.byref(m), C.byref(n)) == 0 and n.value > 0 and m.value == 0
    for call, args in ((lib.stgn_rms_norm_grad, args), (lib.stgn_quantize, quantize_args(columns=1, rows=2000, ld_q=2000))):
        if call is lib.stgn_quantize:
            assert lib.stgn_quantize_workspace(C.byref(args), C.byref(n)) == 0 and n.value > 0
        assert call(C.byref(args), None, n.value, None) == WORKSPACE
        assert call(C.byref(args), 1 << 30, n.value - 1, None) == WORKSPACE
        assert call(C.byref(args), (1 << 30) + 128, n.value, None) == WORKSPACE
    assert lib.stgn_rms_norm_workspace(C.byref(norm_args(dgain=None)), None, C.byref(n)) == 0 and n.value == 0


@pytest.mark.parametrize("call", [
    lambda x, g, q, s: binding.rms_norm(x, g[:5]), lambda x, g, q, s: binding.rms_norm(x, g.double()), lambda x, g, q, s: binding.rms_norm(x.int(), g.int()),
    lambda x, g, q, s: binding.rms_norm(x[0], g), lambda x, g, q, s: binding.rms_norm(x.t().contiguous().t(), g), lambda x, g, q, s: binding.rms_norm(x, g, residual=x[:3]),
    lambda x, g, q, s: binding.rms_norm(x[:, :0], g[:0]), lambda x, g, q, s: binding.rms_norm(x[:1].expand(4, 6), g), lambda x, g, q, s: binding.rms_norm(x, g),
    lambda x, g, q, s: binding.rms_norm_i8(x, g), lambda x, g, q, s: binding.rms_norm_grad(x[:3], x, g), lambda x, g, q, s: binding.rms_norm_grad(x, x, g, dh=x.double()),
    lambda x, g, q, s: binding.rms_norm_grad(x, x, g), lambda x, g, q, s: binding.quantize(x.int()), lambda x, g, q, s: binding.quantize(x[0]),
    lambda x, g, q, s: binding.quantize(x), lambda x, g, q, s: binding.quantize(x, columns=True), lambda x, g, q, s: binding.linear_i8(x, s, q, s),
    lambda x, g, q, s: binding.linear_i8(q, s, q[:, :5], s), lambda x, g, q, s: binding.linear_i8(q, s[:3], q, s), lambda x, g, q, s: binding.linear_i8(q, s, q, s[:3]),
    lambda x, g, q, s: binding.linear_i8(q, s.double(), q, s), lambda x, g, q, s: binding.linear_i8(q, s, q, s, bias=g), lambda x, g, q, s: binding.linear_i8(q, s, q, s),
    lambda x, g, q, s: binding.linear_i8(q, s, q, s, activation="tanh"), lambda x, g, q, s: binding.linear_i8(q, s, q, s, residual=x),
    lambda x, g, q, s: binding.linear_i8(q, s, q, s, bias=s, dtype=torch.bfloat16), lambda x, g, q, s: binding.linear_i8(q, s, q, s, dtype=torch.float64),
    lambda x, g, q, s: binding.linear_i8(q.t().contiguous().t(), s, q, s), lambda x, g, q, s: binding.dropout(x, 0.5, torch.ones(2)),
    lambda x, g, q, s: binding.dropout(x, 0.5, torch.ones(3, dtype=torch.int64)), lambda x, g, q, s: binding.dropout(x, 0.5, torch.ones(2, dtype=torch.int64), site=-1),
    lambda x, g, q, s: binding.dropout(x, 0.5, torch.ones(2, dtype=torch.int64)), lambda x, g, q, s: binding.dropout_grad(x, 0.5, torch.ones(2, dtype=torch.int64), site=65536),
])
def test_binding_refuses(lib, call):
    """Shapes, types, strides, and tensors that are not on a GPU."""
    with pytest.raises(ValueError):
        call(torch.ones(4, 6), torch.ones(6), torch.ones(4, 6, dtype=torch.int8), torch.ones(4))


def test_the_generators_published_answers():
    """Known answers of Philox 4x32-10 that its authors publish beside it."""
    for counter, key, want in (([0] * 4, [0] * 2, [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]),
                               ([0xFFFFFFFF] * 4, [0xFFFFFFFF] * 2, [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]),
                               ([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0], [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1])):
        assert [int(w) for w in refs.philox(counter, key)] == want


def test_the_plain_forms_agree_with_automatic_differentiation():
    g = torch.Generator().manual_seed(1)
    n = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64).float()  # noqa: E731
    h, gain, dy, dh = n(5, 7), n(7), n(5, 7), n(5, 7)
    leaves = [t.double().requires_grad_() for t in (h, gain)]
    y = leaves[0] / torch.sqrt(leaves[0].square().mean(1, keepdim=True) + 0.3) * leaves[1]
    assert (y - refs.rms_norm(h, None, gain, 0.3)[0][0]).abs().max() <= 1e-12
    want = torch.autograd.grad((y * dy.double()).sum() + (leaves[0] * dh.double()).sum(), leaves)
    for a, b in zip(want, refs.rms_norm_grad(dy, h, gain, dh, 0.3)):
        assert (a - b[0]).abs().max() <= 1e-12


def test_the_plain_form_in_8_bits():
    """Every number is the nearest one to its quotient, and the largest is 127."""
    g = torch.Generator().manual_seed(2)
    y = torch.randn(50, 33, generator=g)
    q, scale = refs.eight(y)
    assert (q.abs().amax(1) == 127).all()
    assert ((q.double() * y.double().abs().amax(1, keepdim=True) / 127 - y.double()).abs() <= 0.5000001 * scale.double()[:, None]).all()
    q, scale = refs.eight(torch.tensor([[0.0, 0.0], [float("inf"), 1.0], [float("nan"), 1.0]]))
    assert not q.any() and scale[0] == 0 and scale[1:].isnan().all()
    assert np.isnan(scale[1].item())
