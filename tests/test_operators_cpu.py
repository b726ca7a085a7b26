"""Refusals of the operators' entry points: every check runs on the host, before anything is enqueued, so bad calls can be made
without a GPU.  Pointers are made-up addresses that nothing follows."""
import ctypes as C
import os

import pytest
import torch

import operator_refs as refs
from paper_2603_21090_amd import binding

INVALID, WORKSPACE = -1, -8


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2603_21090_amd import build
        build.build_library()
    return binding.load_library()


def linear_args(**kw):
    base = dict(dtype=1, activation=0, rows=100, d_in=64, d_out=32, ld_x=64, ld_w=32, ld_residual=32, ld_y=32, ld_pre=32, ld_dy=32,
                x=1 << 20, w=2 << 20, bias=3 << 20, residual=4 << 20, y=5 << 20, pre=6 << 20, dy=7 << 20, dx=8 << 20, dw=9 << 20, db=10 << 20)
    base.update(kw)
    return binding.LinearArgs(**base)


def attention_args(**kw):
    base = dict(dtype=1, causal=0, window=0, lists=2, q_len=5, k_len=9, heads=4, kv_heads=2, d_head=16, scale=0.25,
                q_list=320, q_row=64, q_head=16, k_list=288, k_row=32, k_head=16, v_list=288, v_row=32, v_head=16,
                out_list=320, out_row=64, out_head=16, dout_list=320, dout_row=64, dout_head=16, q_lens=1 << 20, k_lens=2 << 20, q=3 << 20, k=4 << 20, v=5 << 20,
                out=6 << 20, lse=7 << 20, dout=8 << 20, dq=9 << 20, dk=10 << 20, dv=11 << 20)
    base.update(kw)
    return binding.AttentionArgs(**base)


EITHER = [dict(dtype=3), dict(activation=4), dict(d_in=0), dict(d_out=0), dict(d_in=(1 << 24) + 1, ld_x=1 << 25), dict(rows=(1 << 30) + 1),
          dict(x=None), dict(w=None), dict(ld_x=63), dict(ld_w=31), dict(x=(1 << 20) + 1), dict(ld_x=1 << 41)]


@pytest.mark.parametrize("bad", EITHER + [dict(y=None), dict(ld_y=31), dict(ld_residual=31), dict(ld_pre=31), dict(y=1 << 20), dict(y=2 << 20),
                                          dict(y=3 << 20), dict(y=6 << 20), dict(y=(4 << 20) + 2), dict(pre=1 << 20), dict(pre=4 << 20),
                                          dict(residual=5 << 20, ld_residual=33)], ids=str)
def test_linear_refuses(lib, bad):
    assert lib.stgn_linear(C.byref(linear_args(**bad)), None, 0, None) == INVALID
    assert lib.stgn_last_error(None)


@pytest.mark.parametrize("bad", EITHER + [dict(dy=None), dict(ld_dy=31), dict(activation=2, pre=None), dict(activation=2, ld_pre=31), dict(dx=7 << 20),
                                          dict(dw=1 << 20), dict(db=2 << 20), dict(dw=8 << 20), dict(db=9 << 20), dict(db=(10 << 20) + 1),
                                          dict(activation=1, dx=6 << 20)], ids=str)
def test_linear_grad_refuses(lib, bad):
    assert lib.stgn_linear_grad(C.byref(linear_args(**bad)), None, 0, None) == INVALID
    assert lib.stgn_last_error(None)


MASKS = [dict(dtype=3), dict(d_head=0), dict(d_head=257), dict(heads=0), dict(kv_heads=0), dict(heads=5), dict(causal=2), dict(window=3),
         dict(lists=(1 << 30) + 1), dict(q_len=(1 << 29) + 1), dict(k_len=(1 << 29) + 1), dict(q_len=0, k_len=0, lists=1 << 23), dict(scale=float("nan")), dict(scale=float("inf")),
         dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(lse=None), dict(q=(3 << 20) + 1), dict(lse=(7 << 20) + 2),
         dict(q_lens=(1 << 20) + 2), dict(k_row=1 << 41), dict(lists=1 << 26, q_len=64)]


@pytest.mark.parametrize("bad", MASKS + [dict(out=3 << 20), dict(out_head=15), dict(out_row=0), dict(out_list=319), dict(out=4 << 20), dict(lse=5 << 20), dict(lse=6 << 20)], ids=str)
def test_attention_refuses(lib, bad):
    assert lib.stgn_attention(C.byref(attention_args(**bad)), None, 0, None) == INVALID
    assert lib.stgn_last_error(None)


@pytest.mark.parametrize("bad", MASKS + [dict(dout=None), dict(dq=None), dict(dk=None), dict(dv=None), dict(dq=3 << 20), dict(dk=8 << 20), dict(dv=7 << 20),
                                         dict(dk=11 << 20), dict(dq=11 << 20), dict(dout_head=1 << 41)], ids=str)
def test_attention_grad_refuses(lib, bad):
    assert lib.stgn_attention_grad(C.byref(attention_args(**bad)), None, 0, None) == INVALID
    assert lib.stgn_last_error(None)


@pytest.mark.parametrize("bad", [dict(x=1 << 20, y=(1 << 20) + 126), dict(x=1 << 20, y=(1 << 20) + 2 * 65), dict(y=1 << 20, x=(1 << 20) + 62),
                                 dict(x=1 << 20, y=(1 << 20) + 2 * 96 * 7 + 126), dict(x=1 << 20, y=(1 << 20) + 128, ld_y=97),
                                 dict(pre=1 << 20, residual=(1 << 20) + 2, ld_pre=96, ld_residual=96)], ids=str)
def test_columns_of_one_matrix_that_overlap_are_refused(lib, bad):
    assert lib.stgn_linear(C.byref(linear_args(**{**dict(ld_x=96, ld_y=96), **bad})), None, 0, None) == INVALID
    assert b"overlaps" in lib.stgn_last_error(None)


def test_lengths_are_inputs_that_outputs_may_not_overlap(lib):
    for bad in (dict(out=1 << 20), dict(lse=2 << 20), dict(lse=(2 << 20) + 4)):
        assert lib.stgn_attention(C.byref(attention_args(**bad)), None, 0, None) == INVALID
    for bad in (dict(dq=1 << 20), dict(dk=2 << 20), dict(dv=(1 << 20) + 4)):
        assert lib.stgn_attention_grad(C.byref(attention_args(**bad)), None, 0, None) == INVALID


def test_a_failed_create_is_told_to_threads_without_failures(lib):
    import threading
    seen, n = [], C.c_size_t(0)

    def other():
        seen.append((lib.stgn_query_workspace(None, C.byref(n)), lib.stgn_last_error(None)))
    for read in (other, lambda: seen.append(lib.stgn_last_error(None))):
        t = threading.Thread(target=read)
        t.start()
        t.join()
    assert seen[0][0] == INVALID and seen[0][1] and seen[1] == seen[0][1]


def test_null_arguments_and_workspaces(lib):
    n = C.c_size_t(0)
    for op, args in (("linear", linear_args(activation=2)), ("attention", attention_args())):
        assert getattr(lib, f"stgn_{op}")(None, None, 0, None) == INVALID
        assert getattr(lib, f"stgn_{op}_grad")(None, None, 0, None) == INVALID
        assert getattr(lib, f"stgn_{op}_workspace")(None, C.byref(n), C.byref(n)) == INVALID
        assert getattr(lib, f"stgn_{op}_workspace")(C.byref(args), None, None) == 0
        assert getattr(lib, f"stgn_{op}_workspace")(C.byref(args), None, C.byref(n)) == 0 and n.value > 0
        grad = getattr(lib, f"stgn_{op}_grad")
        assert grad(C.byref(args), None, n.value, None) == WORKSPACE
        assert grad(C.byref(args), 1 << 30, n.value - 1, None) == WORKSPACE
        assert grad(C.byref(args), (1 << 30) + 128, n.value, None) == WORKSPACE


def test_messages_belong_to_the_thread(lib):
    import threading
    assert lib.stgn_linear(C.byref(linear_args(x=None)), None, 0, None) == INVALID
    mine, seen = lib.stgn_last_error(None), []

    def other():
        lib.stgn_attention(C.byref(attention_args(window=3)), None, 0, None)
        seen.append(lib.stgn_last_error(None))
    t = threading.Thread(target=other)
    t.start()
    t.join()
    assert lib.stgn_last_error(None) == mine and seen[0] != mine


@pytest.mark.parametrize("call", [
    lambda x, w: binding.linear(x, w[:5]), lambda x, w: binding.linear(x, w.double()), lambda x, w: binding.linear(x.int(), w.int()),
    lambda x, w: binding.linear(x, w.t().contiguous().t()), lambda x, w: binding.linear(x, w, bias=torch.ones(3)),
    lambda x, w: binding.linear(x, w, residual=torch.ones(4, 7)), lambda x, w: binding.linear(x[0], w), lambda x, w: binding.linear(x, w),
    lambda x, w: binding.linear(x[:1].expand(4, 6), w), lambda x, w: binding.linear_grad(torch.ones(4, 8), x, w, activation="gelu"),
    lambda x, w: binding.linear_grad(torch.ones(3, 8), x, w),
    lambda x, w: binding.attention(x, x, x), lambda x, w: binding.attention(x[None, None], x[None, None], w[None, None]),
    lambda x, w: binding.attention(*(x[None, None],) * 3, causal=True, window=-1), lambda x, w: binding.attention(*(x[None, None, :, :0],) * 3),
    lambda x, w: binding.linear(x, w, activation="tanh"), lambda x, w: binding.attention(*(x[None, None],) * 3, k_lens=torch.ones(1)), lambda x, w: binding.attention(*(x[None, None],) * 3),
    lambda x, w: binding.attention_grad(*(x[None, None],) * 5, torch.ones(1, 4, 2)),
])
def test_binding_refuses(lib, call):
    """Shapes, types, strides, and tensors that are not on a GPU."""
    with pytest.raises(ValueError):
        call(torch.ones(4, 6), torch.ones(6, 8))


def test_the_plain_forms_agree_with_automatic_differentiation():
    g = torch.Generator().manual_seed(1)
    n = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64).float()  # noqa: E731
    x, w, b, dy = n(5, 7), n(7, 4), n(4), n(5, 4)
    for name, f in (("none", lambda t: t), ("relu", torch.relu), ("gelu", torch.nn.functional.gelu), ("silu", torch.nn.functional.silu)):
        leaves = [t.double().requires_grad_() for t in (x, w, b)]
        z = leaves[0] @ leaves[1] + leaves[2]
        y = f(z)
        want = torch.autograd.grad(y, leaves, dy.double())
        refs.within(y, (refs.linear(x, w, b, name, None)[0][0], torch.full_like(y, 1e-12)))
        for a, got in zip(want, refs.linear_grad(dy, x, w, name, z.detach())):
            refs.within(a, (got[0], torch.full_like(got[0], 1e-12)))
    q, k, v, do = n(2, 6, 4, 5), n(2, 9, 2, 5), n(2, 9, 2, 5), n(2, 6, 4, 5)
    kn, qn = torch.tensor([9, 4]), torch.tensor([6, 3])
    see = refs.visible(2, 6, 9, qn, kn, True, 3)
    leaves = [t.double().requires_grad_() for t in (q, k, v)]
    Q, K, V = (t.transpose(1, 2) for t in leaves)
    K, V = K.repeat_interleave(2, 1), V.repeat_interleave(2, 1)
    s = (0.4 * Q @ K.transpose(2, 3)).masked_fill(~see[:, None], -1e300)
    out = (torch.softmax(s, -1) * see.any(2)[:, None, :, None]) @ V
    want = torch.autograd.grad(out.transpose(1, 2), leaves, do.double())
    got = refs.attention(q, k, v, see, 0.4, do)
    for a, name in zip((out.transpose(1, 2),) + want, ("out", "dq", "dk", "dv")):
        refs.within(a, (got[name][0], torch.full_like(got[name][0], 1e-12)), name)


HAMMER = r"""
import ctypes as C, sys, threading, time
lib = C.CDLL(sys.argv[1])
lib.stgn_last_error.restype, lib.stgn_last_error.argtypes = C.c_char_p, [C.c_void_p]
class Cfg(C.Structure):
    _fields_ = [("bytes", C.c_uint8 * 256)]
n, cfg = C.c_size_t(0), Cfg()
fail = (lambda: lib.stgn_query_workspace(None, C.byref(n)), lambda: lib.stgn_query_workspace(C.byref(cfg), C.byref(n)),
        lambda: lib.stgn_create(None, None, None, None, C.c_size_t(0), None, None))
told = set()
for f in fail:
    assert f() != 0
    told.add(lib.stgn_last_error(None))
assert len(told) >= 2 and all(told)
end, odd = time.monotonic() + 1.5, []
def write(f):
    while time.monotonic() < end:
        f()
def read():
    while time.monotonic() < end:
        m = lib.stgn_last_error(None)
        if m not in told:
            odd.append(m)
threads = [threading.Thread(target=write, args=(fail[i % 3],)) for i in range(4)] + [threading.Thread(target=read) for _ in range(4)]
[t.start() for t in threads]
[t.join() for t in threads]
assert not odd, odd[:3]
"""


def test_messages_of_failures_in_other_threads_are_whole(lib):
    """Threads that fail to create, in turn with different messages, while threads without failures read them (in a process of its own)."""
    import subprocess
    import sys
    r = subprocess.run([sys.executable, "-c", HAMMER, binding.LIB_PATH], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0, r.stderr[-2000:]


FAR = 1 << 40


@pytest.mark.parametrize("bad", [dict(ld_x=FAR), dict(ld_w=FAR, rows=100, d_in=1 << 20, ld_x=1 << 20), dict(ld_y=FAR), dict(ld_residual=FAR), dict(ld_pre=FAR),
                                 dict(ld_x=FAR, y=1 << 20), dict(ld_y=FAR, ld_x=1 << 20)], ids=str)
def test_matrices_that_reach_past_every_address_are_refused(lib, bad):
    """2^24 rows 2^40 numbers apart: their length in bytes is no 64-bit number, and an output that lies on an input would not be seen."""
    args = linear_args(**{**dict(rows=1 << 24), **bad})
    assert lib.stgn_linear(C.byref(args), None, 0, None) == INVALID
    assert b"2^48" in lib.stgn_last_error(None)


@pytest.mark.parametrize("bad", [dict(ld_x=FAR), dict(ld_dy=FAR), dict(ld_pre=FAR, activation=1)], ids=str)
def test_gradients_of_matrices_that_reach_past_every_address_are_refused(lib, bad):
    assert lib.stgn_linear_grad(C.byref(linear_args(**{**dict(rows=1 << 24), **bad})), None, 0, None) == INVALID
    assert b"2^48" in lib.stgn_last_error(None)


@pytest.mark.parametrize("bad", ["q_list", "q_row", "k_list", "k_row", "k_head", "v_list", "v_row", "out_list", "out_head", "dout_list", "dout_row", "dout_head"])
def test_tensors_that_reach_past_every_address_are_refused(lib, bad):
    args = attention_args(**{bad: FAR, "lists": 1 << 12, "q_len": 1 << 10, "k_len": 1 << 10} if not bad.endswith("head") else
                          {bad: FAR, "heads": 1 << 10, "kv_heads": 1 << 10})
    for call in (lib.stgn_attention, lib.stgn_attention_grad) if not bad.startswith("dout") else (lib.stgn_attention_grad,):
        assert call(C.byref(args), None, 0, None) == INVALID
        assert b"2^48" in lib.stgn_last_error(None)


def test_reserved_numbers_are_zero(lib):
    n = C.c_size_t(0)
    args = linear_args(reserved=1)
    for rc in (lib.stgn_linear(C.byref(args), None, 0, None), lib.stgn_linear_grad(C.byref(args), None, 0, None),
               lib.stgn_linear_workspace(C.byref(args), C.byref(n), None)):
        assert rc == INVALID and b"reserved" in lib.stgn_last_error(None)
