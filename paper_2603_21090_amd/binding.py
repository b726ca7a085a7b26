"""Thin ctypes binding of libstreamtgn (argument marshalling only).

PyTorch is used for two things: the device workspace (one uint8 tensor) and the HIP stream the
library enqueues its kernels on.  Every step of the method runs inside the library's kernels;
there is no Python or CPU fallback -- if the shared library is missing this module raises.
"""
from __future__ import annotations

import ctypes as C
import os
import struct

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libstreamtgn.so")

STGN_MAX_LAYERS = 4
ERRORS = {0: "OK", -1: "INVALID_ARG", -2: "NODE_OUT_OF_RANGE", -3: "TIME_ORDER", -4: "SELF_LOOP",
          -5: "BATCH_TOO_LARGE", -6: "EDGE_CAPACITY", -7: "DEVICE", -8: "WORKSPACE"}

_f32p = C.POINTER(C.c_float)
_u32p = C.POINTER(C.c_uint32)
_f64p = C.POINTER(C.c_double)


class Config(C.Structure):
    _fields_ = [("num_nodes", C.c_uint32), ("max_edges", C.c_uint64), ("max_batch", C.c_uint32),
                ("d_mem", C.c_uint32), ("d_node", C.c_uint32), ("d_edge", C.c_uint32), ("d_time", C.c_uint32),
                ("d_emb", C.c_uint32), ("d_msg", C.c_uint32), ("k", C.c_uint32), ("heads", C.c_uint32),
                ("layers", C.c_uint32), ("window", C.c_double), ("aggregator", C.c_uint32), ("delta_mode", C.c_uint32),
                ("drift_gamma", C.c_double)]


class Weights(C.Structure):
    _fields_ = [(n, _f32p) for n in
                ("omega", "phase", "W_msg", "b_msg", "W_z", "U_z", "b_z", "W_r", "U_r", "b_r", "W_h", "U_h", "b_h")] + \
               [(n, C.POINTER(_f32p)) for n in ("W_Q", "W_K", "W_V", "W_O", "b_O")]


class BatchStats(C.Structure):
    _fields_ = [("n_edges", C.c_uint32), ("n_direct", C.c_uint32), ("n_affected", C.c_uint32),
                ("frontier", C.c_uint32 * (STGN_MAX_LAYERS + 1)), ("entries_scanned", C.c_uint64),
                ("pull_hops", C.c_uint32), ("reserved", C.c_uint32), ("us_stage", C.c_float * 6)]

    def as_dict(self):
        return dict(n_edges=self.n_edges, n_direct=self.n_direct, n_affected=self.n_affected,
                    frontier=list(self.frontier), entries_scanned=self.entries_scanned, pull_hops=self.pull_hops,
                    us_stage=dict(zip(("sort", "memory", "apply", "propagate", "embed", "total"), self.us_stage)))


class LinearArgs(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in ("dtype", "activation", "rows", "d_in", "d_out", "reserved")] + \
               [(n, C.c_uint64) for n in ("ld_x", "ld_w", "ld_residual", "ld_y", "ld_pre", "ld_dy")] + \
               [(n, C.c_void_p) for n in ("x", "w", "bias", "residual", "y", "pre", "dy", "dx", "dw", "db")]


class AttentionArgs(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in ("dtype", "causal", "window", "lists", "q_len", "k_len", "heads", "kv_heads", "d_head")] + \
               [("scale", C.c_float)] + \
               [(f"{t}_{n}", C.c_uint64) for t in ("q", "k", "v", "out", "dout") for n in ("list", "row", "head")] + \
               [(n, C.c_void_p) for n in ("q_lens", "k_lens", "q", "k", "v", "out", "lse", "dout", "dq", "dk", "dv")]


# the same two, packed at once: a call's arguments cost the host a microsecond, not one per field
_PACK_LINEAR, _PACK_ATTENTION = struct.Struct("@6I6Q10P"), struct.Struct("@9If15Q11P")
assert _PACK_LINEAR.size == C.sizeof(LinearArgs) and _PACK_ATTENTION.size == C.sizeof(AttentionArgs)


class StgnError(RuntimeError):
    def __init__(self, code, msg=""):
        super().__init__(f"libstreamtgn: {ERRORS.get(code, code)} ({code}) {msg}")
        self.code = code


_lib = None

EXPORTS = ("stgn_query_workspace", "stgn_create", "stgn_destroy", "stgn_ingest_batch", "stgn_get_embeddings",
           "stgn_full_rebuild", "stgn_sync", "stgn_get_affected", "stgn_get_neighbors", "stgn_get_history",
           "stgn_get_memory", "stgn_get_totals", "stgn_kernel_times", "stgn_last_error", "stgn_version",
           "stgn_set_predictor", "stgn_predict_batch", "stgn_predict_batch_static", "stgn_drift_status",
           "stgn_maintain", "stgn_probe_gather", "stgn_linear_workspace", "stgn_linear", "stgn_linear_grad",
           "stgn_attention_workspace", "stgn_attention", "stgn_attention_grad", "stgn_predictor_mlp_workspace",
           "stgn_set_predictor_mlp")


def load_library():
    """Loads libstreamtgn.so from the package directory; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2603_21090_amd.build` "
                          "(there is no fallback path)")
    L = C.CDLL(LIB_PATH)
    vp = C.c_void_p
    L.stgn_query_workspace.argtypes = [C.POINTER(Config), C.POINTER(C.c_size_t)]
    L.stgn_create.argtypes = [C.POINTER(Config), C.POINTER(Weights), vp, vp, C.c_size_t, vp, C.POINTER(vp)]
    L.stgn_destroy.argtypes = [vp]
    L.stgn_destroy.restype = None
    L.stgn_ingest_batch.argtypes = [vp, C.c_uint32, vp, vp, vp, vp, C.c_int, C.POINTER(BatchStats)]
    L.stgn_get_embeddings.argtypes = [vp, C.c_uint32, C.c_uint32, vp, vp, C.c_int]
    L.stgn_full_rebuild.argtypes = [vp]
    L.stgn_sync.argtypes = [vp]
    L.stgn_get_affected.argtypes = [vp, vp, C.c_uint32, _u32p]
    L.stgn_get_neighbors.argtypes = [vp, C.c_uint32, vp, vp, vp, _u32p]
    L.stgn_get_history.argtypes = [vp, C.c_uint32, C.c_uint32, C.c_uint32, vp, vp, _u32p]
    L.stgn_get_memory.argtypes = [vp, C.c_uint32, vp, vp, vp]
    L.stgn_get_totals.argtypes = [vp] + [C.POINTER(C.c_uint64)] * 6
    L.stgn_kernel_times.argtypes = [vp, C.c_int, C.c_int, C.c_uint32, C.POINTER(C.c_char_p), _f64p,
                                    C.POINTER(C.c_uint64)]
    L.stgn_set_predictor.argtypes = [vp, vp, C.c_float]
    L.stgn_predictor_mlp_workspace.argtypes = [vp, C.c_uint32, C.POINTER(C.c_size_t)]
    L.stgn_set_predictor_mlp.argtypes = [vp, C.c_uint32, C.c_uint32, vp, vp, vp, C.c_float, vp, C.c_size_t]
    L.stgn_predict_batch.argtypes = [vp, C.c_uint32, vp, vp, vp, C.c_int, C.c_int, vp]
    L.stgn_predict_batch_static.argtypes = [vp, C.c_uint32, vp, vp, vp, C.c_int, vp]
    L.stgn_drift_status.argtypes = [vp, C.POINTER(C.c_double), _u32p, vp]
    L.stgn_maintain.argtypes = [vp, C.c_double, C.c_double, C.POINTER(C.c_int), _u32p]
    L.stgn_probe_gather.argtypes = [vp, C.c_uint64, C.c_uint32, vp, C.c_uint32, C.c_uint32, vp, vp]
    for op in ("linear", "attention"):
        getattr(L, f"stgn_{op}_workspace").argtypes = [vp, vp, vp]
        for name in (f"stgn_{op}", f"stgn_{op}_grad"):
            getattr(L, name).argtypes = [vp, vp, C.c_size_t, vp]
    L.stgn_last_error.argtypes = [vp]
    L.stgn_last_error.restype = C.c_char_p
    L.stgn_version.restype = C.c_char_p
    _lib = L
    return L


def _host_f32(a):
    return None if a is None else np.ascontiguousarray(a, dtype=np.float32)


def _ptr(a):
    return None if a is None else C.c_void_p(a.ctypes.data)


def make_config(*, num_nodes, max_edges, max_batch, d_mem, d_node, d_edge, d_time, d_emb, d_msg, k, heads, layers,
                window=0.0, aggregator=0, delta_mode=0, drift_gamma=0.0):
    return Config(num_nodes, max_edges, max_batch, d_mem, d_node, d_edge, d_time, d_emb, d_msg, k, heads, layers,
                  float(window), int(aggregator), int(delta_mode), float(drift_gamma))


def query_workspace(cfg: Config) -> int:
    n = C.c_size_t(0)
    rc = load_library().stgn_query_workspace(C.byref(cfg), C.byref(n))
    if rc:
        raise StgnError(rc, load_library().stgn_last_error(None).decode())
    return n.value


def probe_gather(table, idx, per_group, out, stream=0):
    """One launch of the bare gather (stgn_probe_gather) on torch device tensors: table [rows, 64 or 256] fp32,
    idx [groups * per_group] int32, out [groups * 16] fp32.  Asynchronous."""
    row_bytes = table.shape[1] * 4
    groups = idx.numel() // per_group
    rc = load_library().stgn_probe_gather(table.data_ptr(), table.shape[0], row_bytes, idx.data_ptr(), groups, per_group,
                                          out.data_ptr(), stream)
    if rc:
        raise StgnError(rc)


# ---- operators on the caller's tensors: torch device tensors in, new tensors out, on the current stream of their device.  They
# record nothing for automatic differentiation, whatever their inputs require: the gradients are calls of their own.
ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
_dtypes = None


def _dtype_code(t):
    global _dtypes
    if _dtypes is None:
        import torch
        _dtypes = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
    code = _dtypes.get(t.dtype)
    if code is None:
        raise ValueError(f"elements must be float32, bfloat16 or float16, not {t.dtype}")
    return code


def _expect(name, t, like, shape):
    """The address of a tensor of this shape, of `like`'s type and device, whose last dimension lies side by side."""
    if t.dtype != like.dtype or t.device != like.device:
        raise ValueError(f"{name}: {t.dtype} on {t.device}, expected {like.dtype} on {like.device}")
    if t.shape != shape:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    if shape[-1] > 1 and t.stride(-1) != 1 and t.numel():
        raise ValueError(f"{name}: the numbers of a row must lie side by side (last stride {t.stride(-1)})")
    return t.data_ptr()


def _ld(t):
    """Elements between the rows of a matrix; any value that covers a row where there is one row at most."""
    ld, width = t.stride(0), t.shape[1]
    if ld < width:
        if t.shape[0] > 1:
            raise ValueError(f"rows of {width} numbers lie {ld} apart")
        return width
    return ld


def _run_operator(ask, call, args, grad, device):
    """Workspace of the call (the caching allocator's, on the current stream), then the call."""
    import torch
    if device.type != "cuda":
        raise ValueError(f"tensors must be on the GPU, not on {device}")
    if torch.cuda.current_device() != device.index:
        with torch.cuda.device(device):
            return _run_operator(ask, call, args, grad, device)
    n = C.c_size_t(0)
    rc = ask(args, None, C.byref(n)) if grad else ask(args, C.byref(n), None)
    if rc == 0:
        size, ws = n.value, None
        if size:
            ws = torch.empty(size, dtype=torch.uint8, device=device)
        # (the handle alone: building a Stream object around it takes as long as the launch)
        rc = call(args, ws.data_ptr() if size else None, size, torch._C._cuda_getCurrentRawStream(device.index))
    if rc:
        raise StgnError(rc, load_library().stgn_last_error(None).decode())


def _linear_sizes(x, w, activation):
    if x.dim() != 2 or w.dim() != 2:
        raise ValueError("x and w must be matrices")
    if activation not in ACTIVATIONS:
        raise ValueError(f"activation must be one of {', '.join(ACTIVATIONS)}")
    (rows, d_in), d_out = x.shape, w.shape[1]
    return (_dtype_code(x), ACTIVATIONS[activation], rows, d_in, d_out, 0), (rows, d_out)


def linear(x, w, bias=None, activation="none", residual=None, keep_pre=False):
    """y = act(x w + bias) + residual (stgn_linear): x [rows, d_in], w [d_in, d_out], bias [d_out], residual [rows, d_out], all
    of one type (float32, bfloat16, float16); activation: "none", "relu", "gelu", "silu".  Returns y, or (y, pre) with
    keep_pre: the values in front of the activation, which linear_grad needs.  y has no autograd graph, also where an input
    requires gradients: linear_grad computes them."""
    import torch
    L = load_library()
    sizes, shape = _linear_sizes(x, w, activation)
    d_out = shape[1]
    xp, wp = _expect("x", x, x, x.shape), _expect("w", w, x, (x.shape[1], d_out))
    bp = _expect("bias", bias, x, (d_out,)) if bias is not None else 0
    rp = _expect("residual", residual, x, shape) if residual is not None else 0
    y = torch.empty(shape, dtype=x.dtype, device=x.device)
    pre = torch.empty_like(y) if keep_pre else None
    args = _PACK_LINEAR.pack(*sizes, _ld(x), _ld(w), _ld(residual) if rp else 0, d_out, d_out, 0,
                             xp, wp, bp, rp, y.data_ptr(), pre.data_ptr() if keep_pre else 0, 0, 0, 0, 0)
    _run_operator(L.stgn_linear_workspace, L.stgn_linear, args, False, x.device)
    return (y, pre) if keep_pre else y


def linear_grad(dy, x, w, activation="none", pre=None, bias=True, need_x=True, need_w=True):
    """Gradients of linear (stgn_linear_grad): (dx, dw, db), None for those not asked for.  pre: what linear kept, needed with an
    activation.  The residual's gradient is dy itself."""
    import torch
    L = load_library()
    sizes, shape = _linear_sizes(x, w, activation)
    xp, wp, gp = _expect("x", x, x, x.shape), _expect("w", w, x, (x.shape[1], shape[1])), _expect("dy", dy, x, shape)
    pp = 0
    if activation != "none":
        if pre is None:
            raise ValueError("the gradient of an activation needs pre")
        pp = _expect("pre", pre, x, shape)
    dx = torch.empty(x.shape, dtype=x.dtype, device=x.device) if need_x else None
    dw = torch.empty(w.shape, dtype=x.dtype, device=x.device) if need_w else None
    db = torch.empty(shape[1:], dtype=x.dtype, device=x.device) if bias else None
    args = _PACK_LINEAR.pack(*sizes, _ld(x), _ld(w), 0, 0, _ld(pre) if activation != "none" else 0, _ld(dy), xp, wp, 0, 0, 0, pp, gp,
                             dx.data_ptr() if need_x else 0, dw.data_ptr() if need_w else 0, db.data_ptr() if bias else 0)
    _run_operator(L.stgn_linear_workspace, L.stgn_linear_grad, args, True, x.device)
    return dx, dw, db


def _attention_call(q, k, v, q_lens, k_lens, causal, window, scale):
    """Sizes and strides of the packed arguments, and the addresses of the lengths, q, k and v."""
    if q.dim() != 4 or k.dim() != 4:
        raise ValueError("q, k and v must be [lists, rows, heads, numbers]")
    (lists, q_len, heads, d), (_, k_len, kv_heads, _) = q.shape, k.shape
    if d < 1 or window < 0:
        raise ValueError("a head has one number at least, a window is 0 or more")
    shape = (lists, k_len, kv_heads, d)
    where = [0, 0, _expect("q", q, q, q.shape), _expect("k", k, q, shape), _expect("v", v, q, shape)]
    for at, t in enumerate((q_lens, k_lens)):
        if t is not None:
            import torch
            if t.dtype != torch.int32 or t.device != q.device or t.shape != (lists,) or not t.is_contiguous():
                raise ValueError(f"q_lens and k_lens: a dense int32 tensor [lists] on {q.device} is expected")
            where[at] = t.data_ptr()
    sizes = (_dtype_code(q), 1 if causal else 0, window, lists, q_len, k_len, heads, kv_heads, d, d ** -0.5 if scale is None else scale)
    return sizes + q.stride()[:3] + k.stride()[:3] + v.stride()[:3], where


def attention(q, k, v, q_lens=None, k_lens=None, causal=False, window=0, scale=None):
    """Softmax attention (stgn_attention): q [lists, q_len, heads, d], k and v [lists, k_len, kv_heads, d], any strides but for the
    last; q_lens, k_lens: int32 [lists] on the device, None: all rows.  causal aligns the lists at their ends; window: only the last
    `window` keys up to the query (0: all).  scale: d ** -0.5 by default.  Returns out (as q) and lse [lists, heads, q_len] fp32,
    without an autograd graph, also where an input requires gradients: attention_grad computes them."""
    import torch
    L = load_library()
    sizes, where = _attention_call(q, k, v, q_lens, k_lens, causal, window, scale)
    lists, q_len, heads, d = q.shape
    out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    lse = torch.empty((lists, heads, q_len), dtype=torch.float32, device=q.device)
    args = _PACK_ATTENTION.pack(*sizes, q_len * heads * d, heads * d, d, 0, 0, 0, *where, out.data_ptr(), lse.data_ptr(), 0, 0, 0, 0)
    _run_operator(L.stgn_attention_workspace, L.stgn_attention, args, False, q.device)
    return out, lse


def attention_grad(dout, q, k, v, out, lse, q_lens=None, k_lens=None, causal=False, window=0, scale=None):
    """Gradients of attention (stgn_attention_grad) from its inputs and outputs and dout (out, dout: any strides but for the last):
    (dq, dk, dv), dense.  Heads that share a key head add up in dk and dv."""
    import torch
    L = load_library()
    sizes, where = _attention_call(q, k, v, q_lens, k_lens, causal, window, scale)
    gp, op = _expect("dout", dout, q, q.shape), _expect("out", out, q, q.shape)
    lists, q_len, heads, _ = q.shape
    if lse.dtype != torch.float32 or lse.device != q.device or lse.shape != (lists, heads, q_len) or not lse.is_contiguous():
        raise ValueError("lse must be what attention returned")
    dq = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    dk = torch.empty(k.shape, dtype=q.dtype, device=q.device)
    dv = torch.empty(k.shape, dtype=q.dtype, device=q.device)
    args = _PACK_ATTENTION.pack(*sizes, *out.stride()[:3], *dout.stride()[:3], *where, op, lse.data_ptr(), gp,
                                dq.data_ptr(), dk.data_ptr(), dv.data_ptr())
    _run_operator(L.stgn_attention_workspace, L.stgn_attention_grad, args, True, q.device)
    return dq, dk, dv


def _marshal_weights(weights: dict, layers: int, has_memory: bool):
    keep = []
    w = Weights()
    names = ["omega", "phase"] + (["W_msg", "b_msg", "W_z", "U_z", "b_z", "W_r", "U_r", "b_r", "W_h", "U_h", "b_h"]
                                   if has_memory else [])
    for name in names:
        a = _host_f32(weights[name])
        keep.append(a)
        setattr(w, name, a.ctypes.data_as(_f32p))
    for name in ("W_Q", "W_K", "W_V", "W_O", "b_O"):
        arrs = [_host_f32(a) for a in weights[name]]
        if len(arrs) != layers:
            raise ValueError(f"{name}: expected {layers} layers")
        ptrs = (_f32p * layers)(*[a.ctypes.data_as(_f32p) for a in arrs])
        keep += [arrs, ptrs]
        setattr(w, name, ptrs)
    return w, keep


class StreamTGN:
    """One device-resident serving state.  Methods mirror the C entry points one to one."""

    def __init__(self, cfg: Config, weights: dict, node_feat=None, device="cuda:0", stream=None):
        import torch
        self._L = load_library()
        self.cfg = cfg
        self._torch = torch
        self.device = torch.device(device)
        torch.cuda.set_device(self.device)
        nbytes = query_workspace(cfg)
        self.workspace_bytes = nbytes
        self._ws = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
        self._head_ws = {}
        base = (self._ws.data_ptr() + 255) & ~255
        self._stream = stream if stream is not None else torch.cuda.current_stream(self.device)
        w, keep = _marshal_weights(weights, cfg.layers, cfg.d_mem > 0)
        nf = _host_f32(node_feat)
        if nf is not None and nf.shape != (cfg.num_nodes, cfg.d_node):
            raise ValueError("node_feat shape")
        h = C.c_void_p(None)
        rc = self._L.stgn_create(C.byref(cfg), C.byref(w), _ptr(nf), C.c_void_p(base), nbytes,
                                 C.c_void_p(self._stream.cuda_stream), C.byref(h))
        if rc:
            raise StgnError(rc, self._L.stgn_last_error(None).decode())
        self._h = h

    @classmethod
    def from_workload(cls, w, weights, node_feat=None, max_edges=None, max_batch=None, delta_mode=0, drift_gamma=0.0, **kw):
        cfg = make_config(num_nodes=w.num_nodes, max_edges=max_edges or w.num_edges, max_batch=max_batch or w.batch,
                          d_mem=w.d_mem, d_node=w.d_node, d_edge=w.d_edge, d_time=w.d_time, d_emb=w.d_emb,
                          d_msg=w.d_msg, k=w.k, heads=w.heads, layers=w.layers, window=getattr(w, "window", 0.0),
                          aggregator=getattr(w, "aggregator", 0), delta_mode=delta_mode, drift_gamma=drift_gamma)
        return cls(cfg, weights, node_feat, **kw)

    def close(self):
        if getattr(self, "_h", None):
            self._L.stgn_destroy(self._h)
            self._h = None
            self._ws = self._head_ws = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, rc):
        if rc:
            raise StgnError(rc, self._L.stgn_last_error(self._h).decode())

    def last_error(self) -> str:
        return self._L.stgn_last_error(self._h).decode()

    # ---- hot path
    def ingest_batch(self, src, dst, ts, efeat, stats=False, check=True):
        """Host (NumPy) or device (torch, on this device) arrays; returns the code, or stats dict."""
        torch = self._torch
        on_dev = isinstance(src, torch.Tensor)
        n = int(src.shape[0])
        if on_dev:
            assert src.dtype == torch.int32 or src.dtype == torch.uint32
            assert ts.dtype == torch.float64 and (efeat is None or efeat.dtype == torch.float32)
            assert src.is_contiguous() and dst.is_contiguous() and ts.is_contiguous()
            assert efeat is None or efeat.is_contiguous()
            ptrs = [C.c_void_p(t.data_ptr()) if t is not None and t.numel() else None for t in (src, dst, ts, efeat)]
        else:
            src = np.ascontiguousarray(src, dtype=np.uint32)
            dst = np.ascontiguousarray(dst, dtype=np.uint32)
            ts = np.ascontiguousarray(ts, dtype=np.float64)
            efeat = None if efeat is None else np.ascontiguousarray(efeat, dtype=np.float32)
            ptrs = [_ptr(a) for a in (src, dst, ts, efeat)]
        st = BatchStats() if stats else None
        rc = self._L.stgn_ingest_batch(self._h, n, *ptrs, 1 if on_dev else 0, C.byref(st) if stats else None)
        if check:
            self._check(rc)
        if stats:
            return st.as_dict() if rc == 0 else rc
        return rc

    def get_embeddings(self, nodes, layer=0):
        torch = self._torch
        if isinstance(nodes, torch.Tensor):
            out = torch.empty((nodes.shape[0], self.cfg.d_emb), dtype=torch.float32, device=nodes.device)
            self._check(self._L.stgn_get_embeddings(self._h, layer, nodes.shape[0], C.c_void_p(nodes.data_ptr()),
                                                    C.c_void_p(out.data_ptr()), 1))
            return out
        nodes = np.ascontiguousarray(nodes, dtype=np.uint32)
        out = np.empty((len(nodes), self.cfg.d_emb), dtype=np.float32)
        self._check(self._L.stgn_get_embeddings(self._h, layer, len(nodes), _ptr(nodes), _ptr(out), 0))
        return out

    def set_predictor(self, w, b):
        w = np.ascontiguousarray(w, dtype=np.float32)
        assert w.shape == (2 * self.cfg.d_emb,)
        self._check(self._L.stgn_set_predictor(self._h, _ptr(w), float(b)))

    def set_predictor_mlp(self, w1, b1, w2, b2, activation="relu"):
        """The head act([h_u | h_v] w1 + b1) . w2 + b2: w1 [2 d_emb, hidden], b1 and w2 [hidden]; activation as in linear.  Captured
        predictions keep their head's width and activation, and follow the parameters set last for those; the workspaces of every width and
        activation set so far are held until close."""
        if activation not in ACTIVATIONS:
            raise ValueError(f"activation must be one of {', '.join(ACTIVATIONS)}")
        w1, b1, w2 = (np.ascontiguousarray(a, dtype=np.float32) for a in (w1, b1, w2))
        hidden = w1.shape[1]
        assert w1.shape == (2 * self.cfg.d_emb, hidden) and b1.shape == (hidden,) and w2.shape == (hidden,)
        n = C.c_size_t(0)
        self._check(self._L.stgn_predictor_mlp_workspace(self._h, hidden, C.byref(n)))
        # one workspace a width and activation, kept: captured predictions, which have both in them, go on reading it, with the parameters set
        # last for that width and activation
        ws = self._head_ws.get((hidden, activation))
        if ws is None:
            # (from the context's own stream: what ran last in memory that another stream has given back may still be running there)
            with self._torch.cuda.stream(self._stream):
                ws = self._head_ws[hidden, activation] = self._torch.empty(n.value + 256, dtype=self._torch.uint8, device=self.device)
        self._check(self._L.stgn_set_predictor_mlp(self._h, hidden, ACTIVATIONS[activation], _ptr(w1), _ptr(b1), _ptr(w2), float(b2),
                                                   C.c_void_p((ws.data_ptr() + 255) & ~255), n.value))

    def predict_batch(self, src, dst, ts, at_edge_time=False):
        """Link scores of edges that have not been ingested yet: numpy in, numpy out (synchronises), or
        torch device tensors in, a device tensor out (asynchronous)."""
        torch = self._torch
        if isinstance(src, torch.Tensor):
            out = torch.empty(src.shape[0], dtype=torch.float32, device=src.device)
            self._check(self._L.stgn_predict_batch(self._h, src.shape[0], C.c_void_p(src.data_ptr()),
                                                   C.c_void_p(dst.data_ptr()), C.c_void_p(ts.data_ptr()),
                                                   int(at_edge_time), 1, C.c_void_p(out.data_ptr())))
            return out
        src = np.ascontiguousarray(src, dtype=np.uint32)
        dst = np.ascontiguousarray(dst, dtype=np.uint32)
        ts = np.ascontiguousarray(ts, dtype=np.float64)
        out = np.empty(len(src), dtype=np.float32)
        self._check(self._L.stgn_predict_batch(self._h, len(src), _ptr(src), _ptr(dst), _ptr(ts), int(at_edge_time), 0,
                                               _ptr(out)))
        return out

    def predict_batch_static(self, src, dst, ts, at_edge_time=False, out=None, check=True):
        """The variant that allocates nothing inside the library: device tensors in, scores into `out`
        (a device tensor the caller provides; created here when omitted).  Returns `out`, or the
        error code when check is off and the call failed."""
        torch = self._torch
        if out is None:
            out = torch.empty(src.shape[0], dtype=torch.float32, device=src.device)
        rc = self._L.stgn_predict_batch_static(self._h, src.shape[0], C.c_void_p(src.data_ptr()),
                                               C.c_void_p(dst.data_ptr()), C.c_void_p(ts.data_ptr()),
                                               int(at_edge_time), C.c_void_p(out.data_ptr()))
        if check:
            self._check(rc)
        return out if rc == 0 else rc

    def full_rebuild(self):
        self._check(self._L.stgn_full_rebuild(self._h))

    def drift_status(self, per_node=False):
        """(global drift metric, size of the cumulative affected set[, per-node estimates]) -- delta mode."""
        g, n = C.c_double(0.0), C.c_uint32(0)
        out = np.empty(self.cfg.num_nodes, dtype=np.float32) if per_node else None
        self._check(self._L.stgn_drift_status(self._h, C.byref(g), C.byref(n), _ptr(out)))
        return (g.value, n.value, out) if per_node else (g.value, n.value)

    def maintain(self, delta_max, alpha):
        """Adaptive rebuild policy; returns (action 0 none / 1 partial / 2 full, |V_drift|) -- delta mode."""
        act, nd = C.c_int(0), C.c_uint32(0)
        self._check(self._L.stgn_maintain(self._h, C.c_double(delta_max), C.c_double(alpha), C.byref(act), C.byref(nd)))
        return act.value, nd.value

    def sync(self, check=True):
        rc = self._L.stgn_sync(self._h)
        if check:
            self._check(rc)
        return rc

    # ---- inspection hooks
    def get_affected(self):
        out = np.empty(self.cfg.num_nodes, dtype=np.uint32)
        cnt = C.c_uint32(0)
        self._check(self._L.stgn_get_affected(self._h, _ptr(out), len(out), C.byref(cnt)))
        return out[:cnt.value].copy()

    def get_neighbors(self, node):
        k = self.cfg.k
        nbr, eid, ts = np.empty(k, np.uint32), np.empty(k, np.uint32), np.empty(k, np.float64)
        cnt = C.c_uint32(0)
        self._check(self._L.stgn_get_neighbors(self._h, int(node), _ptr(nbr), _ptr(eid), _ptr(ts), C.byref(cnt)))
        return nbr[:cnt.value].copy(), eid[:cnt.value].copy(), ts[:cnt.value].copy()

    def get_degree(self, node) -> int:
        dg = C.c_uint32(0)
        self._check(self._L.stgn_get_history(self._h, int(node), 0, 0, None, None, C.byref(dg)))
        return dg.value

    def get_history(self, node, first=0, count=None):
        dg = self.get_degree(node)
        count = dg - first if count is None else count
        nbr, eid = np.empty(count, np.uint32), np.empty(count, np.uint32)
        self._check(self._L.stgn_get_history(self._h, int(node), first, count, _ptr(nbr), _ptr(eid), None))
        return nbr, eid

    def get_memory(self, nodes):
        nodes = np.ascontiguousarray(nodes, dtype=np.uint32)
        mem = np.empty((len(nodes), self.cfg.d_mem), dtype=np.float32)
        tl = np.empty(len(nodes), dtype=np.float64)
        self._check(self._L.stgn_get_memory(self._h, len(nodes), _ptr(nodes), _ptr(mem) if self.cfg.d_mem else None,
                                            _ptr(tl)))
        return mem, tl

    def totals(self):
        v = [C.c_uint64(0) for _ in range(6)]
        self._check(self._L.stgn_get_totals(self._h, *[C.byref(x) for x in v]))
        return dict(zip(("edges", "direct", "affected", "scanned", "gathered", "rows"), [x.value for x in v]))

    def kernel_times(self, enable=True, reset=False):
        cap = 16
        names = (C.c_char_p * cap)()
        us = (C.c_double * cap)()
        ln = (C.c_uint64 * cap)()
        n = self._L.stgn_kernel_times(self._h, int(enable), int(reset), cap, names, us, ln)
        if n < 0:
            self._check(n)
        return {names[i].decode(): dict(usec=us[i], launches=ln[i]) for i in range(n)}


def paper_affected_bound(batch: int, fanout: int, layers: int) -> int:
    """The paper's bound 2 B L^K on the affected-set size (Eq. affected_bound); reported beside
    the measured |A| as context -- it belongs to a looser propagation rule than the exact one."""
    return 2 * batch * fanout ** layers
