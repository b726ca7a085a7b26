"""What stands between the dense products of a residual block, trained and served, as operators on the caller's own tensors.

  rms_norm       y = h g / sqrt(mean h^2 + eps) with h = x + residual, h handed out too: the residual stream and its norm
  rms_norm_grad  its gradients: of the stream (what comes down the stream added) and of the gain
  linear_i8      y = act(x_scale w_scale sum x w + b) + r from operands in 8 bits, a scale for each row and each output column; the rows come
                 given in 8 bits, from a tensor that is brought to 8 bits first, or straight out of the norm
  quantize       a weight in 8 bits, its columns' scales, laid out for linear_i8
  dropout        y = residual + kept x / (1 - p), kept or not by numbers of a counter-based generator (seed, step, call site, place); its
                 gradient is the same call on dy

A case holds sizes, type and which parts take part."""
from __future__ import annotations

import math

import torch

own = False

DEVICE = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-6


def _norm(name, op, dtype, rows, width, residual=False):
    c = dict(op=op, dtype=dtype, rows=rows, width=width, residual=residual)
    return dict(c, name=name) if name else c


def _product(name, dtype, m, k, n, act, entry, bias=True, residual=False):
    c = dict(op="linear_i8", dtype=dtype, m=m, k=k, n=n, act=act, entry=entry, bias=bias, residual=residual)
    return dict(c, name=name) if name else c


def _quantize(name, dtype, rows, width):
    c = dict(op="quantize", dtype=dtype, rows=rows, width=width)
    return dict(c, name=name) if name else c


def _dropout(name, dtype, rows, width, p, residual=False, grad=False):
    c = dict(op="dropout", dtype=dtype, rows=rows, width=width, p=p, residual=residual, grad=grad)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the norm in front of a block, for one new token
        _norm("norm_token", "rms_norm", "bf16", 1, 4_096, residual=True),
        # key|value inputs of 4,000 roots' ten neighbours each, brought to one length before they are projected
        _norm("norm_rows", "rms_norm", "f32", 40_000, 200),
        # a training batch: the residual stream and its norm
        _norm("norm_batch", "rms_norm", "bf16", 16_384, 4_096, residual=True),
        # gradients of the neighbours' rows
        _norm("norm_rows_grad", "rms_norm_grad", "f32", 40_000, 200),
        # gradients of the training batch, with the stream's own gradient added
        _norm("norm_batch_grad", "rms_norm_grad", "bf16", 16_384, 4_096, residual=True),
        # four new tokens: the norm into 8 bits and a dense layer, its weights read once for four rows
        _product("token_block", "bf16", 4, 4_096, 4_096, "silu", "rms_norm"),
        # a layer of odd sizes on activations that come in 16 bits
        _product("odd_layer", "f16", 1_531, 1_027, 777, "relu", "quantize", residual=True),
        # a prompt's rows through the norm and a layer that widens them
        _product("prompt_block", "bf16", 2_048, 4_096, 8_192, "gelu", "rms_norm", bias=False),
        # a large batch through a wide dense layer, rows in 8 bits already
        _product("wide_layer", "bf16", 8_192, 4_096, 4_096, "gelu", "given", residual=True),
        # the weight of the wide layer brought to 8 bits, once it has been learnt
        _quantize("weight", "bf16", 4_096, 4_096),
        # the hidden rows of a link-prediction head in training, 4,000 candidate edges
        _dropout("dropout_rows", "f32", 4_000, 200, 0.1),
        # a training batch's sublayer added to the residual stream
        _dropout("dropout_batch", "bf16", 16_384, 4_096, 0.1, residual=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {}
    for c in listed():
        w = work(c)
        b, f = most.get(c["op"], (0, 0))
        most[c["op"]] = (max(b, w["bytes"]), max(f, w["flops"]))
    op = rng.choice(["rms_norm", "rms_norm_grad", "linear_i8", "linear_i8", "quantize", "dropout"])
    while True:
        dtype = rng.choice(["f32", "bf16", "f16"])
        rows = _log(rng, 1, 64) if rng.random() < 0.35 else _log(rng, 65, 100_000)
        width = _log(rng, 8, 16_384)
        if rng.random() < 0.5:
            width = max(8, width // 8 * 8)
        if op.startswith("rms_norm"):
            c = _norm(None, op, dtype, rows, width, residual=rng.random() < 0.6)
        elif op == "linear_i8":
            k, n = min(width, 8_192), _log(rng, 1, 8_192)
            if rng.random() < 0.5:
                k, n = max(16, k // 16 * 16), max(16, n // 16 * 16)
            c = _product(None, dtype, rows, k, n, rng.choice(["none", "relu", "gelu", "silu"]), rng.choice(["given", "quantize", "rms_norm"]),
                         bias=rng.random() < 0.7, residual=rng.random() < 0.4)
        elif op == "quantize":
            c = _quantize(None, dtype, _log(rng, 16, 8_192), min(width, 8_192))
        else:
            grad = rng.random() < 0.4
            c = _dropout(None, dtype, rows, width, rng.choice([0.05, 0.1, 0.25, 0.5]), residual=not grad and rng.random() < 0.5, grad=grad)
        w = work(c)
        # (a product's rows may be wider or more than the largest case's: its bytes are bounded by their sum)
        if w["bytes"] <= most[op][0] * (2 if op == "linear_i8" else 1) and w["flops"] <= most[op][1]:
            return c


def work(case):
    c, e = case, BYTES[case["dtype"]]
    if c["op"] == "linear_i8":
        m, k, n = c["m"], c["k"], c["n"]
        rows = {"given": m * k + 4 * m, "quantize": e * m * k, "rms_norm": e * (3 * m * k + k)}[c["entry"]]     # (norm: x, residual, h)
        return dict(bytes=rows + n * k + 4 * n + e * (n * c["bias"] + m * n * (1 + c["residual"])), flops=2 * m * k * n)
    n = c["rows"] * c["width"]
    if c["op"] == "rms_norm":
        return dict(bytes=e * (n * (2 + 2 * c["residual"]) + c["width"]), flops=5 * n)
    if c["op"] == "rms_norm_grad":
        return dict(bytes=e * (n * (3 + c["residual"]) + 2 * c["width"]), flops=12 * n)
    if c["op"] == "quantize":
        return dict(bytes=(e + 1) * n + 4 * c["width"], flops=3 * n)
    return dict(bytes=e * n * (2 + c["residual"]), flops=20 * n)                     # (ten rounds of two wide products for eight numbers)


def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _normed(x, residual, gain):
    """(h, y) in 32 bits.  The mean is a sum of 64 bits rounded once: what becomes of a value next to a border of two 8-bit numbers shall not hang
    on the order of a sum."""
    h = x.float() if residual is None else x.float() + residual.float()
    wide = h.double()
    r = (1.0 / torch.sqrt((wide * wide).mean(1, keepdim=True) + EPS)).float()
    return h, h * r * gain.float()


def _eight(y):
    """(numbers of 8 bits as floats, scales [rows, 1]) of rows in 32 bits: the quotient in 64, where halves stay halves (and go to the even
    neighbour)."""
    top = y.abs().amax(1, keepdim=True).double()
    q = torch.round(y.double() * 127.0 / torch.where(top > 0, top, torch.ones_like(top)))
    return q.float(), (top / 127.0).float()


M0, M1, W0, W1, LOW = 0xD2511F53, 0xCD9E8D57, 0x9E3779B9, 0xBB67AE85, 0xFFFFFFFF


def _kept(rng, site, rows, width, p):
    """Philox 4x32 with ten rounds (Salmon, Moraes, Dror and Shaw, 2011), eight numbers of 16 bits a call."""
    groups = (width + 7) // 8
    at = torch.arange(rows * groups, device=DEVICE)
    seed, step = rng[0], rng[1]
    zero = torch.zeros_like(at)
    a, b, c, d = at & LOW, (at >> 32) | site << 16, zero + (step & LOW), zero + ((step >> 32) & LOW)
    k0, k1 = seed & LOW, (seed >> 32) & LOW
    for _ in range(10):
        u, v = a * M0, c * M1
        a, b, c, d = (v >> 32) & LOW ^ b ^ k0, v & LOW, (u >> 32) & LOW ^ d ^ k1, u & LOW
        k0, k1 = (k0 + W0) & LOW, (k1 + W1) & LOW
    words = torch.stack([a, b, c, d], 1)
    halves = torch.stack([words & 0xFFFF, words >> 16], 2).reshape(rows, groups * 8)
    return halves[:, :width] >= round(p * 65536)


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    dt = DTYPES[c["dtype"]]

    def normal(*shape, scale=1.0, about=0.0):
        return (torch.randn(*shape, generator=g, device=DEVICE, dtype=torch.float32) * scale + about).to(dt)

    if c["op"] == "linear_i8":
        m, k, n = c["m"], c["k"], c["n"]
        s = dict(case=c, x=normal(m, k), gain=normal(k, scale=0.1, about=1.0), bias=normal(n, scale=0.1) if c["bias"] else None,
                 residual=normal(m, n) if c["residual"] else None, stream=normal(m, k) if c["entry"] == "rms_norm" else None)
        q, scale = _eight(normal(n, k, scale=k ** -0.5).float())       # the learnt weight, in 8 bits once and for all
        s["w"], s["w_scale"] = q.to(torch.int8), scale[:, 0].contiguous()
        if c["entry"] == "given":
            q, scale = _eight(s["x"].float())
            s["xq"], s["x_scale"] = q.to(torch.int8), scale[:, 0].contiguous()
        return s
    rows, width = c["rows"], c["width"]
    s = dict(case=c, x=normal(rows, width, scale=width ** -0.5 if c["op"] == "quantize" else 1.0))
    if c["op"] == "dropout":
        s["residual"] = normal(rows, width) if c["residual"] else None
        s["rng"] = torch.randint(0, 1 << 40, (2,), generator=g, device=DEVICE)       # seed, step
    elif c["op"] != "quantize":
        s["residual"] = normal(rows, width) if c["residual"] else None               # (gradient: what comes down the stream)
        s["gain"] = normal(width, scale=0.1, about=1.0)
        s["dy"] = normal(rows, width) if c["op"] == "rms_norm_grad" else None
    return s


def _run_own(s, c):
    from paper_2603_21090_amd import binding
    if c["op"] == "rms_norm":
        if c["residual"]:
            return binding.rms_norm(s["x"], s["gain"], residual=s["residual"], eps=EPS)
        return binding.rms_norm(s["x"], s["gain"], eps=EPS)
    if c["op"] == "rms_norm_grad":
        return binding.rms_norm_grad(s["dy"], s["x"], s["gain"], dh=s["residual"], eps=EPS)
    if c["op"] == "quantize":
        q, scale = binding.quantize(s["x"], columns=True)
        return q * scale[:, None]                             # the values that the numbers stand for
    if c["op"] == "dropout":
        if c["grad"]:
            return binding.dropout_grad(s["x"], c["p"], s["rng"], site=3)
        return binding.dropout(s["x"], c["p"], s["rng"], site=3, residual=s["residual"])
    tail = dict(bias=s["bias"], activation=c["act"], residual=s["residual"], dtype=s["x"].dtype)
    if c["entry"] == "rms_norm":
        q, scale, h = binding.rms_norm_i8(s["x"], s["gain"], residual=s["stream"], eps=EPS)
        return binding.linear_i8(q, scale, s["w"], s["w_scale"], **tail), h
    q, scale = binding.quantize(s["x"]) if c["entry"] == "quantize" else (s["xq"], s["x_scale"])
    return binding.linear_i8(q, scale, s["w"], s["w_scale"], **tail)


def run(state):
    s, c = state, state["case"]
    if own:
        return _run_own(s, c)
    dt = s["x"].dtype
    if c["op"] == "rms_norm":
        h, y = _normed(s["x"], s["residual"], s["gain"])
        return (y.to(dt), h.to(dt)) if c["residual"] else y.to(dt)
    if c["op"] == "rms_norm_grad":
        h, dy, gain = s["x"].float(), s["dy"].float(), s["gain"].float()
        r = 1.0 / torch.sqrt((h * h).mean(1, keepdim=True) + EPS)
        t = dy * gain
        dx = t * r - h * (r * r * r * (t * h).mean(1, keepdim=True))
        if c["residual"]:
            dx = dx + s["residual"].float()
        return dx.to(dt), (dy * h * r).sum(0, dtype=torch.float64).to(dt)
    if c["op"] == "quantize":
        q, scale = _eight(s["x"].float().t())
        return q * scale
    if c["op"] == "dropout":
        border = round(c["p"] * 65536)
        y = torch.where(_kept(s["rng"], 3, c["rows"], c["width"], c["p"]), s["x"].float() * (65536 / (65536 - border)), torch.zeros((), device=DEVICE))
        return (y + s["residual"].float()).to(dt) if c["residual"] else y.to(dt)
    h = None
    if c["entry"] == "rms_norm":
        h, y = _normed(s["x"], s["stream"], s["gain"])
        x, scale = _eight(y)
    elif c["entry"] == "quantize":
        x, scale = _eight(s["x"].float())
    else:
        x, scale = s["xq"].float(), s["x_scale"][:, None]
    z = (x @ s["w"].float().t()) * scale * s["w_scale"]
    if s["bias"] is not None:
        z = z + s["bias"].float()
    y = _act(z, c["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return (y.to(dt), h.to(dt)) if c["entry"] == "rms_norm" else y.to(dt)


def _steps(rows):
    """Rows as steps of a 127th of their largest magnitude: (whole numbers, the step)."""
    top = rows.abs().max(1).values
    return torch.round(127.0 * rows / top.clamp_min(1e-300)[:, None]), top / 127.0


def exact(case, seed):
    """The same from the definitions in 64 bits."""
    c, s = case, prepare(case, seed)
    x = s["x"].double()
    if c["op"] == "quantize":
        whole, step = _steps(x.T.contiguous())
        return whole * step[:, None]
    if c["op"] == "dropout":
        kept = _philox_mask(s["rng"].tolist(), 3, c)
        border = int(round(c["p"] * 65536))
        y = x.masked_fill(~kept, 0.0).div(1.0 - border / 65536)
        return y if s["residual"] is None else y.add(s["residual"].double())
    gain = s["gain"].double()
    if c["op"] == "rms_norm_grad":
        lead, g = x.requires_grad_(), gain.requires_grad_()
        y = lead / lead.pow(2).mean(-1, keepdim=True).add(EPS).sqrt() * g
        dx, dg = torch.autograd.grad(y, (lead, g), s["dy"].double())
        return (dx if s["residual"] is None else dx + s["residual"].double()), dg
    residual = s["stream"] if c["op"] == "linear_i8" else s["residual"]
    h = x if residual is None else x + residual.double()
    unit = h * torch.rsqrt(h.square().sum(-1, keepdim=True) / h.shape[1] + EPS)
    if c["op"] == "rms_norm":
        return unit * gain if residual is None else (unit * gain, h)
    if c["entry"] == "given":
        whole, step = s["xq"].double(), s["x_scale"].double()
    else:
        whole, step = _steps(unit * gain if c["entry"] == "rms_norm" else x)
    y = torch.matmul(whole * step[:, None], (s["w"].double() * s["w_scale"].double()[:, None]).T)
    if c["bias"]:
        y += s["bias"].double()
    y = {"none": lambda t: t, "relu": torch.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu}[c["act"]](y)
    if c["residual"]:
        y += s["residual"].double()
    return (y, h) if c["entry"] == "rms_norm" else y


def _philox_mask(rng, site, c):
    """Which elements are kept, by the generator's definition on the host: words of 32 bits in numpy's wrapping arithmetic."""
    import numpy as np
    seed, step = rng
    rows, groups = c["rows"], -(-c["width"] // 8)
    n = np.arange(rows * groups, dtype=np.uint64)
    low = np.uint64(32)
    mask = np.uint64(0xFFFFFFFF)
    x = [n & mask, (n >> low) | np.uint64(site << 16), np.full_like(n, step & 0xFFFFFFFF), np.full_like(n, step >> 32)]
    key = [seed & 0xFFFFFFFF, seed >> 32]
    for i in range(10):
        k = [np.uint64((key[j] + i * (0x9E3779B9, 0xBB67AE85)[j]) & 0xFFFFFFFF) for j in range(2)]
        p, q = np.uint64(0xD2511F53) * x[0], np.uint64(0xCD9E8D57) * x[2]
        x = [(q >> low) ^ x[1] ^ k[0], q & mask, (p >> low) ^ x[3] ^ k[1], p & mask]
    numbers = np.stack([h for w in x for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))], 1).astype(np.int32)
    kept = numbers.reshape(rows, groups * 8)[:, :c["width"]] >= int(round(c["p"] * 65536))
    return torch.from_numpy(np.ascontiguousarray(kept)).to(DEVICE)
