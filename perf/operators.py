"""The dense product and the attention of a temporal-attention model as operators on the caller's own tensors, with
their gradients: what a program that learns the link-prediction head or an attention layer from the stream calls, and
what it calls again to answer.

  linear          y = act(x W + b) + r, the values in front of the activation kept where a gradient will need them
  linear_grad     its gradients: inputs, weights, bias
  attention       softmax attention of each list's queries over the list's keys: lists of one query (a node over its
                  neighbours, a new event over a history) up to whole sequences, causal or not, with a window,
                  shared key heads and lists of any length up to the padded one
  attention_grad  its gradients, from the outputs and the logarithms of the softmax sums

A case holds sizes, type and masks; the lists' lengths are a fixed set of numbers that the seed deals out."""
from __future__ import annotations

import math

import torch

own = False

DEVICE = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


def _linear(name, op, dtype, m, k, n, act, bias=True, residual=False, pre=False):
    c = dict(op=op, dtype=dtype, m=m, k=k, n=n, act=act, bias=bias, residual=residual, pre=pre)
    return dict(c, name=name) if name else c


def _attention(name, op, dtype, lists, lq, lk, heads, kv_heads, d, causal=False, window=0, shortest=None):
    c = dict(op=op, dtype=dtype, lists=lists, lq=lq, lk=lk, heads=heads, kv_heads=kv_heads, d=d, causal=causal,
             window=window, shortest=lk if shortest is None else shortest)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the hidden layer of a link-prediction head, for the 2,000 candidate edges of one batch
        _linear("head_hidden", "linear", "f32", 2_000, 200, 100, "relu"),
        # one dense layer for four new tokens: the weights are read once for four rows
        _linear("few_rows", "linear", "bf16", 4, 4_096, 4_096, "silu", residual=True),
        # a training batch through a wide dense layer, the values in front of the activation kept for the gradient
        _linear("wide_dense", "linear", "bf16", 8_192, 4_096, 4_096, "gelu", residual=True, pre=True),
        # gradients of the key|value projection of 4,000 roots' ten neighbours each: inputs [h | e | phi]
        _linear("projection_grad", "linear_grad", "f32", 40_000, 372, 200, "none", bias=False),
        # gradients of a small layer of odd sizes
        _linear("odd_grad", "linear_grad", "f16", 1_531, 1_027, 777, "relu"),
        # gradients of the wide dense layer
        _linear("wide_dense_grad", "linear_grad", "bf16", 8_192, 4_096, 4_096, "gelu"),
        # a layer's attention for the 4,000 roots of a batch over their ten most recent neighbours, some with none
        _attention("neighbours", "attention", "f32", 4_000, 1, 10, 2, 2, 50, shortest=0),
        # one new event per history over histories of up to 32,768 events
        _attention("event_over_history", "attention", "bf16", 24, 1, 32_768, 32, 8, 128, shortest=1_000),
        # whole sequences, each event over the events before it
        _attention("sequences", "attention", "bf16", 4, 4_096, 4_096, 16, 4, 128, causal=True, shortest=2_049),
        # gradients of a layer's attention for 40,000 rows and their twenty neighbours
        _attention("neighbours_grad", "attention_grad", "f32", 40_000, 1, 20, 2, 2, 50, shortest=0),
        # gradients over odd lengths, a window of the last 512 events, narrower heads
        _attention("window_grad", "attention_grad", "f16", 3, 1_777, 1_777, 6, 2, 80, causal=True, window=512, shortest=300),
        # gradients of whole sequences
        _attention("sequences_grad", "attention_grad", "bf16", 4, 4_096, 4_096, 16, 4, 128, causal=True, shortest=2_049),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {op: max((work(c) for c in listed() if c["op"] == op), key=lambda w: w["flops"])["flops"]
            for op in ("linear", "linear_grad", "attention", "attention_grad")}
    op = rng.choice(sorted(most))
    while True:
        dtype = rng.choice(["f32", "bf16", "f16"])
        if op.startswith("linear"):
            rows = rng.choice(["few", "many", "many"])
            c = _linear(None, op, dtype, _log(rng, 1, 16) if rows == "few" else _log(rng, 17, 100_000), _log(rng, 16, 8_192),
                        _log(rng, 1, 8_192), rng.choice(["none", "relu", "gelu", "silu"]), bias=rng.random() < 0.7)
            if op == "linear":
                c["residual"], c["pre"] = rng.random() < 0.4, c["act"] != "none" and rng.random() < 0.3
            if rng.random() < 0.5:
                c["k"], c["n"] = (max(8, v // 8 * 8) for v in (c["k"], c["n"]))
            big = (c["m"] * (c["k"] + 3 * c["n"]) + c["k"] * c["n"]) > 3e8
        else:
            form = rng.choice(["neighbours", "history", "sequences"])
            kv, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 1, 2, 4, 8])
            d = rng.choice([16, 25, 32, 50, 64, 80, 96, 100, 128])
            if form == "neighbours":
                lk = _log(rng, 4, 64)
                c = _attention(None, op, dtype, _log(rng, 100, 60_000), 1, lk, rng.choice([1, 2, 4]), 1, d, shortest=rng.randint(0, lk))
                c["kv_heads"] = c["heads"] if rng.random() < 0.7 else 1
            elif form == "history":
                lk = _log(rng, 500, 60_000)
                c = _attention(None, op, dtype, _log(rng, 1, 64), rng.choice([1, 1, 1, 2, 5]), lk, kv * group, kv, d, causal=rng.random() < 0.5,
                               shortest=rng.randint(lk // 8, lk))
            else:
                lk = _log(rng, 12, 4_096)
                c = _attention(None, op, dtype, _log(rng, 1, 200), lk, lk, kv * group, kv, d, causal=rng.random() < 0.7,
                               shortest=rng.randint(lk // 3, lk))
                if c["causal"] and rng.random() < 0.4:
                    c["window"] = rng.randint(2, lk)
            big = c["lists"] * c["heads"] * c["lq"] * c["lk"] > 1.1e9 or c["lists"] * (c["lk"] * c["kv_heads"] + c["lq"] * c["heads"]) * d > 8e8
        w = work(c)
        if big or max(w["flops"] * (8 if dtype == "f32" else 1), w["bytes"] * 20) > most[op]:
            continue
        return c


def _lengths(c):
    """The lists' numbers of keys: evenly spread from the shortest to the padded length."""
    n, lo, hi = c["lists"], c["shortest"], c["lk"]
    return [hi if n == 1 else lo + (hi - lo) * i // (n - 1) for i in range(n)]


def _seen(c):
    """Pairs of a query and a key that it sees, over all lists, for one head."""
    total = 0
    for lk in _lengths(c):
        lq = min(c["lq"], lk) if c["lq"] > 1 else c["lq"]
        if not c["causal"]:
            total += lq * lk
            continue
        last = lk - lq                                        # the first query sees keys 0 .. last
        w = c["window"] or lk
        whole = max(0, min(lq, w - last - 1))                 # queries that the window does not cut
        total += whole * (last + 1) + whole * (whole - 1) // 2 + (lq - whole) * w
    return total


def work(case):
    c, e = case, BYTES[case["dtype"]]
    if c["op"].startswith("linear"):
        m, k, n = c["m"], c["k"], c["n"]
        if c["op"] == "linear":
            return dict(bytes=e * (m * k + k * n + n * c["bias"] + m * n * (1 + c["residual"] + c["pre"])), flops=2 * m * k * n)
        return dict(bytes=e * (2 * m * k + 2 * k * n + m * n * (1 + (c["act"] != "none")) + n * c["bias"]), flops=4 * m * k * n)
    keys = sum(_lengths(c))
    queries = sum(min(c["lq"], n) if c["lq"] > 1 else 1 for n in _lengths(c))
    kv, q = keys * c["kv_heads"] * c["d"], queries * c["heads"] * c["d"]
    pairs = _seen(c) * c["heads"] * c["d"]
    if c["op"] == "attention":
        return dict(bytes=e * (2 * kv + 2 * q) + 4 * queries * c["heads"], flops=4 * pairs)
    return dict(bytes=e * (4 * kv + 4 * q) + 4 * queries * c["heads"], flops=10 * pairs)


def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if act == "silu":
        s = 1.0 / (1.0 + torch.exp(-z))
        return s * (1.0 + z * (1.0 - s))
    return torch.ones_like(z)


def _masks(s):
    """What each query sees [lists, 1, 1, lq, lk], or None where every list is full; which queries there are [lists, lq]."""
    c = s["case"]
    qn, kn = s["q_lens"], s["k_lens"]
    i = torch.arange(c["lq"], device=DEVICE)
    j = torch.arange(c["lk"], device=DEVICE)
    there = i[None] < qn[:, None]
    see = (j[None, None] < kn[:, None, None]) & there[:, :, None]
    if c["causal"]:
        at = i[None] + (kn - qn)[:, None]
        see &= j[None, None] <= at[:, :, None]
        if c["window"]:
            see &= j[None, None] > at[:, :, None] - c["window"]
    return see[:, None, None]


def _grouped(t, kv_heads):
    """[lists, length, heads, d] -> [lists, kv_heads, heads / kv_heads, length, d] in 32 bits."""
    b, l, h, d = t.shape
    return t.float().reshape(b, l, kv_heads, h // kv_heads, d).permute(0, 2, 3, 1, 4)


def _ungrouped(t, dtype):
    b, kv, g, l, d = t.shape
    return t.permute(0, 3, 1, 2, 4).reshape(b, l, kv * g, d).to(dtype)


def _times(a, b):
    """Products [.., g, i, x] [.., 1, x, j] of the heads that share b, b read once for all of them."""
    n, kv, g, i, x = a.shape
    return (a.reshape(n, kv, g * i, x) @ b[:, :, 0]).reshape(n, kv, g, i, b.shape[-1])


def _shared(a, b):
    """Sums over the heads that share a key head: [.., g, i, x] [.., g, i, y] -> [.., 1, x, y]."""
    n, kv, g, i, x = a.shape
    return (a.reshape(n, kv, g * i, x).transpose(-1, -2) @ b.reshape(n, kv, g * i, b.shape[-1]))[:, :, None]


def _weights(s):
    c = s["case"]
    q, k = _grouped(s["q"], c["kv_heads"]), _grouped(s["k"], c["kv_heads"])
    x = _times(q, k.transpose(-1, -2)) * s["scale"]
    x = x.masked_fill(~_masks(s), -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(torch.isfinite(top), top, torch.zeros_like(top))
    p = torch.exp(x - top)
    total = p.sum(-1, keepdim=True)
    lse = (torch.log(total) + top)[..., 0]
    return q, k, p / torch.where(total > 0, total, torch.ones_like(total)), lse


def _forward(s):
    c = s["case"]
    _, _, p, lse = _weights(s)
    out = _times(p, _grouped(s["v"], c["kv_heads"]))
    n, kv, g, lq = lse.shape
    return _ungrouped(out, s["q"].dtype), lse.reshape(n, kv * g, lq)


def _backward(s):
    c = s["case"]
    q, k, p, _ = _weights(s)
    v, do = _grouped(s["v"], c["kv_heads"]), _grouped(s["dout"], c["kv_heads"])
    do = do * (torch.arange(c["lq"], device=DEVICE)[None] < s["q_lens"][:, None])[:, None, None, :, None]
    dv = _shared(p, do)
    dp = _times(do, v.transpose(-1, -2))
    ds = p * (dp - (p * dp).sum(-1, keepdim=True)) * s["scale"]
    dt = s["q"].dtype
    return _ungrouped(_times(ds, k), dt), _ungrouped(_shared(ds, q), dt), _ungrouped(dv, dt)


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    dt = DTYPES[c["dtype"]]

    def normal(*shape, scale=1.0):
        return (torch.randn(*shape, generator=g, device=DEVICE, dtype=torch.float32) * scale).to(dt)

    if c["op"].startswith("linear"):
        m, k, n = c["m"], c["k"], c["n"]
        s = dict(case=c, x=normal(m, k), w=normal(k, n, scale=k ** -0.5), bias=normal(n, scale=0.1) if c["bias"] else None)
        if c["op"] == "linear":
            s["residual"] = normal(m, n) if c["residual"] else None
        else:
            s["dy"] = normal(m, n)
            s["pre"] = None
            if c["act"] != "none":                            # what the forward call kept
                z = s["x"].float() @ s["w"].float()
                s["pre"] = (z + s["bias"].float() if c["bias"] else z).to(dt)
        return s
    n, lq, lk, d = c["lists"], c["lq"], c["lk"], c["d"]
    lens = torch.tensor(_lengths(c), dtype=torch.int32, device=DEVICE)
    lens = lens[torch.randperm(n, generator=g, device=DEVICE)].contiguous()
    s = dict(case=c, scale=d ** -0.5, k_lens=lens, q_lens=torch.clamp(lens, max=lq) if lq > 1 else torch.ones_like(lens),
             q=normal(n, lq, c["heads"], d), k=normal(n, lk, c["kv_heads"], d), v=normal(n, lk, c["kv_heads"], d))
    if c["op"] == "attention_grad":
        s["dout"] = normal(n, lq, c["heads"], d)
        s["out"], s["lse"] = _forward(s)                      # what the forward call returned
    return s


def run(state):
    s, c = state, state["case"]
    if own:
        from paper_2603_21090_amd import binding
        if c["op"] == "linear":
            return binding.linear(s["x"], s["w"], bias=s["bias"], activation=c["act"], residual=s["residual"], keep_pre=c["pre"])
        if c["op"] == "linear_grad":
            return binding.linear_grad(s["dy"], s["x"], s["w"], activation=c["act"], pre=s["pre"], bias=c["bias"])
        masks = dict(q_lens=s["q_lens"], k_lens=s["k_lens"], causal=c["causal"], window=c["window"], scale=s["scale"])
        if c["op"] == "attention":
            return binding.attention(s["q"], s["k"], s["v"], **masks)
        return binding.attention_grad(s["dout"], s["q"], s["k"], s["v"], s["out"], s["lse"], **masks)
    if c["op"] == "attention":
        return _forward(s)
    if c["op"] == "attention_grad":
        return _backward(s)
    dt = s["x"].dtype
    if c["op"] == "linear":
        z = s["x"].float() @ s["w"].float()
        if s["bias"] is not None:
            z = z + s["bias"].float()
        y = _act(z, c["act"])
        if s["residual"] is not None:
            y = y + s["residual"].float()
        return (y.to(dt), z.to(dt)) if c["pre"] else y.to(dt)
    dz = s["dy"].float()
    if s["pre"] is not None:
        dz = dz * _act_slope(s["pre"].float(), c["act"])
    dx = dz @ s["w"].float().t()
    dw = s["x"].float().t() @ dz
    return dx.to(dt), dw.to(dt), dz.sum(0, dtype=torch.float64).to(dt) if c["bias"] else None


def exact(case, seed):
    """The same from the definitions in 64 bits, list by list."""
    c, s = case, prepare(case, seed)
    if c["op"].startswith("linear"):
        x, w = s["x"].double(), s["w"].double()
        if c["op"] == "linear":
            z = torch.addmm(s["bias"].double(), x, w) if c["bias"] else x @ w
            y = {"none": lambda t: t, "relu": torch.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu}[c["act"]](z)
            y = y if s["residual"] is None else y + s["residual"].double()
            return (y, z) if c["pre"] else y
        dz = s["dy"].double()
        if c["act"] != "none":
            z = s["pre"].double().requires_grad_()
            y = {"relu": torch.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu}[c["act"]](z)
            dz, = torch.autograd.grad(y, z, dz)
        return dz @ w.T, x.T @ dz, dz.sum(0) if c["bias"] else None
    if c["lists"] > 2_000:
        return _exact_short(c, s)
    group = c["heads"] // c["kv_heads"]
    grad = c["op"] == "attention_grad"
    q, k, v = s["q"], s["k"], s["v"]
    out = torch.zeros(q.shape, dtype=torch.float64, device=DEVICE)
    lse = torch.full((c["lists"], c["heads"], c["lq"]), -math.inf, dtype=torch.float64, device=DEVICE)
    dq, dk, dv = (torch.zeros(t.shape, dtype=torch.float64, device=DEVICE) for t in (q, k, v)) if grad else (None,) * 3
    for b, (nq, nk) in enumerate(zip(s["q_lens"].tolist(), s["k_lens"].tolist())):
        if nq == 0 or nk == 0:
            continue
        at = torch.arange(nk - nq, nk, device=DEVICE)[:, None]
        j = torch.arange(nk, device=DEVICE)[None]
        hidden = (j > at) if c["causal"] else torch.zeros(nq, nk, dtype=torch.bool, device=DEVICE)
        if c["window"]:
            hidden = hidden | (j + c["window"] <= at)
        for h in range(c["kv_heads"]):
            heads = slice(h * group, (h + 1) * group)
            qq, kk, vv = q[b, :nq, heads].double().transpose(0, 1), k[b, :nk, h].double(), v[b, :nk, h].double()
            x = torch.where(hidden, -math.inf, (qq @ kk.T) * s["scale"])
            lse[b, heads, :nq] = torch.logsumexp(x, -1)
            p = torch.exp(x - lse[b, heads, :nq, None])
            o = p @ vv
            out[b, :nq, heads] = o.transpose(0, 1)
            if grad:
                do = s["dout"][b, :nq, heads].double().transpose(0, 1)
                dx = p * (do @ vv.T - (do * o).sum(-1, keepdim=True)) * s["scale"]
                dq[b, :nq, heads] = (dx @ kk).transpose(0, 1)
                dk[b, :nk, h] = (dx.transpose(1, 2) @ qq).sum(0)
                dv[b, :nk, h] = (p.transpose(1, 2) @ do).sum(0)
    return (dq, dk, dv) if grad else (out, lse)


def _exact_short(c, s):
    """Many short lists of one query, every list at once: [lists, heads, keys] as sums over the heads' numbers."""
    group = c["heads"] // c["kv_heads"]
    if c["lq"] != 1:
        return None
    q = s["q"][:, 0].double()                                                        # lists, heads, d
    k, v = (s[t].double().repeat_interleave(group, 2) for t in ("k", "v"))           # lists, keys, heads, d
    there = torch.arange(c["lk"], device=DEVICE)[None, :, None] < s["k_lens"][:, None, None]
    x = torch.where(there, (q[:, None] * k).sum(-1) * s["scale"], -math.inf)         # lists, keys, heads
    lse = torch.logsumexp(x, 1)
    p = torch.where(there, torch.exp(x - lse[:, None]), 0.0)
    out = (p[..., None] * v).sum(1)
    if c["op"] == "attention":
        return out[:, None], lse[..., None]
    do = s["dout"][:, 0].double()
    dx = p * ((do[:, None] * v).sum(-1) - (do * out).sum(-1)[:, None]) * s["scale"]
    fold = lambda t: t.reshape(c["lists"], c["lk"], c["kv_heads"], group, c["d"]).sum(3)  # noqa: E731
    return (dx[..., None] * k).sum(1)[:, None], fold(dx[..., None] * q[:, None]), fold(p[..., None] * do[:, None])
