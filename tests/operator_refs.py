"""The operators in 64 bits, plainly, with the largest error that a kernel's roundings can make beside each result.

u = 2^-24 is half a step of the fp32 sums.  A sum of n products of exact factors, in any order, is off by at most n u times
the sum of the products' magnitudes (products of 16-bit factors are exact in fp32); twice that is allowed, for matrix
instructions whose inner additions round in a way of their own.  h is half a step of the element type (2^-8 for bf16,
2^-11 for fp16, 2^-24 for fp32): one for every rounding to the type, that is for results and for the factors of a second product."""
import math

import torch

U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -25}      # half a step of the smallest numbers (of what is normal)


def act(z, name):
    if name == "relu":
        return z.clamp_min(0.0)
    if name == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z / math.sqrt(2.0)))
    if name == "silu":
        return z * torch.sigmoid(z)
    return z


def act_slope(z, name):
    if name == "relu":
        return (z > 0).double()
    if name == "gelu":
        return 0.5 * (1.0 + torch.erf(z / math.sqrt(2.0))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if name == "silu":
        s = torch.sigmoid(z)
        return s * (1.0 + z * (1.0 - s))
    return torch.ones_like(z)


def rounded(value, err, dtype):
    """The error bound of a value that is off by err when it is rounded to the type."""
    return err + HALF[dtype] * (value.abs() + err) + TINY[dtype]


def linear(x, w, bias, name, residual):
    """(y, its bound), (z, its bound).  act's slope is at most 1.13; the function itself is good to 2^-21 of |z| (erf and exp in fp32)."""
    dt = x.dtype
    x, w = x.double(), w.double()
    z, mag = x @ w, x.abs() @ w.abs()
    if bias is not None:
        z, mag = z + bias.double(), mag + bias.double().abs()
    ez = 2 * (x.shape[1] + 1) * U * mag
    y, ey = act(z, name), 1.13 * ez + (2.0 ** -21 * z.abs() if name in ("gelu", "silu") else 0.0)
    if residual is not None:
        y = y + residual.double()
        ey = ey + 2 * U * (y.abs() + residual.double().abs())
    return (y, rounded(y, ey, dt)), (z, rounded(z, ez, dt))


def linear_grad(dy, x, w, name, pre):
    """(dx, bound), (dw, bound), (db, bound)."""
    dt = x.dtype
    h = HALF[dt] if name != "none" else 0.0                   # dz is dy itself without an activation
    dz = dy.double() * (act_slope(pre.double(), name) if name != "none" else 1.0)
    slack = 2.0 ** -20 * dy.double().abs() if name in ("gelu", "silu") else 0.0 * dz      # slopes to 2^-20: two functions and their products
    edz = (h * dz.abs() + slack + (TINY[dt] if h else 0.0))
    x, w = x.double(), w.double()

    def bound(value, a, ea, b, n):
        return rounded(value, ea @ b.abs() + 2 * (n + 1) * U * (a.abs() @ b.abs()), dt)
    dx, dw, db = dz @ w.T, x.T @ dz, dz.sum(0)
    return ((dx, bound(dx, dz, edz, w.T, w.shape[1])), (dw, bound(dw.T, dz.T, edz.T, x, x.shape[0]).T),
            (db, rounded(db, edz.sum(0) + 2 * (x.shape[0] + 1) * U * dz.abs().sum(0), dt)))


def visible(lists, q_len, k_len, q_lens, k_lens, causal, window):
    qn = q_lens if q_lens is not None else torch.full((lists,), q_len)
    kn = k_lens if k_lens is not None else torch.full((lists,), k_len)
    i, j = torch.arange(q_len)[None, :, None], torch.arange(k_len)[None, None]
    qn, kn = qn.long()[:, None, None], kn.long()[:, None, None]
    see = (i < qn) & (j < kn)
    if causal:
        see &= j <= i + kn - qn
        if window:
            see &= j > i + kn - qn - window
    return see


def attention(q, k, v, see, scale, dout=None):
    """dict of name -> (value, bound): out and lse, and dq, dk, dv where dout is given (from the out and lse a kernel returned,
    which are off by their own bounds).  What no query sees is taken as zero, whatever it holds."""
    dt, h, group, d = q.dtype, HALF[q.dtype], q.shape[2] // k.shape[2], q.shape[3]
    hp = h if dt != torch.float32 else 0.0                    # softmax weights and ds as factors of a second product
    used_q, used_k = see.any(2)[..., None, None], see.any(1)[..., None, None]
    clean = lambda t, use: torch.where(use, t.double(), 0.0).permute(0, 2, 1, 3)  # noqa: E731  lists, heads, rows, d
    q, k, v = clean(q, used_q), clean(k, used_k).repeat_interleave(group, 1), clean(v, used_k).repeat_interleave(group, 1)
    see = see[:, None]
    n = see.shape[-1]
    s = scale * (q @ k.transpose(2, 3))
    es = 2 * (d + 2) * U * abs(scale) * (q.abs() @ k.abs().transpose(2, 3)) + 2.0 ** -22 * s.abs()
    some = see.any(-1)
    s = torch.where(see, s, -math.inf)
    es = torch.where(see, es, 0.0)
    lse = torch.logsumexp(s, -1)
    worst = es.amax(-1)                                       # of the row's scores
    elk = 2 * (n + 8) * U + 2.0 ** -20                        # exp2, log2 and the sum of the weights
    elem = worst + elk + 2.0 ** -22 * torch.where(some, lse, 0.0).abs()
    p = torch.where(see, torch.exp(s - torch.where(some, lse, 0.0)[..., None]), 0.0)
    ep = p * 2.5 * (es + elem[..., None])                     # e^x - 1 <= 1.25 x here, numerator and denominator
    out = p @ v
    eout = ep @ v.abs() + (hp + 2 * (n + 2) * U) * (p @ v.abs())
    eout = rounded(out, eout, dt)
    back = lambda t: t.permute(0, 2, 1, 3)                    # noqa: E731
    got = {"out": (back(out), back(eout)), "lse": (torch.where(some, lse, -math.inf), elem)}
    if dout is None:
        return got
    fold = lambda t: back(t.reshape(t.shape[0], t.shape[1] // group, group, t.shape[2], d).sum(2))  # noqa: E731
    do = clean(dout, used_q)
    dv, mag = p.transpose(2, 3) @ do, p.transpose(2, 3) @ do.abs()
    edv = ep.transpose(2, 3) @ do.abs() + (hp + 2 * (group * see.shape[2] + 2) * U) * mag
    dp = do @ v.transpose(2, 3)
    edp = 2 * (d + 2) * U * (do.abs() @ v.abs().transpose(2, 3))
    delta = (do * out).sum(-1, keepdim=True)
    edelta = (do.abs() * eout).sum(-1, keepdim=True) + 2 * (d + 2) * U * (do * out).abs().sum(-1, keepdim=True)
    ds = p * (dp - delta)
    eds = ep * (dp - delta).abs() + (p + ep) * (edp + edelta + 2 * U * (dp.abs() + delta.abs()))
    eds = eds + hp * (ds.abs() + eds) + (TINY[dt] if hp else 0.0) * see
    dq, edq = scale * (ds @ k), abs(scale) * (eds @ k.abs() + 2 * (n + 2) * U * (ds.abs() @ k.abs()))
    dk = scale * (ds.transpose(2, 3) @ q)
    edk = abs(scale) * (eds.transpose(2, 3) @ q.abs() + 2 * (group * see.shape[2] + 2) * U * (ds.abs().transpose(2, 3) @ q.abs()))
    dk, edk, dv, edv = fold(dk), fold(edk), fold(dv), fold(edv)
    got["dq"] = (back(dq), back(rounded(dq, edq, dt)))
    got["dk"] = (dk, rounded(dk, edk, dt))
    got["dv"] = (dv, rounded(dv, edv, dt))
    return got


def within(got, want, name=""):
    """got (any device) lies within the bound of want = (value, bound); infinities equal."""
    value, bound = want
    got = got.detach().double().cpu()
    assert got.shape == value.shape, name
    same = torch.isinf(value)
    assert torch.equal(got[same], value[same]), name
    off = torch.where(same, 0.0, (got - torch.where(same, 0.0, value)).abs())
    bad = ~(off <= torch.where(same, 1.0, bound))             # (a NaN is bad)
    if bad.any():
        at = tuple(int(x) for x in bad.nonzero()[0])
        raise AssertionError(f"{name}: {int(bad.sum())} of {bad.numel()} outside, first at {at}: got {got[at]}, want {value[at]} +- {bound[at]}")
