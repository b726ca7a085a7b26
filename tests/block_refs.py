"""The norm, operands in 8 bits, their product and dropout in 64 bits, plainly, with the largest error that a kernel's roundings can make
beside each result (U, HALF and `rounded`: operator_refs)."""
import numpy as np
import torch

from operator_refs import U, act, rounded

EPS = 1e-6


def rms_norm(x, residual, gain, eps=EPS):
    """(y, bound), (h, bound), both rounded to the type.  h: one fp32 addition, u |h|.  r: the mean moves by 2 u with h, r by u, and is rounded,
    u.  y = h r g: those and two products."""
    dt = x.dtype
    h = x.double() + (residual.double() if residual is not None else 0.0)
    r = 1.0 / torch.sqrt((h * h).mean(1, keepdim=True) + eps)
    y = h * r * gain.double()
    return (y, rounded(y, 6 * U * y.abs(), dt)), (h, rounded(h, U * h.abs(), dt))


def rms_norm_grad(dy, h, gain, dh, eps=EPS):
    """(dx, bound), (dgain, bound).  dx = r (t - (h r) back): t = g dy (u), r (u), back = r mean(t h), a sum of 64 bits of t's errors (u),
    r's and its own rounding (2 u), h r (2 u), the difference one u, the product with r two, with dh's addition in it one more."""
    dt = h.dtype
    h, dy, gain = h.double(), dy.double(), gain.double()
    r = 1.0 / torch.sqrt((h * h).mean(1, keepdim=True) + eps)
    t = gain * dy
    back = r ** 3 * (t * h).mean(1, keepdim=True)
    dx = r * t - h * back
    e = 3 * U * (r * t).abs() + 7 * U * h.abs() * r ** 3 * (t * h).abs().mean(1, keepdim=True) + U * dx.abs()
    if dh is not None:
        dx = dx + dh.double()
        e = e + U * dx.abs()
    terms = dy * h * r
    dg = terms.sum(0)
    return (dx, rounded(dx, 2 * e, dt)), (dg, rounded(dg, 2 * (h.shape[0] + 4) * U * terms.abs().sum(0), dt))


def eight(y):
    """(q, scale) of fp32 rows, exactly: the quotient in 64 bits, where halves are halves (127 y is exact there)."""
    y = y.double()
    top = y.abs().amax(1, keepdim=True) if y.shape[1] else torch.zeros(y.shape[0], 1, dtype=torch.float64)
    bad = ~torch.isfinite(top)                                # (amax hands a NaN on)
    q = torch.round(127.0 * y / torch.where((top > 0) & ~bad, top, torch.ones_like(top)))
    q = torch.where(bad, 0.0, q).to(torch.int8)
    return q, torch.where(bad, float("nan"), top / 127.0).float()[:, 0]


def linear_i8(x, xs, w, ws, bias, name, residual, dtype):
    """(y, bound): an exact sum, its conversion and two scales 3 u of it, the bias's addition, then as the dense product of other types."""
    z0 = (x.double() @ w.double().T) * xs.double()[:, None] * ws.double()
    z, ez = z0, 3 * U * z0.abs()
    if bias is not None:
        z = z0 + bias.double()
        ez = ez + U * z.abs()
    y, ey = act(z, name), 1.13 * 1.1 * ez + (2.0 ** -21 * z.abs() if name in ("gelu", "silu") else 0.0)
    if residual is not None:
        y = y + residual.double()
        ey = ey + 2 * U * (y.abs() + residual.double().abs())
    return y, rounded(y, ey, dtype)


def philox(counter, key):
    """Philox 4x32 with ten rounds: counter four arrays, key two numbers of 32 bits."""
    low, mask = np.uint64(32), np.uint64(0xFFFFFFFF)
    x = [np.asarray(c, dtype=np.uint64) for c in counter]
    key = list(key)
    for _ in range(10):
        p, q = np.uint64(0xD2511F53) * x[0], np.uint64(0xCD9E8D57) * x[2]
        x = [(q >> low) ^ x[1] ^ np.uint64(key[0]), q & mask, (p >> low) ^ x[3] ^ np.uint64(key[1]), p & mask]
        key = [(key[0] + 0x9E3779B9) & 0xFFFFFFFF, (key[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return x


def kept(rows, width, p, seed, step, site, first_row=0):
    """Which numbers dropout keeps [rows, width]; seed and step as unsigned 64-bit numbers."""
    groups = -(-width // 8)
    at = np.arange(first_row * groups, (first_row + rows) * groups, dtype=np.uint64)
    same = lambda v: np.full_like(at, v)  # noqa: E731
    words = philox([at & np.uint64(0xFFFFFFFF), (at >> np.uint64(32)) | same(site << 16), same(step & 0xFFFFFFFF), same(step >> 32)],
                   [seed & 0xFFFFFFFF, seed >> 32])
    halves = np.stack([h for w in words for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))], 1).astype(np.int64)
    return torch.from_numpy(halves.reshape(rows, groups * 8)[:, :width] >= round(p * 65536))


def dropout(x, p, mask, residual):
    """(y, bound): the factor and the product round once each, the residual's addition once."""
    border = round(p * 65536)
    y = torch.where(mask, x.double() * (65536 / (65536 - border) if border < 65536 else 0.0), 0.0)
    e = 2.01 * U * y.abs()
    if residual is not None:
        y = y + residual.double()
        e = e + U * y.abs()
    return y, rounded(y, 1.01 * e, x.dtype)
