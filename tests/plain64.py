"""Plain 64-bit statements of the operators around the projection, and the error bounds of 32-bit sums.

``U`` is the unit roundoff of fp32.  A sum formed by chains of at most ``CHAIN`` additions and a tree
over at most 1024 partial sums is off by at most (CHAIN + 10) U times the sum of the magnitudes."""
import math

import torch

U = 2.0 ** -24
CHAIN = 64
ROUND = {torch.float32: U, torch.bfloat16: 2.0 ** -8}      # half a unit in the last place of 24 and of 8 significant bits


def norm_forward(x, w=None, c=None, r=None, eps=1e-5, rms=False):
    h = x.double() if r is None else x.double() + r.double()
    mean = torch.zeros(h.shape[0], dtype=torch.float64, device=h.device) if rms else h.sum(1) / h.shape[1]
    d = h - mean[:, None]
    rstd = 1.0 / torch.sqrt((d * d).sum(1) / h.shape[1] + eps)
    y = d * rstd[:, None]
    if w is not None:
        y = y * w.double()
    if c is not None:
        y = y + c.double()
    return y, h, mean, rstd


def norm_forward_bounds(x, w=None, c=None, r=None, eps=1e-5, rms=False):
    """Element-wise bounds for y before it is stored, for h, mean and rstd."""
    y, h, mean, rstd = norm_forward(x, w, c, r, eps, rms)
    s = (CHAIN + 10) * U
    size = h.abs().sum(1) / h.shape[1]
    off = (0.0 if rms else s) * size + 2 * U * size          # the mean's error, and that of r's addition
    rel = s + 8 * U + (off * rstd) ** 2 + 2 * U * size * rstd       # of rstd
    scale = torch.ones_like(h[0]) if w is None else w.double().abs()
    d = (h - mean[:, None]).abs()
    by = (d * (rel * rstd + 4 * U * rstd)[:, None] + (2 * U * h.abs() + off[:, None]) * rstd[:, None]) * scale
    by = by + 2 * U * (y.abs() + (0 if c is None else c.double().abs()))
    return by, 2 * U * h.abs(), off + 2 * U * mean.abs(), rel * rstd


def norm_backward(dy, x, mean, rstd, w=None, dh=None, rms=False):
    x, dy = x.double(), dy.double()
    n = x.shape[1]
    u = (x if rms else x - mean.double()[:, None]) * rstd.double()[:, None]
    g = dy if w is None else dy * w.double()
    dx = g - u * ((g * u).sum(1) / n)[:, None]
    if not rms:
        dx = dx - (g.sum(1) / n)[:, None]
    dx = dx * rstd.double()[:, None]
    if dh is not None:
        dx = dx + dh.double()
    return dx, (dy * u).sum(0), dy.sum(0)


def norm_backward_bounds(dy, x, mean, rstd, w=None, dh=None, rms=False):
    x, dy = x.double(), dy.double()
    b, n = x.shape
    s = (CHAIN + 10) * U
    u = ((x if rms else x - mean.double()[:, None]) * rstd.double()[:, None]).abs()
    g = (dy if w is None else dy * w.double()).abs()
    size = g + u * ((g * u).sum(1) / n)[:, None]
    if not rms:
        size = size + (g.sum(1) / n)[:, None]
    dx = (s + 10 * U) * size * rstd.double().abs()[:, None]
    if dh is not None:
        dx = dx + 2 * U * dh.double().abs()
    chain = (min(b, 1000) + 16) * U          # rows of a range, and the ranges
    return dx, chain * (dy.abs() * u).sum(0), chain * dy.abs().sum(0)


def rotary_frequencies(rot, base=10000.0):
    return [base ** (-2.0 * i / rot) for i in range(rot // 2)]


def rotary(x, cos, sin, rotated, rot, interleaved, transposed):
    """x: (batch, tokens, heads, head_dim); cos, sin: (batch or 1, tokens, rot / 2).  Also the magnitudes |x1 cos| + |x2 sin|."""
    y = x.double().clone()
    size = torch.zeros_like(y)
    c, s = cos.double()[:, :, None, :], sin.double()[:, :, None, :]
    if transposed:
        s = -s
    i = torch.arange(rot // 2, device=x.device)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
    head = x.double()[:, :, :rotated]
    x1, x2 = head[..., a], head[..., b]
    for idx, v, m in ((a, x1 * c - x2 * s, (x1 * c).abs() + (x2 * s).abs()), (b, x2 * c + x1 * s, (x2 * c).abs() + (x1 * s).abs())):
        y[:, :, :rotated, idx] = v
        size[:, :, :rotated, idx] = m
    return y, size


def global_norm(tensors):
    return math.sqrt(math.fsum(float((t.double() ** 2).sum()) for t in tensors))


def stored(bound, value, dtype):
    """The bound for a value that is rounded to `dtype` after a computation off by `bound`; subnormals of fp32 aside."""
    return bound + (value.abs() + bound) * ROUND[dtype] + 1e-38


def within(got, want, bound):
    """Largest |got - want| / bound."""
    return float(((got.double() - want).abs() / bound).max()) if want.numel() else 0.0
