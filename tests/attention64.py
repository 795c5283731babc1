"""Attention and its gradients in 64 bits from their definitions, with bounds on what fp32 sums and the stated roundings may be off,
and the dropout's mask word by word."""
import math

import numpy as np
import torch

U = 2.0 ** -24                       # half a step of fp32, relative


def pieces(shape, lengths=None, starts=None):
    """(index of the sequence's valid tokens) of every sequence: (b, slice) or (slice,)."""
    if starts is not None:
        return [(slice(a, b),) for a, b in zip(starts[:-1], starts[1:])]
    if len(shape) == 3:
        return [(slice(0, shape[0] if lengths is None else lengths[0]),)]
    return [(b, slice(0, shape[1] if lengths is None else lengths[b])) for b in range(shape[0])]


def _scores(q, k, causal, scale):
    n = q.shape[0]
    s = torch.einsum("id,jd->ij", q, k) * scale
    size = torch.einsum("id,jd->ij", q.abs(), k.abs()) * scale
    mask = torch.ones((n, n), dtype=torch.bool, device=q.device)
    return s, size, mask.tril() if causal else mask


def _score_error(s, size, d):
    """How far exp(s - m) may be off, relatively: the fp32 sum of d products, its scaling by a constant rounded from log2(e) scale, the
    difference from m, and the exponential itself (2 units)."""
    return (d + 4) * U * size + 4 * U * s.abs() + 8 * U


def forward(Q, K, V, causal, lengths=None, starts=None, scale=None, rounded=False):
    """O, lse, and bounds on their errors before O is rounded to its type; ``rounded``: probabilities become bf16 operands."""
    Qd, Kd, Vd = (t.detach().cpu().double() for t in (Q, K, V))
    heads, kv, d = Q.shape[-2], K.shape[-2], Q.shape[-1]
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    O, E = torch.zeros(Q.shape, dtype=torch.float64), torch.zeros(Q.shape, dtype=torch.float64)
    shape = (heads, Q.shape[0]) if Q.dim() == 3 else (Q.shape[0], heads, Q.shape[1])
    L, F = torch.full(shape, -math.inf, dtype=torch.float64), torch.zeros(shape, dtype=torch.float64)
    for at in pieces(Q.shape, lengths, starts):
        for h in range(heads):
            q, k, v = Qd[at][:, h], Kd[at][:, h // (heads // kv)], Vd[at][:, h // (heads // kv)]
            n = q.shape[0]
            if n == 0:
                continue
            s, size, mask = _scores(q, k, causal, scale)
            s = s.masked_fill(~mask, -math.inf)
            m = s.amax(1, keepdim=True)
            p = (s - m).exp()
            total = p.sum(1, keepdim=True)
            err = _score_error(s.masked_fill(~mask, 0.0) - m, size, d).masked_fill(~mask, 0.0).amax(1, keepdim=True)
            sums = (n + 16) * U
            O[at][:, h] = p @ v / total
            E[at][:, h] = (2 * (err + sums) + (2.0 ** -8 if rounded else 0.0)) * (p @ v.abs() / total)
            row = (*at[:-1], h, at[-1]) if Q.dim() == 4 else (h, at[-1])
            L[row] = (m + total.log()).squeeze(1)
            F[row] = (err + sums + 4 * U * (m.abs() + 1)).squeeze(1)
    return O, L, E, F


def backward(dO, Q, K, V, O, lse, causal, lengths=None, starts=None, scale=None, rounded=False):
    """dQ, dK, dV from the given O and lse, and bounds on their errors before they are rounded."""
    dOd, Qd, Kd, Vd, Od, L = (t.detach().cpu().double() for t in (dO, Q, K, V, O, lse))
    heads, kv, d = Q.shape[-2], K.shape[-2], Q.shape[-1]
    group, half = heads // kv, 2.0 ** -8 if rounded else 0.0
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    out = [torch.zeros(t.shape, dtype=torch.float64) for t in (Q, K, V)]
    err = [torch.zeros(t.shape, dtype=torch.float64) for t in (Q, K, V)]
    for at in pieces(Q.shape, lengths, starts):
        for h in range(heads):
            g = h // group
            q, k, v, o, do = Qd[at][:, h], Kd[at][:, g], Vd[at][:, g], Od[at][:, h], dOd[at][:, h]
            n = q.shape[0]
            if n == 0:
                continue
            row = (*at[:-1], h, at[-1]) if Q.dim() == 4 else (h, at[-1])
            l = L[row].unsqueeze(1)
            s, size, mask = _scores(q, k, causal, scale)
            p = (s - l).exp().masked_fill(~mask, 0.0)
            r = _score_error((s - l).masked_fill(~mask, 0.0), size, d) + 4 * U * l.abs()
            dp, delta = do @ v.T, (do * o).sum(1, keepdim=True)
            e_dp = (d + 4) * U * (do.abs() @ v.abs().T + (do * o).abs().sum(1, keepdim=True))
            ds = p * (dp - delta)
            e_ds = p * (2 * r * (dp - delta).abs() + 2 * e_dp) + half * ds.abs()
            sums = (group * n + 16) * U
            out[0][at][:, h] = scale * ds @ k
            err[0][at][:, h] = scale * (e_ds + sums * ds.abs()) @ k.abs()
            out[1][at][:, g] += scale * ds.T @ q
            err[1][at][:, g] += scale * (e_ds + sums * ds.abs()).T @ q.abs()
            out[2][at][:, g] += p.T @ do
            err[2][at][:, g] += (p * (2 * r + sums + half)).T @ do.abs()
    return out, err


def share(got, want, err):
    """The largest error as a share of its bound, where the result is also rounded once to its type; what is not finite has to agree."""
    got_d = got.detach().cpu().double()
    fine = torch.isfinite(want)
    assert torch.equal(fine, torch.isfinite(got_d)) and torch.equal(got_d[~fine], want[~fine])
    bound = err + torch.finfo(got.dtype).eps / 2 * (want.abs() + err) + 1e-37
    return float(((got_d - want).abs()[fine] / bound[fine]).max()) if fine.any() else 0.0


def words(count, seed, offset):
    """The first ``count`` words of the generator: Philox 4x32 with ten rounds, in Python's own integers."""
    out = []
    for block in range((count + 3) // 4):
        c = [block & 0xFFFFFFFF, block >> 32, offset & 0xFFFFFFFF, offset >> 32 & 0xFFFFFFFF]
        k = [seed & 0xFFFFFFFF, seed >> 32]
        for _ in range(10):
            a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
            c = [b >> 32 ^ c[1] ^ k[0], b & 0xFFFFFFFF, a >> 32 ^ c[3] ^ k[1], a & 0xFFFFFFFF]
            k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
        out += c
    return np.array(out[:count], dtype=np.uint64)
