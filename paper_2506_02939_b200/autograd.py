"""A linear layer whose backward pass keeps the compressed input only (Algorithms 2 and 3).

Forward: ``Z = X W`` and ``Compress(flatten(X))``.  For bf16 layers both come out of ONE kernel
of the CUDA library (``pamm_linear_forward``: the scores are extra output columns of the
product, so X is not read a second time); other dtypes take torch's GEMM for Z and the
library's stand-alone compression.  The layer saves (C, f, alpha, W) and lets go of X.
Backward: the weight gradient is ``ApproxMM(C, alpha, f, dZ) = C^T B~`` through the library,
the input gradient ``dX = dZ W^T`` is exact (for bf16 layers the library's tensor-core product
``pamm_linear_backward_input``, else torch).  Meant for the fused Q|K|V projection: ``W`` is n x m
with m = |Q| + |K| + |V|, as in the paper's notation.

Around it: ``Norm`` (layer norm or its root-mean-square form, with the residual addition), whose
output is the projection's input; ``rotary`` on the heads of the projection's output; ``attention`` over
them; ``dropout`` with the residual addition; and ``clip_grad_norm_`` for the end of a training step.

A step that is captured into a CUDA graph starts from parameters whose earlier autograd graphs (a loss that is still held)
are gone: PyTorch accumulates a gradient on the stream of the first graph that it belonged to, which a capture cannot join.
"""
from __future__ import annotations

import math

import torch

from . import pamm


def _rows(t: torch.Tensor, cols: int) -> torch.Tensor:
    """(…, cols) -> (rows, cols) view the library accepts (16-byte aligned rows that do not overlap)."""
    t2 = t.reshape(-1, cols)
    if t2.stride(1) != 1 or t2.stride(0) < cols or (t2.stride(0) * t2.element_size()) % 16 or t2.data_ptr() % 16:
        padded = pamm.alloc_matrix(t2.shape[0], cols, t2.dtype, t2.device)
        padded.copy_(t2)
        t2 = padded
    return t2


class PammLinearFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, X, W, k, seed):
        n, m = W.shape
        X2 = _rows(X.detach(), n)
        b = X2.shape[0]
        f_dtype = torch.uint8 if k <= 256 else torch.int16 if k <= 65536 else torch.int32
        # the pass also leaves its per-block counts of f (a few KiB): the backward's counting sort starts from them
        sp = pamm.alloc_workspace(pamm.WS_COMPRESS, b, n, m, int(k), pamm.BF16 if X2.dtype == torch.bfloat16 else pamm.F32,
                                  X2.device)
        Wd = W.detach()
        one_kernel = (X2.dtype == torch.bfloat16 and Wd.dtype == torch.bfloat16 and 16 <= k <= 4096 and n >= 8 and m >= 8
                      and Wd.is_contiguous() and (m * 2) % 16 == 0 and Wd.data_ptr() % 16 == 0)
        if one_kernel:
            # made in its final shape, not as a view of a matrix: what follows may then work on it in place
            Z = torch.empty((*X.shape[:-1], m), dtype=X2.dtype, device=X2.device)
            _, _, C, _, f, alpha = pamm.linear_forward(X2, Wd, int(k), int(seed), Z=Z.view(-1, m), sort_products=sp, f_dtype=f_dtype)
        else:
            Z = X @ W
            _, C, _, f, alpha = pamm.compress_fused(X2, int(k), int(seed), sort_products=sp, f_dtype=f_dtype)
        ctx.save_for_backward(C, f, alpha, sp, W)      # k n + 2 b scalars instead of b n
        return Z

    @staticmethod
    def backward(ctx, dZ):
        C, f, alpha, sp, W = ctx.saved_tensors
        n, m = W.shape
        dX = None
        if ctx.needs_input_grad[0]:
            Wd = W.detach()
            dZr = _rows(dZ, m)
            own = (dZr.dtype == torch.bfloat16 and Wd.dtype == torch.bfloat16 and n >= 8 and m >= 8 and Wd.is_contiguous()
                   and dZr.stride(1) == 1 and (m * 2) % 16 == 0 and (dZr.stride(0) * 2) % 16 == 0
                   and Wd.data_ptr() % 16 == 0 and dZr.data_ptr() % 16 == 0)
            if own:      # Algorithm 3's other product, through the library's tensor-core kernel
                dX = pamm.linear_backward_input(dZr, Wd).reshape(*dZ.shape[:-1], n)
            else:
                dX = dZ @ W.t()
        dW = None
        if ctx.needs_input_grad[1]:
            dZ2 = _rows(dZ.to(C.dtype), m)
            direct = W.dtype in (torch.float32, torch.bfloat16)      # the product kernel writes these itself
            dW = pamm.contract_weight_grad(C, f, alpha, dZ2, dw_dtype=W.dtype if direct else torch.float32, sort_products=sp)
            if not direct:
                dW = dW.to(W.dtype)
        return dX, dW, None, None


class PammLinear(torch.nn.Module):
    """``Z = X W`` with PAMM in the backward pass; ``r`` is the compression ratio k / b (Section 4.1)."""

    def __init__(self, n: int, m: int, r: float = 1.0 / 512, dtype=torch.bfloat16, device="cuda", seed: int = 0):
        super().__init__()
        self.weight = torch.nn.Parameter(torch.empty((n, m), dtype=dtype, device=device))
        torch.nn.init.normal_(self.weight, std=1.0 / math.sqrt(n))
        self.r = float(r)
        self.seed = int(seed)
        self.calls = 0

    def forward(self, X):
        b = X.numel() // X.shape[-1]
        k = max(1, min(b, math.ceil(self.r * b)))
        self.calls += 1                                   # fresh generators every step (Appendix "LLaMA-1B Runtime Breakdown")
        return PammLinearFunction.apply(X, self.weight, k, self.seed + self.calls)


def _matrix(t: torch.Tensor, n: int) -> torch.Tensor:
    """(…, n) -> (rows, n) with contiguous rows that do not overlap; copied only where it has to be."""
    t2 = t.reshape(-1, n)
    rows = t2.shape[0]
    if (n > 1 and t2.stride(1) != 1) or (rows > 1 and t2.stride(0) < n):
        t2 = t2.contiguous()
    return t2


class NormFunction(torch.autograd.Function):
    """``pamm.norm_forward`` / ``norm_backward`` on the last dimension.  With a residual the outputs are (y, h) and the gradient
    that reaches h joins dX in the same pass.  Saved: the normalised row (h, or X), mean, rstd and the weight."""

    @staticmethod
    def forward(ctx, X, weight, bias, residual, eps, rms):
        n = X.shape[-1]
        X2 = _matrix(X.detach(), n)
        R2 = None if residual is None else _matrix(residual.detach().to(X.dtype), n)
        w, c = (None if p is None else p.detach() for p in (weight, bias))
        # made in their final shape, not as views of matrices: what follows may then work on y in place
        Y = torch.empty(X.shape, dtype=X.dtype, device=X.device)
        H = None if residual is None else torch.empty(X.shape, dtype=X.dtype, device=X.device)
        _, _, mean, rstd = pamm.norm_forward(X2, w, c, residual=R2, eps=eps, rms=rms, Y=Y.view(-1, n), H=None if H is None else H.view(-1, n))
        ctx.save_for_backward(X2 if H is None else H, mean, rstd, weight)
        ctx.shape, ctx.residual_shape = X.shape, None if residual is None else residual.shape
        ctx.vector_type = weight.dtype if weight is not None else bias.dtype if bias is not None else X.dtype
        ctx.set_materialize_grads(False)
        return Y if residual is None else (Y, H)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dY, dH=None):
        H, mean, rstd, weight = ctx.saved_tensors
        n = ctx.shape[-1]
        if dY is None and dH is None:
            return (None,) * 6
        H = H.reshape(-1, n)
        if dY is None:
            dY = torch.zeros(ctx.shape, dtype=H.dtype, device=H.device)
        need_w, need_c = ctx.needs_input_grad[1], ctx.needs_input_grad[2]
        dX, dw, dc = pamm.norm_backward(_matrix(dY.to(H.dtype), n), H, mean, rstd, None if weight is None else weight.detach(),
                                        bias=need_c, dH=None if dH is None else _matrix(dH.to(H.dtype), n),
                                        need_dw=need_w or need_c, dw_dtype=ctx.vector_type)
        dX = dX.reshape(ctx.shape)
        dR = None
        if ctx.needs_input_grad[3]:         # one tensor for both inputs, which autograd then copies; a view of it would be shared
            dR = dX if ctx.residual_shape == ctx.shape else dX.reshape(ctx.residual_shape).clone()
        return dX if ctx.needs_input_grad[0] else None, dw if need_w else None, dc if need_c else None, dR, None, None


class Norm(torch.nn.Module):
    """Layer norm over the last dimension, or (``rms``) its root-mean-square form without a bias.  ``norm(X)`` gives y;
    ``norm(X, residual)`` gives (y, h = X + residual), the step from one block of a network to the next."""

    def __init__(self, n: int, eps: float = 1e-5, rms: bool = False, bias: bool | None = None, dtype=torch.bfloat16, device="cuda"):
        super().__init__()
        self.weight = torch.nn.Parameter(torch.ones(n, dtype=dtype, device=device))
        with_bias = not rms if bias is None else bias
        self.bias = torch.nn.Parameter(torch.zeros(n, dtype=dtype, device=device)) if with_bias else None
        self.eps, self.rms = float(eps), bool(rms)

    def forward(self, X, residual=None):
        return NormFunction.apply(X, self.weight, self.bias, residual, self.eps, self.rms)


class RotaryFunction(torch.autograd.Function):
    """``pamm.rotary`` and its transposed turn.  Nothing but the table and the positions is kept."""

    @staticmethod
    def forward(ctx, X, table, positions, rotated, interleaved, first, inplace):
        ctx.save_for_backward(table, positions)
        ctx.how = dict(rotated=rotated, interleaved=interleaved, first=first)
        if inplace:
            ctx.mark_dirty(X)
        Xd = X.detach()
        out = pamm.rotary(Xd, table, positions, out=Xd if inplace else None, **ctx.how)
        return X if inplace else out

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dY):
        table, positions = ctx.saved_tensors
        if dY.shape[-1] > 1 and dY.stride(-1) != 1:
            dY = dY.contiguous()
        return pamm.rotary(dY, table, positions, transposed=True, **ctx.how), None, None, None, None, None, None


def rotary(X, table, positions=None, rotated=None, interleaved: bool = False, first: int = 0, inplace: bool = False):
    """Rotary positions on the first ``rotated`` heads of X, (tokens, heads, head_dim) or (batch, tokens, heads, head_dim), as
    ``pamm.rotary``; the other heads (V of the fused row) pass through.  ``inplace`` turns X itself, which must not be a leaf
    or needed by the backward pass of what made it (the projection's output is neither)."""
    return RotaryFunction.apply(X, table, positions, rotated, interleaved, first, inplace)


class AttentionFunction(torch.autograd.Function):
    """``pamm.attention_forward`` / ``attention_backward`` on the fused row.  Saved: the row itself, O, the rows' log-sums, and the
    lengths or starts; the gradient is one row [dQ|dK|dV], as the projection takes it."""

    @staticmethod
    def forward(ctx, Z, lengths, starts, kv_heads, causal, scale):
        Zd = Z.detach()
        if (Zd.shape[-1] > 1 and Zd.stride(-1) != 1) or 0 in Zd.stride():      # a broadcast row has no tiles to copy
            Zd = Zd.contiguous()
        heads = Zd.shape[-2] - 2 * kv_heads
        ctx.parts = (heads, kv_heads, kv_heads)
        ctx.how = dict(causal=causal, scale=scale)
        O, lse = pamm.attention_forward(*Zd.split(ctx.parts, -2), lengths=lengths, starts=starts, **ctx.how)
        ctx.save_for_backward(Z if Zd.data_ptr() == Z.data_ptr() else Zd, O, lse, lengths, starts)
        return O

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dO):
        Z, O, lse, lengths, starts = ctx.saved_tensors
        Zd = Z.detach()
        dO = dO.to(Zd.dtype)
        if (dO.shape[-1] > 1 and dO.stride(-1) != 1) or 0 in dO.stride():      # nor has a broadcast gradient
            dO = dO.contiguous()
        dZ = torch.empty(Zd.shape, dtype=Zd.dtype, device=Zd.device)
        dQ, dK, dV = dZ.split(ctx.parts, -2)
        pamm.attention_backward(dO, *Zd.split(ctx.parts, -2), O, lse, lengths=lengths, starts=starts, dQ=dQ, dK=dK, dV=dV, **ctx.how)
        return dZ, None, None, None, None, None


def attention(Z, kv_heads, lengths=None, starts=None, causal: bool = True, scale: float | None = None):
    """Attention over the fused row: Z is (batch, tokens, heads + 2 kv_heads, head_dim), or (tokens, ...) with packed sequences between
    ``starts``; its last 2 ``kv_heads`` heads are K and V, shared evenly by the others.  Returns the heads' outputs in Q's shape; tokens
    from ``lengths`` on have zero outputs and gradients.  See ``pamm.attention_forward``."""
    if not 0 < 2 * kv_heads < Z.shape[-2]:
        raise ValueError(f"{kv_heads} heads of K and as many of V leave none for Q in a row of {Z.shape[-2]}")
    return AttentionFunction.apply(Z, lengths, starts, int(kv_heads), bool(causal), scale)


class DropoutFunction(torch.autograd.Function):
    """``pamm.dropout``.  No mask is kept: the backward pass makes it again from the seed, the offset and the counter."""

    @staticmethod
    def forward(ctx, X, residual, counter, p, seed, offset):
        ctx.save_for_backward(counter)
        ctx.how = (p, seed, offset)
        R = None if residual is None else residual.detach().to(X.dtype).contiguous()
        ctx.residual = None if residual is None else residual.dtype
        return pamm.dropout(X.detach().contiguous(), p, seed, offset, counter=counter, residual=R)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dY):
        counter, = ctx.saved_tensors
        p, seed, offset = ctx.how
        dX = pamm.dropout(dY.contiguous(), p, seed, offset, counter=counter) if ctx.needs_input_grad[0] else None
        return dX, dY.to(ctx.residual) if ctx.needs_input_grad[1] else None, None, None, None, None


def _same_shape(X, residual):
    if residual is not None and residual.shape != X.shape:
        raise ValueError("the residual has X's shape")


def dropout(X, p: float, seed: int, offset: int = 0, counter=None, residual=None):
    """``residual`` + X / (1 - p) where the generator keeps it, as ``pamm.dropout``; ``residual`` has X's shape and, as ``Norm``'s,
    is taken in X's type.  A ``counter`` must not change between the forward and the backward pass."""
    _same_shape(X, residual)
    return DropoutFunction.apply(X, residual, counter, float(p), int(seed), int(offset))


class Dropout(torch.nn.Module):
    """Dropout with an optional residual addition, ``dropout(X)`` or ``dropout(X, residual)``: a fresh mask every call.  In evaluation mode
    X (+ residual) passes.

    Every call draws its key from torch's host generator: modules are independent of each other, ``torch.manual_seed`` repeats them, and
    what restores that generator's state to run a forward pass again (activation checkpointing) gets the same mask again.
    With a ``seed`` the masks follow from it and from ``calls``, the number of the call, alone; the state dict has that number.  Two modules with one seed have the same
    masks then: give each its own.  A call from a backward pass, where activation checkpointing runs a forward pass again, is refused,
    because its number would not be the first call's.

    ``counter``: a one-element int64 tensor on the device that numbers the calls in a captured graph (counted up by the program
    between replays); without it a graph replays the mask that it was captured with."""

    def __init__(self, p: float = 0.1, seed: int | None = None, counter=None):
        super().__init__()
        if not 0.0 <= p <= 1.0:
            raise ValueError(f"p is a probability, got {p}")
        self.p, self.seed, self.counter, self.calls = float(p), None if seed is None else int(seed), counter, 0

    def forward(self, X, residual=None):
        if not self.training or self.p == 0.0:
            _same_shape(X, residual)
            return X if residual is None else X + residual.to(X.dtype)
        if self.seed is None:
            key, offset = int(torch.empty((), dtype=torch.int64, device="cpu").random_()), 0
        elif torch._C._current_graph_task_id() != -1:
            raise RuntimeError("a Dropout with a seed numbers its calls and would draw another mask for the same activations in a backward pass "
                               "(activation checkpointing): give it no seed, or call dropout() with an offset")
        else:
            self.calls += 1
            key, offset = self.seed, self.calls << 32
        return dropout(X, self.p, key, offset, self.counter, residual)

    def get_extra_state(self):
        return torch.tensor(self.calls, dtype=torch.int64, device="cpu")

    def set_extra_state(self, state):
        self.calls = int(state)

    def _load_from_state_dict(self, state_dict, prefix, *args):
        state_dict.setdefault(prefix + "_extra_state", self.get_extra_state())       # one from before there was a number
        super()._load_from_state_dict(state_dict, prefix, *args)


def clip_grad_norm_(parameters, max_norm: float):
    """Clip the gradients of ``parameters`` (or of one) in place to a global norm of ``max_norm``; returns the norm before
    (fp32 on the device), without waiting for it.  Parameters without a gradient are left out."""
    if isinstance(parameters, torch.Tensor):
        parameters = [parameters]
    grads = [p.grad for p in parameters if p.grad is not None]
    return pamm.clip_grad_norm(grads, max_norm)
