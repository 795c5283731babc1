"""The operators around the projection through autograd, and the example that runs them together."""
import sys
from pathlib import Path

import pytest
import torch
import torch.nn.functional as F

from paper_2506_02939_b200 import build as pamm_build

pamm_build.build()
from paper_2506_02939_b200 import pamm  # noqa: E402
from paper_2506_02939_b200.autograd import Norm, PammLinear, clip_grad_norm_, rotary  # noqa: E402
from tests import plain64  # noqa: E402

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def normal(shape, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("shape", [(4, 33, 96), (7, 50), (2, 3, 5, 64)])
def test_norm_module(shape, rms, dtype):
    n = shape[-1]
    layer = Norm(n, rms=rms, dtype=dtype)
    with torch.no_grad():
        layer.weight.copy_(1 + normal((n,), F32, 1, 0.2))
        if layer.bias is not None:
            layer.bias.copy_(normal((n,), F32, 2, 0.2))
    assert (layer.bias is None) == rms
    X, R = normal(shape, dtype, 3).requires_grad_(), normal(shape, dtype, 4).requires_grad_()
    y, h = layer(X, R)
    dy, dh = normal(shape, dtype, 5, 0.1), normal(shape, dtype, 6, 0.1)
    torch.autograd.backward((y, h), (dy, dh))
    flat = [t.detach().reshape(-1, n) for t in (X, R, h, dy, dh)]
    c = None if layer.bias is None else layer.bias.detach()
    want = plain64.norm_forward(flat[0], layer.weight.detach(), c, flat[1], layer.eps, rms)
    by, bh, bm, bs = plain64.norm_forward_bounds(flat[0], layer.weight.detach(), c, flat[1], layer.eps, rms)
    assert plain64.within(y.detach().reshape(-1, n), want[0], plain64.stored(by, want[0], dtype)) <= 1.0
    # the gradients are those of the row that was kept, with the statistics of the forward pass
    _, _, mean, rstd = pamm.norm_forward(flat[0], layer.weight.detach(), c, residual=flat[1], eps=layer.eps, rms=rms)
    gx, gw, gc = plain64.norm_backward(flat[3], flat[2], mean, rstd, layer.weight.detach(), flat[4], rms)
    bx, bw, bc = plain64.norm_backward_bounds(flat[3], flat[2], mean, rstd, layer.weight.detach(), flat[4], rms)
    assert plain64.within(X.grad.reshape(-1, n), gx, plain64.stored(bx, gx, dtype)) <= 1.0
    assert torch.equal(X.grad, R.grad) and X.grad.data_ptr() != R.grad.data_ptr()
    assert plain64.within(layer.weight.grad, gw, plain64.stored(bw, gw, dtype)) <= 1.0
    if layer.bias is not None:
        assert plain64.within(layer.bias.grad, gc, plain64.stored(bc, gc, dtype)) <= 1.0


def test_norm_of_strided_and_broadcast_gradients():
    layer = Norm(64, dtype=F32)
    X = normal((6, 10, 128), F32, 1)[..., ::2].requires_grad_()            # columns apart
    layer(X).sum().backward()                                             # a gradient of one value for all
    again = X.detach().contiguous().requires_grad_()
    w = layer.weight.grad.clone()
    layer.weight.grad = None
    layer(again).backward(torch.ones(again.shape, device="cuda"))
    assert torch.equal(X.grad, again.grad) and torch.equal(layer.weight.grad, w)
    # only one of the two outputs is used; a frozen weight
    layer.weight.requires_grad_(False)
    layer.weight.grad = layer.bias.grad = None
    a, b = normal((5, 64), F32, 2).requires_grad_(), normal((5, 64), F32, 3).requires_grad_()
    y, h = layer(a, b)
    h.backward(torch.ones_like(h))
    assert torch.equal(a.grad, torch.ones_like(a)) and torch.equal(b.grad, torch.ones_like(b)) and layer.weight.grad is None
    y, h = layer(a, b.detach())
    a.grad = None
    y.backward(torch.ones_like(y))
    assert a.grad.shape == a.shape and layer.bias.grad is not None and layer.weight.grad is None
    assert layer(torch.empty((0, 64), device="cuda")).shape == (0, 64)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("inplace", [False, True])
def test_rotary_of_the_fused_row(inplace, dtype):
    table = pamm.rotary_table(20, *pamm.rotary_frequencies(32))
    leaf = normal((2, 20, 6 * 48), dtype, 1).requires_grad_()
    z = (leaf * 1.0).view(2, 20, 6, 48)
    y = rotary(z, table, rotated=4, inplace=inplace)
    dy = normal((2, 20, 6, 48), dtype, 2)
    y.backward(dy)
    assert torch.equal(y.detach(), pamm.rotary(leaf.detach().view(2, 20, 6, 48), table, rotated=4))
    assert torch.equal(leaf.grad.view(2, 20, 6, 48), pamm.rotary(dy, table, rotated=4, transposed=True))
    if inplace:
        assert y.data_ptr() == z.data_ptr()


def test_clip_grad_norm_of_parameters():
    ps = [torch.nn.Parameter(normal((33, 65), BF16, 1)), torch.nn.Parameter(normal((7,), F32, 2)), torch.nn.Parameter(normal((3,), F32, 3))]
    ps[0].grad, ps[1].grad = normal((33, 65), BF16, 4), normal((7,), F32, 5)
    total = plain64.global_norm([ps[0].grad, ps[1].grad])
    before = ps[1].grad.clone()
    norm = clip_grad_norm_(ps, 0.5 * total)
    assert abs(float(norm) - total) <= 1.01 * plain64.U * total
    assert torch.allclose(ps[1].grad, before * 0.5, rtol=1e-5) and ps[2].grad is None
    assert float(clip_grad_norm_([ps[2]], 1.0)) == 0.0


def test_a_block_against_fp32_torch():
    """norm -> projection (every row its own generator: the exact weight gradient) -> rotary, against autograd in fp64."""
    batch, seq, n, heads, d = 2, 64, 128, 3, 64
    torch.manual_seed(1)
    norm, proj = Norm(n, rms=True), PammLinear(n, heads * d, r=1.0)
    table = pamm.rotary_table(seq, *pamm.rotary_frequencies(d))
    x, dz = normal((batch, seq, n), BF16, 2), normal((batch, seq, heads, d), BF16, 3, 0.1)
    xa = x.clone().requires_grad_()
    z = rotary(proj(norm(xa)).view(batch, seq, heads, d), table, rotated=2, inplace=True)
    z.backward(dz)

    xb, w, W = (t.detach().double().requires_grad_() for t in (x, norm.weight, proj.weight))
    y = xb / torch.sqrt((xb * xb).mean(-1, keepdim=True) + norm.eps) * w
    q = (y @ W).view(batch, seq, heads, d)
    c, s = table.double()[:, None, :d // 2], table.double()[:, None, d // 2:]
    q1, q2 = q[:, :, :2, :d // 2], q[:, :, :2, d // 2:]
    q = torch.cat((torch.cat((q1 * c - q2 * s, q2 * c + q1 * s), -1), q[:, :, 2:]), 2)
    q.backward(dz.double())
    for got, want in ((z, q), (xa.grad, xb.grad), (norm.weight.grad, w.grad), (proj.weight.grad, W.grad)):
        err = float(((got.double() - want).norm() / want.norm()).detach())
        assert err <= 1e-2, err            # the framework's relative bound for bf16 storage


def test_the_example_learns():
    sys.path.insert(0, str(Path(__file__).resolve().parent.parent / "examples"))
    import train_qkv_block
    losses = train_qkv_block.train(steps=150, report=None)
    assert torch.isfinite(losses).all()
    assert float(losses[-10:].mean()) < 0.5 * float(losses[:10].mean())


@pytest.mark.parametrize("shape", [(7, 64), (64,), (2, 5, 64)])
def test_outputs_of_the_norm_can_be_changed_in_place(shape):
    layer = Norm(64, dtype=F32)
    X, R, dy = normal(shape, F32, 1), normal(shape, F32, 2), normal(shape, F32, 3)
    grads = []
    for inplace in (False, True):
        x = X.clone().requires_grad_()
        layer.zero_grad()
        y = layer(x)
        assert y.shape == x.shape
        y = torch.relu_(y) if inplace else torch.relu(y)
        y.backward(dy)
        grads.append((x.grad, layer.weight.grad.clone(), layer.bias.grad.clone()))
    assert all(torch.equal(a, b) for a, b in zip(*grads))
    # with a residual: y may be changed; h is what the backward pass reads, and changing it is refused there, as by any saved output
    x, r = X.clone().requires_grad_(), R.clone().requires_grad_()
    y, h = layer(x, r)
    y.mul_(2.0)
    (y + h).backward(dy)
    x2, r2 = X.clone().requires_grad_(), R.clone().requires_grad_()
    y2, h2 = layer(x2, r2)
    (2.0 * y2 + h2).backward(dy)
    assert torch.equal(x.grad, x2.grad) and torch.equal(r.grad, r2.grad)
    y, h = layer(X.clone().requires_grad_(), R)
    h.add_(1.0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        (y + h).backward(dy)
    with torch.no_grad():
        y, h = layer(X, R)
        assert torch.equal(h.add_(1.0), X + R + 1.0)


def test_clip_grad_norm_of_one_parameter():
    p = torch.nn.Parameter(normal((33, 65), F32, 1))
    p.grad = normal((33, 65), F32, 2)
    before, total = p.grad.clone(), plain64.global_norm([p.grad])
    norm = clip_grad_norm_(p, 0.5 * total)
    assert abs(float(norm) - total) <= 1.01 * plain64.U * total
    assert torch.allclose(p.grad, before * 0.5, rtol=1e-5)
    p.grad = None
    assert float(clip_grad_norm_(p, 1.0)) == 0.0


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_the_gradient_of_rows_that_share_one_value_reaches_the_projection(dtype):
    """The gradient of a sum over the rows is one row, repeated at distance zero."""
    grads = []
    for repeated in (True, False):
        layer = PammLinear(64, 96, r=0.5, dtype=dtype)
        with torch.no_grad():
            layer.weight.copy_(normal((64, 96), F32, 1, 0.1))
        x = normal((40, 64), dtype, 2).requires_grad_()
        row = normal((96,), dtype, 3)
        layer(x).backward(row.expand(40, 96) if repeated else row.repeat(40, 1))
        grads.append((x.grad, layer.weight.grad))
    assert all(torch.equal(a, b) for a, b in zip(*grads))


def test_the_gradient_of_a_residual_has_its_own_shape():
    layer = Norm(64, dtype=F32)
    X, R = normal((2, 3, 64), F32, 1).requires_grad_(), normal((6, 64), F32, 2).requires_grad_()       # rows of another shape
    dy, dh = normal((2, 3, 64), F32, 3), normal((2, 3, 64), F32, 4)
    torch.autograd.backward(layer(X, R), (dy, dh))
    assert R.grad.shape == R.shape and torch.equal(R.grad, X.grad.view(6, 64)) and R.grad.data_ptr() != X.grad.data_ptr()
