"""Attention and dropout through autograd, alone and with the operators around the projection."""
import math
import sys
from pathlib import Path

import pytest
import torch

from paper_2506_02939_b200 import build as pamm_build

pamm_build.build()
from paper_2506_02939_b200 import pamm  # noqa: E402
from paper_2506_02939_b200.autograd import Dropout, Norm, PammLinear, attention, clip_grad_norm_, dropout, rotary  # noqa: E402
from tests import attention64  # noqa: E402

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def normal(shape, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def plain(Z, kv, lengths=None, causal=True):
    """The same in elementary operations, in fp64 with autograd's own gradient."""
    batch, seq, total, d = Z.shape
    heads = total - 2 * kv
    q, k, v = Z.split((heads, kv, kv), 2)
    k, v = (t.repeat_interleave(heads // kv, 2) for t in (k, v))
    s = torch.einsum("bihd,bjhd->bhij", q, k) / math.sqrt(d)
    at = torch.arange(seq, device=Z.device)
    known = at < (torch.full((batch,), seq, device=Z.device) if lengths is None else lengths)[:, None]
    mask = known[:, None, :, None] & known[:, None, None, :]
    if causal:
        mask = mask & (at[:, None] >= at)
    p = torch.softmax(s.masked_fill(~mask, -1e30), -1) * mask
    return torch.einsum("bhij,bjhd->bihd", p, v)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("causal", [False, True])
def test_the_gradient_of_the_fused_row(causal, dtype):
    for shape, kv, lengths in (((2, 150, 8, 64), 2, [150, 77]), ((1, 200, 6, 128), 1, None), ((3, 40, 5, 20), 1, [0, 40, 3])):
        lengths = None if lengths is None else torch.tensor(lengths, device="cuda")
        Z = normal(shape, dtype, 1, 1.5).requires_grad_()
        Zd = Z.detach().double().requires_grad_()
        O, want = attention(Z, kv, lengths=lengths, causal=causal), plain(Zd, kv, lengths, causal)
        dO = normal(O.shape, dtype, 2)
        O.backward(dO)
        want.backward(dO.double())
        bound = 1e-2 if dtype == BF16 else 1e-5      # the framework's relative bounds for bf16 and fp32
        for got, ref in ((O.detach().double(), want.detach()), (Z.grad.double(), Zd.grad)):
            assert float((got - ref).norm()) <= bound * float(ref.norm())
        assert Z.grad.is_contiguous()


def test_broadcast_strided_and_packed_gradients():
    Z = normal((2, 70, 6, 64), BF16, 3)
    a, b = Z.clone().requires_grad_(), Z.clone().requires_grad_()
    attention(a, 2).sum().backward()                              # a gradient of one value for all
    attention(b, 2).backward(torch.ones((2, 70, 2, 64), dtype=BF16, device="cuda"))
    assert torch.equal(a.grad, b.grad)
    c = Z.transpose(0, 1).contiguous().transpose(0, 1).requires_grad_()
    g = normal((2, 70, 2, 64), BF16, 4)
    attention(c, 2).backward(g.transpose(2, 3).contiguous().transpose(2, 3))
    b.grad = None
    attention(b, 2).backward(g)
    assert torch.equal(c.grad, b.grad)
    # packed: as its sequences alone
    starts = torch.tensor([0, 50, 50, 140], device="cuda")
    P = Z.flatten(0, 1).clone().requires_grad_()
    O = attention(P, 2, starts=starts)
    O.backward(g.flatten(0, 1))
    for lo, hi in ((0, 50), (50, 140)):
        one = Z.flatten(0, 1)[None, lo:hi].clone().requires_grad_()
        o = attention(one, 2)
        o.backward(g.flatten(0, 1)[None, lo:hi])
        assert torch.equal(o[0], O[lo:hi]) and torch.equal(one.grad[0], P.grad[lo:hi])


def test_a_broadcast_row():
    one = normal((1, 90, 6, 64), BF16, 5).requires_grad_()
    many = one.detach().repeat(3, 1, 1, 1).requires_grad_()
    g = normal((3, 90, 2, 64), BF16, 6)
    a, b = attention(one.expand(3, -1, -1, -1), 2), attention(many, 2)
    a.backward(g)
    b.backward(g)
    assert torch.equal(a, b) and torch.equal(one.grad, many.grad.sum(0, keepdim=True))


def test_attention_of_a_row_changed_in_place_is_refused():
    Z = normal((1, 20, 3, 64), BF16, 5).requires_grad_()
    Y = Z * 1.0
    O = attention(Y, 1)
    Y.mul_(2.0)
    with pytest.raises(RuntimeError):
        O.sum().backward()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_dropout_gradients(dtype):
    x, r = normal((5, 7, 33), dtype, 6).requires_grad_(), normal((5, 7, 33), dtype, 7).requires_grad_()
    y = dropout(x, 0.3, 11, 5, residual=r)
    g = normal(y.shape, dtype, 8)
    y.backward(g)
    kept = torch.from_numpy(attention64.words(x.numel(), 11, 5) >= math.floor(0.3 * 2 ** 32)).view(x.shape).cuda()
    assert torch.equal(r.grad, g) and torch.equal(x.grad == 0, ~kept | (g == 0))
    want = g.double() / 0.7
    assert bool(((x.grad.double() - want).abs()[kept] <= (torch.finfo(dtype).eps / 2 + 2 * attention64.U) * want.abs()[kept]).all())
    # broadcast and strided gradients, and a transposed input
    a, b = x.detach().clone().requires_grad_(), x.detach().transpose(0, 2).contiguous().transpose(0, 2).requires_grad_()
    dropout(a, 0.3, 11, 5).sum().backward()
    dropout(b, 0.3, 11, 5).sum().backward()
    assert torch.equal(a.grad, b.grad) and torch.equal(a.grad != 0, kept)


def test_dropout_module():
    x, r = normal((64, 64), BF16, 9), normal((64, 64), BF16, 10)
    m = Dropout(0.5, seed=4)
    one, two = m(x), m(x)
    assert not torch.equal(one, two)
    m2 = Dropout(0.5, seed=4)
    assert torch.equal(one, m2(x)) and torch.equal(two, m2(x)) and not torch.equal(one, Dropout(0.5, seed=5)(x))
    m.eval()
    assert torch.equal(m(x), x) and torch.equal(m(x, r), x + r)
    assert torch.equal(Dropout(0.0)(x, r), x + r) and not Dropout(1.0)(x).any()


def test_a_captured_step_draws_anew():
    """Forward and backward of norm, projection, attention and dropout in one graph; the counter gives every replay a mask of its own."""
    torch.manual_seed(1)
    batch, seq, n, d = 2, 96, 128, 64
    counter = torch.zeros(1, dtype=torch.int64, device="cuda")
    norm, proj, drop = Norm(n, rms=True), PammLinear(n, 4 * d, r=1.0 / 4), Dropout(0.25, seed=2, counter=counter)
    x, g = normal((batch, seq, n), BF16, 11), normal((batch, seq, 2 * d), BF16, 12)
    params = [*norm.parameters(), *proj.parameters()]

    def step():
        proj.calls = drop.calls = 0
        y = drop(attention(proj(norm(x)).view(batch, seq, 4, d), 1).flatten(2))
        return (y, *torch.autograd.grad(y, params, g))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    seen = []
    for i in range(3):
        counter.fill_(i)
        graph.replay()
        now = [t.clone() for t in out]
        want = step()
        assert all(torch.equal(a, b) for a, b in zip(now, want))
        seen.append(now[0])
    assert not torch.equal(seen[0], seen[1]) and not torch.equal(seen[1], seen[2])


def test_a_whole_block_against_fp64():
    """norm with the residual -> projection (every row its own generator: the exact weight gradient) -> rotary -> attention -> dropout with
    the residual, and back."""
    batch, seq, n, heads, kv, d = 2, 96, 128, 4, 2, 64
    torch.manual_seed(2)
    norm, proj = Norm(n, rms=True), PammLinear(n, (heads + 2 * kv) * d, r=1.0)
    table = pamm.rotary_table(seq, *pamm.rotary_frequencies(d))
    lengths = torch.tensor([96, 61], device="cuda")
    x, s, res, g = (normal((batch, seq, m), BF16, 13 + i) for i, m in enumerate((n, n, heads * d, heads * d)))
    xa, sa = x.clone().requires_grad_(), s.clone().requires_grad_()
    y, _ = norm(xa, sa)
    z = rotary(proj(y).view(batch, seq, -1, d), table, rotated=heads + kv, inplace=True)
    out = dropout(attention(z, kv, lengths=lengths).flatten(2), 0.2, 21, residual=res)
    out.backward(g)
    kept = torch.from_numpy(attention64.words(out.numel(), 21, 0) >= math.floor(0.2 * 2 ** 32)).view(out.shape).cuda()
    xb, sb, w, W = (t.detach().double().requires_grad_() for t in (x, s, norm.weight, proj.weight))
    h = xb + sb
    q = ((h / torch.sqrt((h * h).mean(-1, keepdim=True) + norm.eps) * w) @ W).view(batch, seq, -1, d)
    c, t = table.double()[:, None, :d // 2], table.double()[:, None, d // 2:]
    q1, q2 = q[:, :, :heads + kv, :d // 2], q[:, :, :heads + kv, d // 2:]
    q = torch.cat((torch.cat((q1 * c - q2 * t, q2 * c + q1 * t), -1), q[:, :, heads + kv:]), 2)
    want = torch.where(kept, plain(q, kv, lengths).flatten(2) / 0.8, 0.0) + res.double()
    want.backward(g.double())
    # four roundings to bf16 on the way to `out` (norm, projection, rotation, attention), 2^-8 at most each and independent: 2^-8 in norm is
    # above what they leave; the gradients go through as many again
    for got, ref, bound in ((out, want, 1e-2), (xa.grad, xb.grad, 2e-2), (sa.grad, sb.grad, 2e-2), (norm.weight.grad, w.grad, 2e-2), (proj.weight.grad, W.grad, 2e-2)):
        assert float((got.detach().double() - ref.detach()).norm()) <= bound * float(ref.detach().norm())
    before = float(pamm.grad_norm([norm.weight.grad, proj.weight.grad]))
    clip_grad_norm_([norm.weight, proj.weight], 0.5 * before)
    assert abs(float(pamm.grad_norm([norm.weight.grad, proj.weight.grad])) / before - 0.5) < 1e-2


def test_the_example_runs_with_dropout():
    sys.path.insert(0, str(Path(__file__).resolve().parent.parent / "examples"))
    import train_qkv_block
    losses = train_qkv_block.train(steps=5, report=None, dropout=0.1)
    assert torch.isfinite(losses).all()
    model = train_qkv_block.Model(dropout=0.1)
    loss = model(torch.randint(0, 64, (4, 50), device="cuda")).float().square().mean()
    loss.backward()
    assert all(p.grad is not None and torch.isfinite(p.grad).all() for p in model.parameters())
