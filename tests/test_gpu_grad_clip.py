"""The gradients' global norm and their clipping against 64-bit statements."""
import math

import pytest
import torch

from paper_2506_02939_b200 import build as pamm_build

pamm_build.build()
from paper_2506_02939_b200 import pamm  # noqa: E402
from tests import plain64  # noqa: E402

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def normal(shape, dtype, seed, scale=1e-2):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def lists():
    yield "one value", [normal((1,), F32, 1)]
    yield "a scalar", [normal((), BF16, 1)]
    yield "one row", [normal((70001,), BF16, 2)]
    yield "mixed", [normal((300, 257), BF16, 3), normal((513,), F32, 4), normal((2, 3, 5), BF16, 5), normal((8192,), F32, 6),
                    normal((3, 8191), F32, 7), normal((8193,), BF16, 8)]
    flat = normal((200_000,), BF16, 9)
    views, at = [], 0
    for i in range(60):
        size = 1 + (i * 977) % 5003
        views.append(flat[at:at + size])
        at += size
    yield "a bucket of odd sizes", views
    flat = normal((100_000,), F32, 10)
    yield "fp32 at every alignment", [flat[k * 1000 + k:k * 1000 + k + 900] for k in range(9)]
    yield "rows apart", [normal((70, 96), BF16, 11)[:, :91], normal((5, 9000), F32, 12)[:, 3:8700], normal((33, 8), F32, 13)[:, :1],
                         normal((1, 50), F32, 14)[:, 7:]]
    yield "columns apart", [normal((96, 70), F32, 15)[:91].t(), normal((40, 30), BF16, 16).t()]
    yield "empty ones among them", [normal((0,), F32, 17), normal((7,), F32, 18), normal((0, 5), BF16, 19)]
    yield "more than a launch holds", [normal((1 + (i * 37) % 300,), (F32, BF16)[i % 2], 100 + i) for i in range(1000)]
    yield "nothing", []


LISTS = ["one value", "a scalar", "one row", "mixed", "a bucket of odd sizes", "fp32 at every alignment", "rows apart", "columns apart",
         "empty ones among them", "more than a launch holds", "nothing"]


@pytest.mark.parametrize("which", LISTS)
def test_norm_and_clipping(which):
    grads = dict(lists())[which]
    total = plain64.global_norm(grads)
    norm = pamm.grad_norm(grads)
    assert norm.shape == () and norm.dtype == F32
    assert abs(float(norm) - total) <= 1.01 * plain64.U * total
    assert torch.equal(norm, pamm.grad_norm(grads))
    for limit in (0.3 * total, 0.0, 2 * total + 1, math.inf):
        factor = min(1.0, limit / (total + 1e-6))
        for out_dtype in (None, F32, BF16):
            src = [torch.empty_strided(g.shape, g.stride(), dtype=g.dtype, device="cuda").copy_(g) for g in grads]
            out = None if out_dtype is None else [torch.empty_strided(g.shape, g.stride(), dtype=out_dtype, device="cuda") for g in grads]
            got = pamm.clip_grad_norm(src, limit, out=out)
            assert torch.equal(got, norm)
            for g, s, t in zip(grads, src, src if out is None else out):
                want = g.double() * factor
                # the factor is rounded to fp32 and the product once more, then stored
                assert plain64.within(t, want, plain64.stored(2.1 * plain64.U * want.abs(), want, t.dtype)) <= 1.0
                if out is not None:
                    assert torch.equal(s, g)
                elif factor == 1.0:
                    assert torch.equal(t, g)


def test_views_of_buckets_leave_their_neighbours_alone():
    for dtype in (F32, BF16):
        flat, out = normal((50_000,), dtype, 1), torch.full((50_000,), 7.0, dtype=dtype, device="cuda")
        spans = [(5, 1001), (1003, 1004), (2001, 20_000), (20_003, 49_993)]
        grads, outs = [flat[a:b] for a, b in spans], [out[a:b] for a, b in spans]
        shifted = torch.full((50_003,), 7.0, dtype=dtype, device="cuda")
        outs2 = [shifted[a + 3:b + 3] for a, b in spans]
        total = plain64.global_norm(grads)
        pamm.clip_grad_norm(grads, 0.5 * total, out=outs)
        pamm.clip_grad_norm(grads, 0.5 * total, out=outs2)
        inside = torch.zeros(50_000, dtype=torch.bool, device="cuda")
        for a, b in spans:
            inside[a:b] = True
        assert (out[~inside] == 7.0).all() and torch.equal(shifted[3:], out) and (shifted[:3] == 7.0).all()
        kept = flat.clone()
        pamm.clip_grad_norm(grads, 0.5 * total)
        assert torch.equal(flat[~inside], kept[~inside]) and torch.equal(flat[inside], out[inside])


def test_outputs_laid_out_differently():
    g = [normal((40, 61), F32, 1), normal((40, 96), BF16, 2)[:, :61], normal((61, 40), F32, 3).t()]
    total = plain64.global_norm(g)
    out = [torch.full((40, 64), 7.0, device="cuda")[:, :61], torch.empty((40, 61), device="cuda"), torch.empty((61, 44), device="cuda")[:, :40].t()]
    pamm.clip_grad_norm(g, 0.5 * total, out=out)
    for s, t in zip(g, out):
        want = s.double() * (0.5 * total / (total + 1e-6))
        assert plain64.within(t, want, plain64.stored(2.1 * plain64.U * want.abs(), want, F32)) <= 1.0
    with pytest.raises(ValueError):
        pamm.clip_grad_norm([normal((40, 61), F32, 1)], 1.0, out=[normal((61, 40), F32, 1).t()])


def test_range_of_the_squares():
    big = torch.full((1000,), 1e30, device="cuda")
    assert abs(float(pamm.grad_norm([big])) / (1e30 * math.sqrt(1000)) - 1) < 1e-6
    small = torch.full((1000,), 1e-30, device="cuda")
    assert abs(float(pamm.grad_norm([small])) / (1e-30 * math.sqrt(1000)) - 1) < 1e-6
    assert float(pamm.clip_grad_norm([small], 1.0)) > 0 and torch.equal(small, torch.full((1000,), 1e-30, device="cuda"))
    huge = torch.full((1000,), 3e38, device="cuda")
    assert math.isinf(float(pamm.grad_norm([huge])))         # the norm itself leaves fp32's range
    out = torch.empty_like(huge)
    pamm.clip_grad_norm([huge], 1.0, out=[out])               # the factor does not
    assert torch.allclose(out, torch.full_like(out, 1 / math.sqrt(1000)), rtol=1e-6)


def test_infinities_and_nan():
    for value, factor in ((float("inf"), 0.0), (float("nan"), float("nan"))):
        g = torch.tensor([1.0, value, -2.0], device="cuda")
        norm = pamm.clip_grad_norm([g], 1.0)
        assert not math.isfinite(float(norm)) and math.isnan(float(norm)) == math.isnan(value)
        want = torch.tensor([1.0, value, -2.0]) * factor
        assert torch.equal(torch.nan_to_num(g.cpu(), 9.0), torch.nan_to_num(want, 9.0))
        g = torch.tensor([1.0, value, -2.0], device="cuda")
        pamm.clip_grad_norm([g], math.inf)                    # no limit: nothing is scaled
        assert float(g[0]) == 1.0 and float(g[2]) == -2.0


def test_the_frameworks_own_gradients():
    C, Bt = normal((16, 40), BF16, 1, 1.0), pamm.alloc_matrix(16, 70, F32)
    Bt.copy_(normal((16, 70), F32, 2, 1.0))
    dW = pamm.weight_grad(C, Bt, dw_dtype=BF16)
    assert not dW.is_contiguous()
    total = plain64.global_norm([dW])
    norm = pamm.clip_grad_norm([dW], 0.5 * total)
    assert abs(float(norm) - total) <= 1.01 * plain64.U * total
    assert abs(plain64.global_norm([dW]) - 0.5 * total) <= 2.0 ** -8 * total


def test_more_than_2_to_the_31_elements():
    g = torch.full((2 ** 31 + 11,), 0.5, dtype=BF16, device="cuda")
    want = 0.5 * math.sqrt(2 ** 31 + 11)
    assert abs(float(pamm.clip_grad_norm([g], 0.5 * want)) - want) <= 1.01 * plain64.U * want
    assert float(g[-1]) == 0.25 and float(g[2 ** 31]) == 0.25 and float(g[0]) == 0.25 and float(g.min()) == 0.25


def test_on_another_stream_in_a_graph_and_prepared():
    g = [normal((500, 300), BF16, 1), normal((300,), F32, 2)]
    norm = pamm.grad_norm(g)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = pamm.grad_norm(g, stream=side)
    side.synchronize()
    assert torch.equal(got, norm)
    out = [torch.zeros_like(t) for t in g]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        n2 = pamm.clip_grad_norm(g, 0.1, out=out)
    for t in out:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    want = [torch.zeros_like(t) for t in g]
    assert torch.equal(pamm.clip_grad_norm(g, 0.1, out=want), n2) and all(torch.equal(a, b) for a, b in zip(out, want))
    for t in out:
        t.zero_()
    pamm.prepared(pamm.clip_grad_norm, g, 0.1, out=out)()
    assert all(torch.equal(a, b) for a, b in zip(out, want))


def bucket(total, dtype, seed, step=977):
    """Views of odd sizes of one piece of memory."""
    flat, views, at, i = normal((total,), dtype, seed), [], 0, 0
    while at < total:
        size = min(total - at, total // 40 + 1 + (i * step) % 5003)
        views.append(flat[at:at + size])
        at, i = at + size, i + 1
    return views


def large_lists():
    """Total sizes on both sides of the switches of the scaling (2^21 elements into others, 14 2^20 in place) and of the sum's chunks."""
    def apart(k):          # rows narrower and wider than a chunk, at a distance
        return [normal((20_000 * k, 96), BF16, 1)[:, :91], normal((5, 70_008 * k), F32, 2)[:, 3:70_004 * k], normal((3000, 1), F32, 3)]
    yield "2 M", bucket(2 ** 21 - 100, F32, 14)
    yield "2 M and some", bucket(2 ** 21 + 100, BF16, 15)
    yield "4 M", bucket(2 ** 22 - 100, BF16, 4)
    yield "4 M and some", bucket(2 ** 22 + 100, F32, 5)
    yield "rows apart", apart(1) + bucket(2_000_003, F32, 6) + bucket(1_000_001, BF16, 7)
    yield "14 M", bucket(7 * 2 ** 20, BF16, 8) + bucket(7 * 2 ** 20 - 100, F32, 9)
    yield "14 M and some", bucket(7 * 2 ** 20, BF16, 10) + bucket(7 * 2 ** 20 + 100, F32, 11)
    yield "80 M", apart(4) + bucket(50_000_001, BF16, 12) + bucket(22_000_003, F32, 13)
    yield "600 tensors", [normal((19_997 + 7 * i,), (BF16, F32)[i % 3 == 0], 100 + i) for i in range(600)]
    yield "600 larger ones", [normal((59_999 + 7 * i,), (F32, BF16)[i % 3 == 0], 100 + i) for i in range(600)]


LARGE = ["2 M", "2 M and some", "4 M", "4 M and some", "rows apart", "14 M", "14 M and some", "80 M", "600 tensors", "600 larger ones"]


def check(grads, total, norm, limit, src, out):
    factor = min(1.0, limit / (total + 1e-6))
    got = pamm.clip_grad_norm(src, limit, out=out)
    assert torch.equal(got, norm)
    for g, s, t in zip(grads, src, src if out is None else out):
        want = g.double() * factor
        assert plain64.within(t, want, plain64.stored(2.1 * plain64.U * want.abs(), want, t.dtype)) <= 1.0
        if out is not None:
            assert torch.equal(s, g)
        elif factor == 1.0:
            assert torch.equal(t, g)


@pytest.mark.parametrize("which", LARGE)
def test_large_lists(which):
    grads = next(g for name, g in large_lists() if name == which)
    total = plain64.global_norm(grads)
    norm = pamm.grad_norm(grads)
    assert abs(float(norm) - total) <= 1.01 * plain64.U * total
    assert torch.equal(norm, pamm.grad_norm(grads))
    for limit in (0.3 * total, 2 * total + 1):
        for out_dtype in (None, F32, BF16):
            src = [torch.empty_strided(g.shape, g.stride(), dtype=g.dtype, device="cuda").copy_(g) for g in grads] if out_dtype is None else grads
            out = None if out_dtype is None else [torch.empty_strided(g.shape, g.stride(), dtype=out_dtype, device="cuda") for g in grads]
            check(grads, total, norm, limit, src, out)


@pytest.mark.parametrize("size", [300, 200_000])
@pytest.mark.parametrize("count", [1, 23, 24, 25, 31, 32, 33, 95, 96, 97, 127, 128, 129, 447, 448, 449, 897])
def test_any_number_of_tensors(count, size):
    """Lists around what one launch holds, of tensors that the scaling joins the sums of itself and that it does not."""
    if size * count > 30_000_000:
        size = 30_000_000 // count
    grads = [normal((size + i % 5,), (BF16, F32)[i % 2], 100 + i) for i in range(count)]
    total = plain64.global_norm(grads)
    norm = pamm.grad_norm(grads)
    assert abs(float(norm) - total) <= 1.01 * plain64.U * total
    check(grads, total, norm, 0.4 * total, grads, [torch.empty_like(g) for g in grads])
    check(grads, total, norm, 0.4 * total, [g.clone() for g in grads], None)
