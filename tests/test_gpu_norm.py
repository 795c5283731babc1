"""Layer norm and its root-mean-square form against 64-bit statements, element by element."""
import pytest
import torch

from paper_2506_02939_b200 import build as pamm_build

pamm_build.build()
from paper_2506_02939_b200 import pamm  # noqa: E402
from tests import plain64  # noqa: E402

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def rows(b, n, dtype, seed, scale=1.0, pad=0, shift=0):
    """b x n with `pad` elements between rows and a base `shift` elements off, inside memory filled with NaN."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    ld = n + pad
    room = torch.full((shift + b * ld + 64,), float("nan"), device="cuda", dtype=dtype)
    view = room[shift:shift + b * ld].view(b, ld)[:, :n]
    view.copy_(torch.randn((b, n), generator=g, device="cuda") * scale)
    return view, room


def untouched(view, room, pad, shift):
    b, n = view.shape
    mask = torch.ones(room.shape, dtype=torch.bool, device="cuda")
    mask[shift:shift + b * (n + pad)].view(b, n + pad)[:, :n] = False
    return bool(torch.isnan(room[mask].float()).all())


def vector(n, dtype, seed, centre=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (centre + 0.2 * torch.randn(n, generator=g, device="cuda")).to(dtype)


SIZES = [(1, 1), (3, 2), (2, 7), (5, 8), (9, 31), (300, 64), (37, 100), (64, 512), (33, 520), (3, 1000), (17, 1999), (150, 2048),
         (11, 4096), (5, 5003), (3, 8192), (2, 16384), (2, 16391), (1, 32768), (90, 8200), (170, 9001), (41, 20000), (39, 32761)]


@pytest.mark.parametrize("dtype,w_dtype", [(F32, F32), (BF16, BF16), (BF16, F32), (F32, BF16)])
@pytest.mark.parametrize("b,n", SIZES)
def test_forward_and_backward_of_all_sizes(b, n, dtype, w_dtype):
    for k, (rms, bias, add, pad, shift) in enumerate([(False, True, False, 0, 0), (True, False, True, 8, 8), (False, False, True, 3, 1),
                                                      (True, True, False, 16 - n % 16 if n % 16 else 0, 0)]):
        seed = 100 * k + n
        x, _ = rows(b, n, dtype, seed, pad=pad, shift=shift)
        r = rows(b, n, dtype, seed + 1, 0.5, pad, shift)[0] if add else None
        w, c = vector(n, w_dtype, seed + 2), vector(n, w_dtype, seed + 3, 0.0) if bias else None
        y, y_room = rows(b, n, dtype, 0, pad=pad, shift=shift)
        y, h, mean, rstd = pamm.norm_forward(x, w, c, residual=r, rms=rms, Y=y)
        want = plain64.norm_forward(x, w, c, r, 1e-5, rms)
        by, bh, bm, bs = plain64.norm_forward_bounds(x, w, c, r, 1e-5, rms)
        assert plain64.within(y, want[0], plain64.stored(by, want[0], dtype)) <= 1.0
        assert untouched(y, y_room, pad, shift)
        assert plain64.within(rstd, want[3], plain64.stored(bs, want[3], F32)) <= 1.0
        assert (mean is None) == rms
        if not rms:
            assert plain64.within(mean, want[2], plain64.stored(bm, want[2], F32)) <= 1.0
        if add:
            assert plain64.within(h, want[1], plain64.stored(bh, want[1], dtype)) <= 1.0
        else:
            assert h is x
        dy, _ = rows(b, n, dtype, seed + 4, 1e-2, pad, shift)
        dh = rows(b, n, dtype, seed + 5, 1e-2, pad, shift)[0] if add else None
        dx, dx_room = rows(b, n, dtype, 0, pad=pad, shift=shift)
        dx, dw, dc = pamm.norm_backward(dy, h, mean, rstd, w, bias=bias, dH=dh, dX=dx)
        gx, gw, gc = plain64.norm_backward(dy, h, mean, rstd, w, dh, rms)
        bx, bw, bc = plain64.norm_backward_bounds(dy, h, mean, rstd, w, dh, rms)
        assert plain64.within(dx, gx, plain64.stored(bx, gx, dtype)) <= 1.0
        assert untouched(dx, dx_room, pad, shift)
        assert dw.dtype == w_dtype and plain64.within(dw, gw, plain64.stored(bw, gw, w_dtype)) <= 1.0
        assert (dc is None) != bias
        if bias:
            assert plain64.within(dc, gc, plain64.stored(bc, gc, w_dtype)) <= 1.0


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("b,n", [(70, 31), (40, 1000), (9, 5003), (21, 9001), (5, 20000), (3, 32768)])
def test_matrices_aligned_differently(b, n, dtype):
    for rms in (False, True):
        pads = [(0, 0), (1, 0), (8, 3), (5, 1), (2, 2)]             # of x, r (dy), y (dx), h (dh): distances and bases apart
        x, r = (rows(b, n, dtype, k, pad=pads[k][0], shift=pads[k][1])[0] for k in (0, 1))
        w, c = vector(n, F32, 2), vector(n, F32, 3, 0.0)
        (y, y_room), (h, h_room) = (rows(b, n, dtype, 0, pad=pads[k][0], shift=pads[k][1]) for k in (2, 3))
        y, h, mean, rstd = pamm.norm_forward(x, w, c, residual=r, rms=rms, Y=y, H=h)
        want = plain64.norm_forward(x, w, c, r, 1e-5, rms)
        by, bh, _, _ = plain64.norm_forward_bounds(x, w, c, r, 1e-5, rms)
        assert plain64.within(y, want[0], plain64.stored(by, want[0], dtype)) <= 1.0 and untouched(y, y_room, *pads[2])
        assert plain64.within(h, want[1], plain64.stored(bh, want[1], dtype)) <= 1.0 and untouched(h, h_room, *pads[3])
        dy, dh = (rows(b, n, dtype, 10 + k, 1e-2, *pads[k])[0] for k in (1, 3))
        dx, dx_room = rows(b, n, dtype, 0, pad=pads[2][0], shift=pads[2][1])
        dx, dw, dc = pamm.norm_backward(dy, h, mean, rstd, w, bias=True, dH=dh, dX=dx)
        gx, gw, gc = plain64.norm_backward(dy, h, mean, rstd, w, dh, rms)
        bx, bw, bc = plain64.norm_backward_bounds(dy, h, mean, rstd, w, dh, rms)
        assert plain64.within(dx, gx, plain64.stored(bx, gx, dtype)) <= 1.0 and untouched(dx, dx_room, *pads[2])
        assert plain64.within(dw, gw, plain64.stored(bw, gw, F32)) <= 1.0 and plain64.within(dc, gc, plain64.stored(bc, gc, F32)) <= 1.0


@pytest.mark.parametrize("b", [1, 2, 31, 147, 149, 1000, 4099, 20000])
@pytest.mark.parametrize("n,dtype", [(256, BF16), (1024, F32), (2048, BF16), (64, BF16), (40, F32), (128, F32), (100, BF16), (333, BF16), (480, BF16), (200, F32)])
def test_weight_gradients_over_many_rows(b, n, dtype):
    x, _ = rows(b, n, dtype, b)
    dy, _ = rows(b, n, dtype, b + 1, 1e-3)
    y, _, mean, rstd = pamm.norm_forward(x)
    want, by = plain64.norm_forward(x)[0], plain64.norm_forward_bounds(x)[0]
    assert plain64.within(y, want, plain64.stored(by, want, dtype)) <= 1.0
    for w_dtype in (F32, BF16):
        w = vector(n, w_dtype, 3)
        dx, dw, dc = pamm.norm_backward(dy, x, mean, rstd, w, bias=True, dw_dtype=F32)
        gx, gw, gc = plain64.norm_backward(dy, x, mean, rstd, w)
        bx, bw, bc = plain64.norm_backward_bounds(dy, x, mean, rstd, w)
        assert dw.dtype == F32
        for got, want, bound, dt in ((dx, gx, bx, dtype), (dw, gw, bw, F32), (dc, gc, bc, F32)):
            assert plain64.within(got, want, plain64.stored(bound, want, dt)) <= 1.0
        again = pamm.norm_backward(dy, x, mean, rstd, w, bias=True, dw_dtype=F32)
        assert all(torch.equal(p, q) for p, q in zip((dx, dw, dc), again))       # the same bits every time


def test_empty_batch():
    for dtype in (F32, BF16):
        x = torch.empty((0, 96), dtype=dtype, device="cuda")
        w = vector(96, dtype, 1)
        y, h, mean, rstd = pamm.norm_forward(x, w)
        assert y.shape == (0, 96) and mean.shape == rstd.shape == (0,)
        dw = torch.full((96,), float("nan"), device="cuda")
        dx, dw, dc = pamm.norm_backward(x, x, mean, rstd, w, bias=True, dw=dw)
        assert dx.shape == (0, 96) and not dw.any() and not dc.any()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [40, 2048, 2051, 20000])
def test_rows_of_infinities_nan_and_zeros_keep_to_themselves(n, dtype):
    x, _ = rows(7, n, dtype, 5)
    x[1] = 0.0
    x[2, n // 2] = float("inf")
    x[3, n - 1] = float("nan")
    x[4] = -torch.finfo(dtype).max
    x[5] = 3.0
    dy, _ = rows(7, n, dtype, 6)
    for rms in (False, True):
        y, _, mean, rstd = pamm.norm_forward(x, rms=rms)
        dx, _, _ = pamm.norm_backward(dy, x, mean, rstd)
        want, _, _, s = plain64.norm_forward(x, rms=rms)
        for row in (0, 1, 5, 6):
            by = plain64.norm_forward_bounds(x[row:row + 1], rms=rms)[0]
            if not rms and row == 5:         # the row of a constant: what is left of it is the mean's rounding
                by = by + 80 * plain64.U * 3.0 * float(rstd[row])
            assert plain64.within(y[row:row + 1], want[row:row + 1], plain64.stored(by, want[row:row + 1], dtype)) <= 1.0
            assert torch.isfinite(dx[row]).all()
        assert abs(float(rstd[1]) - 1e-5 ** -0.5) < 1e-3 and not y[1].any()
        assert torch.isnan(y[3]).all() and torch.isnan(rstd[3])
        assert torch.isnan(y[2, n // 2]) if rms else torch.isnan(y[2]).all()


@pytest.mark.parametrize("dtype,w_dtype", [(F32, F32), (BF16, BF16), (BF16, F32), (F32, BF16)])
@pytest.mark.parametrize("n,pad", [(64, 0), (256, 0), (777, 0), (2040, 3), (2048, 0)])
def test_weights_anywhere(n, pad, dtype, w_dtype):
    """Weights and biases that start off the 16-byte grid, at the very ends of memory filled with NaN."""
    b = 37
    x, dy = rows(b, n, dtype, 1, pad=pad)[0], rows(b, n, dtype, 2, 1e-2, pad)[0]
    for shift in range(0, 9):
        room = torch.full((2, shift + n), float("nan"), device="cuda", dtype=w_dtype)
        w, c = room[0, shift:], room[1, shift:]
        w.copy_(vector(n, w_dtype, 3))
        c.copy_(vector(n, w_dtype, 4, 0.0))
        y, _, mean, rstd = pamm.norm_forward(x, w, c)
        want = plain64.norm_forward(x, w, c)[0]
        by = plain64.norm_forward_bounds(x, w, c)[0]
        assert plain64.within(y, want, plain64.stored(by, want, dtype)) <= 1.0
        dx, dw, dc = pamm.norm_backward(dy, x, mean, rstd, w, bias=True)
        gx, gw, gc = plain64.norm_backward(dy, x, mean, rstd, w)
        bx, bw, bc = plain64.norm_backward_bounds(dy, x, mean, rstd, w)
        for got, wanted, bound, dt in ((dx, gx, bx, dtype), (dw, gw, bw, w_dtype), (dc, gc, bc, w_dtype)):
            assert plain64.within(got, wanted, plain64.stored(bound, wanted, dt)) <= 1.0


def test_a_large_mean_does_not_cost_the_variance():
    n = 4096
    x = (1000.0 + rows(8, n, F32, 7, 0.01)[0]).contiguous()
    y, _, mean, rstd = pamm.norm_forward(x)
    want, _, m, s = plain64.norm_forward(x)
    by, _, bm, bs = plain64.norm_forward_bounds(x)
    assert plain64.within(rstd, s, plain64.stored(bs, s, F32)) <= 1.0
    assert plain64.within(y, want, plain64.stored(by, want, F32)) <= 1.0
    assert float((rstd.double() / s - 1).abs().max()) < 0.2           # a sum of squares around zero would have lost it all


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("b,n", [(70, 2048), (70, 1001), (3, 20000)])
def test_outputs_in_the_place_of_inputs(b, n, dtype):
    x, _ = rows(b, n, dtype, 1)
    r, _ = rows(b, n, dtype, 2)
    dy, dh = rows(b, n, dtype, 3)[0], rows(b, n, dtype, 4)[0]
    w = vector(n, dtype, 5)
    y, h, mean, rstd = pamm.norm_forward(x, w, residual=r)
    x1, r1 = x.clone(), r.clone()
    y1, h1, _, _ = pamm.norm_forward(x1, w, residual=r1, H=x1)
    assert h1 is x1 and torch.equal(x1, h) and torch.equal(y1, y)
    x2, r2 = x.clone(), r.clone()
    pamm.norm_forward(x2, w, residual=r2, H=r2, Y=x2)
    assert torch.equal(r2, h) and torch.equal(x2, y)
    x3 = h.clone()
    pamm.norm_forward(x3, w, Y=x3)
    assert torch.equal(x3, pamm.norm_forward(h, w)[0])
    want = pamm.norm_backward(dy, h, mean, rstd, w, bias=True, dH=dh)
    for place in range(3):
        a = [dy.clone(), h.clone(), dh.clone()]
        got = pamm.norm_backward(a[0], a[1], mean, rstd, w, bias=True, dH=a[2], dX=a[place])
        assert got[0] is a[place] and all(torch.equal(p, q) for p, q in zip(got, want))


def test_frozen_weight_and_no_weight():
    x, dy = rows(50, 384, BF16, 1)[0], rows(50, 384, BF16, 2)[0]
    ones = torch.ones(384, dtype=BF16, device="cuda")
    y, _, mean, rstd = pamm.norm_forward(x)
    assert torch.equal(y, pamm.norm_forward(x, ones)[0])
    dx, dw, dc = pamm.norm_backward(dy, x, mean, rstd, need_dw=False)
    full = pamm.norm_backward(dy, x, mean, rstd, ones, bias=True)
    assert dw is None and dc is None and torch.equal(dx, full[0])
    only_bias = pamm.norm_backward(dy, x, mean, rstd, ones, need_dw=False, dc=torch.empty_like(ones))
    assert torch.equal(only_bias[2], full[2])


@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gradients_against_differences(dtype, rms):
    """<gradient, direction> against central differences of the 64-bit loss <dy, y> (+ <dh, h>) along x, w and c."""
    b, n, t = 6, 200, 1e-4
    x, dy = rows(b, n, dtype, 11)[0].contiguous(), rows(b, n, dtype, 12, 0.1)[0].contiguous()
    dh = rows(b, n, dtype, 13, 0.1)[0].contiguous()
    w, c = vector(n, F32, 14), vector(n, F32, 15, 0.0)
    _, _, mean, rstd = pamm.norm_forward(x, w, c, rms=rms)
    dx, dw, dc = pamm.norm_backward(dy, x, mean, rstd, w, bias=True, dH=dh)
    bx, bw, bc = plain64.norm_backward_bounds(dy, x, mean, rstd, w, dh, rms)
    g = torch.Generator(device="cuda").manual_seed(16)

    def loss(x, w, c):
        y, h, _, _ = plain64.norm_forward(x, w, c, rms=rms)
        return float((dy.double() * y).sum() + (dh.double() * h).sum())

    for which, grad, bound, dt in ((0, dx, bx, dtype), (1, dw, bw, F32), (2, dc, bc, F32)):
        args = [x.double(), w.double(), c.double()]
        v = torch.randn(args[which].shape, generator=g, device="cuda", dtype=torch.float64)
        up, down = list(args), list(args)
        up[which], down[which] = args[which] + t * v, args[which] - t * v
        slope = (loss(*up) - loss(*down)) / (2 * t)
        # storage and arithmetic of the gradient; mean and rstd were rounded to fp32 (about 100 U of each term); t^2 of the differences
        room = float((plain64.stored(bound, grad.double(), dt) * v.abs()).sum()) + 100 * plain64.U * float((grad.double() * v).abs().sum())
        room += 100 * t * t * float((grad.double() * v).abs().sum())
        assert abs(float((grad.double() * v).sum()) - slope) <= room


def test_row_distances_beyond_32_bits():
    n, far = 1000, 2 ** 30 + 8
    room = torch.zeros(2 * far + n, dtype=BF16, device="cuda")
    out = torch.zeros(2 * far + n, dtype=BF16, device="cuda")
    x, y = (torch.as_strided(t, (3, n), (far, 1)) for t in (room, out))
    near, dy = rows(3, n, BF16, 3)[0].contiguous(), rows(3, n, BF16, 4)[0].contiguous()
    x.copy_(near)
    w = vector(n, BF16, 1)
    _, _, mean, rstd = pamm.norm_forward(x, w, Y=y)
    assert torch.equal(y, pamm.norm_forward(near, w)[0])
    want = pamm.norm_backward(dy, near, mean, rstd, w)
    got = pamm.norm_backward(dy, x, mean, rstd, w, dX=y)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_on_another_stream_and_in_a_graph():
    x, dy = rows(400, 768, BF16, 1)[0].contiguous(), rows(400, 768, BF16, 2)[0].contiguous()
    w = vector(768, BF16, 3)
    y, _, mean, rstd = pamm.norm_forward(x, w)
    want = pamm.norm_backward(dy, x, mean, rstd, w)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    y1, _, m1, s1 = pamm.norm_forward(x, w, stream=side)
    got = pamm.norm_backward(dy, x, m1, s1, w, stream=side)
    side.synchronize()
    assert torch.equal(y, y1) and all(torch.equal(a, b) for a, b in zip(got[:2], want[:2]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y2, _, m2, s2 = pamm.norm_forward(x, w)
        got2 = pamm.norm_backward(dy, x, m2, s2, w)
    y2.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, y2) and all(torch.equal(a, b) for a, b in zip(got2[:2], want[:2]))


def test_prepared_calls():
    x, w = rows(64, 512, BF16, 1)[0].contiguous(), vector(512, BF16, 2)
    y = torch.zeros_like(x)
    call = pamm.prepared(pamm.norm_forward, x, w, rms=True, Y=y)
    assert not y.any()
    call()
    assert torch.equal(y, pamm.norm_forward(x, w, rms=True)[0])
    dy, (_, _, _, rstd) = rows(64, 512, BF16, 3)[0].contiguous(), pamm.norm_forward(x, w, rms=True)
    dw = torch.zeros_like(w)
    pamm.prepared(pamm.norm_backward, dy, x, None, rstd, w, dw=dw)()
    assert torch.equal(dw, pamm.norm_backward(dy, x, None, rstd, w)[1])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,pad,shift", [(40, 0, 0), (128, 0, 0), (250, 0, 1), (333, 0, 0), (512, 0, 0), (1000, 0, 0), (1999, 0, 3), (2048, 0, 0),
                                         (8200, 0, 0), (20000, 0, 0)])
def test_rows_of_the_types_largest_and_lowest_values(n, pad, shift, dtype):
    """Masked rows hold the type's lowest value; the squares of values from 1e19 on leave fp32's range, mean, s and y do not."""
    top = torch.finfo(dtype).max
    x, _ = rows(9, n, dtype, 5, pad=pad, shift=shift)
    x[1] = -top
    x[2, 3:] = -top
    x[3, ::2], x[3, 1::2] = top, -top
    x[4, n // 2] = top
    x[5] *= 1e25
    x[6] = top
    x[6, n // 3] = -top
    x[7] *= 1e19
    dy, dh = rows(9, n, dtype, 6, pad=pad, shift=shift)[0], rows(9, n, dtype, 7, pad=pad, shift=shift)[0]
    w, c = vector(n, F32, 8), vector(n, F32, 9, 0.0)
    for rms in (False, True):
        y, _, mean, rstd = pamm.norm_forward(x, w, c, rms=rms)
        want = plain64.norm_forward(x, w, c, rms=rms)
        by, _, bm, bs = plain64.norm_forward_bounds(x, w, c, rms=rms)
        assert torch.isfinite(y).all() and torch.isfinite(rstd).all() and (rstd > 0).all()
        assert plain64.within(y, want[0], plain64.stored(by, want[0], dtype)) <= 1.0
        # s of the largest values is a subnormal of fp32: half a unit of those beside the relative bound
        assert plain64.within(rstd, want[3], bs + want[3] * plain64.U + 2.0 ** -149) <= 1.0
        if not rms:
            assert torch.isfinite(mean).all() and plain64.within(mean, want[2], plain64.stored(bm, want[2], F32)) <= 1.0
        dx, dw, dc = pamm.norm_backward(dy, x, mean, rstd, w, bias=True, dH=dh)
        gx, gw, gc = plain64.norm_backward(dy, x, mean, rstd, w, dh, rms)
        bx, bw, bc = plain64.norm_backward_bounds(dy, x, mean, rstd, w, dh, rms)
        for got, wanted, bound, dt in ((dx, gx, bx, dtype), (dw, gw, bw, F32), (dc, gc, bc, F32)):
            assert torch.isfinite(got).all()
            assert plain64.within(got, wanted, plain64.stored(bound, wanted, dt)) <= 1.0


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [100, 333, 520, 2048, 9001])
def test_a_constant_row_of_the_lowest_value_has_finite_gradients(n, dtype):
    """Its mean is the value itself and s = eps^-1/2: what a thread holds beside the row's end must not count."""
    top = torch.finfo(dtype).max
    x = torch.full((3, n), -top, dtype=dtype, device="cuda")
    dy, w = rows(3, n, dtype, 6)[0], vector(n, F32, 8)
    mean = x[:, 0].float().contiguous()
    rstd = torch.full((3,), 1e-5 ** -0.5, device="cuda")
    dx, dw, dc = pamm.norm_backward(dy, x, mean, rstd, w, bias=True)
    gx, gw, gc = plain64.norm_backward(dy, x, mean, rstd, w)
    bx, bw, bc = plain64.norm_backward_bounds(dy, x, mean, rstd, w)
    for got, wanted, bound, dt in ((dx, gx, bx, dtype), (dw, gw, bw, F32), (dc, gc, bc, F32)):
        assert plain64.within(got, wanted, plain64.stored(bound, wanted, dt)) <= 1.0


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("b,n", [(9, 40), (4800, 250), (9, 333), (4801, 512), (9600, 1024), (9, 2048), (9, 20000)])
def test_extreme_rows_with_a_residual_in_and_out_of_place(b, n, dtype):
    top = torch.finfo(dtype).max
    x, r = rows(b, n, dtype, 1)[0].contiguous(), rows(b, n, dtype, 2, 0.5)[0].contiguous()
    x[2] = -top
    x[3, 1:] = -top
    x[5, ::2] = top
    x[b - 1] *= 1e25
    w = vector(n, F32, 3)
    for rms in (False, True):
        y, h, mean, rstd = pamm.norm_forward(x, w, residual=r, rms=rms)
        want = plain64.norm_forward(x, w, None, r, 1e-5, rms)
        by = plain64.norm_forward_bounds(x, w, None, r, 1e-5, rms)[0]
        assert torch.isfinite(y).all() and torch.isfinite(h).all()
        assert plain64.within(y, want[0], plain64.stored(by, want[0], dtype)) <= 1.0
        # in place: these rows are those of the stored h
        stored = plain64.norm_forward(h, w, None, None, 1e-5, rms)
        bs = plain64.norm_forward_bounds(h, w, None, None, 1e-5, rms)[0]
        extreme = [2, 3, 5, b - 1]
        for place in range(2):
            both = [x.clone(), r.clone()]
            y1, h1, _, _ = pamm.norm_forward(both[0], w, residual=both[1], rms=rms, H=both[place], Y=both[1 - place])
            assert torch.equal(h1, h)
            keep = torch.ones(b, dtype=torch.bool, device="cuda")
            keep[extreme] = False
            assert torch.equal(y1[keep], y[keep])
            assert plain64.within(y1[extreme], stored[0][extreme], plain64.stored(bs, stored[0], dtype)[extreme]) <= 1.0


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [40, 2048, 2051, 20000])
def test_gradients_of_rows_of_infinities_and_nan(n, dtype):
    """NaN exactly where the formula has it, in dx, dw and dc; the other rows and columns as without them."""
    x, _ = rows(6, n, dtype, 5)
    x[2, n // 2] = float("inf")
    x[3, n - 1] = float("nan")
    dy, _ = rows(6, n, dtype, 6)
    dy[4, 1] = float("nan")
    dy[5, 2] = float("-inf")
    w = vector(n, F32, 8)
    for rms in (False, True):
        _, _, mean, rstd = pamm.norm_forward(x, w, rms=rms)
        dx, dw, dc = pamm.norm_backward(dy, x, mean, rstd, w, bias=True)
        want = plain64.norm_backward(dy, x, mean, rstd, w, None, rms)
        bounds = plain64.norm_backward_bounds(dy, x, mean, rstd, w, None, rms)
        for got, wanted, bound, dt in zip((dx, dw, dc), want, bounds, (dtype, F32, F32)):
            assert torch.equal(torch.isnan(got), torch.isnan(wanted))
            fine = torch.isfinite(wanted)
            assert torch.equal(got[~fine & ~torch.isnan(wanted)].double(), wanted[~fine & ~torch.isnan(wanted)])
            assert plain64.within(got[fine], wanted[fine], plain64.stored(bound, wanted, dt)[fine]) <= 1.0


@pytest.mark.parametrize("dtype,w_dtype", [(F32, F32), (BF16, BF16), (BF16, F32), (F32, BF16)])
@pytest.mark.parametrize("n,b", [(40, 20001), (128, 20001), (250, 20001), (480, 20001), (481, 20001), (512, 20001), (1024, 20001), (2048, 20001), (1999, 9001)])
def test_many_rows_in_every_form(n, b, dtype, w_dtype):
    """Rows enough for the kernels of large batches: two rows a thread (an odd number of them), parts of a warp, a shared-memory
    ring that goes round, with the residual, its gradient and the bias each there and not there."""
    x, r = rows(b, n, dtype, 1)[0], rows(b, n, dtype, 2, 0.5)[0]
    dy, dh = rows(b, n, dtype, 3, 1e-2)[0], rows(b, n, dtype, 4, 1e-2)[0]
    w, c = vector(n, w_dtype, 5), vector(n, w_dtype, 6, 0.0)
    for rms in (False, True):
        for add in (False, True):
            for bias in (False, True):
                args = (x, w, c if bias else None, r if add else None, 1e-5, rms)
                y, h, mean, rstd = pamm.norm_forward(x, w, args[2], residual=args[3], rms=rms)
                want = plain64.norm_forward(*args)
                by, bh, bm, bs = plain64.norm_forward_bounds(*args)
                assert plain64.within(y, want[0], plain64.stored(by, want[0], dtype)) <= 1.0
                assert plain64.within(rstd, want[3], plain64.stored(bs, want[3], F32)) <= 1.0
                if add:
                    assert plain64.within(h, want[1], plain64.stored(bh, want[1], dtype)) <= 1.0
                if not rms:
                    assert plain64.within(mean, want[2], plain64.stored(bm, want[2], F32)) <= 1.0
                dx, dw, dc = pamm.norm_backward(dy, h, mean, rstd, w, bias=bias, dH=dh if add else None)
                args = (dy, h, mean, rstd, w, dh if add else None, rms)
                gx, gw, gc = plain64.norm_backward(*args)
                bx, bw, bc = plain64.norm_backward_bounds(*args)
                assert plain64.within(dx, gx, plain64.stored(bx, gx, dtype)) <= 1.0
                assert plain64.within(dw, gw, plain64.stored(bw, gw, w_dtype)) <= 1.0
                if bias:
                    assert plain64.within(dc, gc, plain64.stored(bc, gc, w_dtype)) <= 1.0


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("b,n", [(9001, 250), (9001, 509), (5001, 2048), (3001, 8200)])
def test_many_rows_of_matrices_aligned_differently(b, n, dtype):
    pads = [(0, 0), (1, 0), (8, 3), (5, 1)]             # of x, r (dy), y (dx), h (dh)
    x, r = (rows(b, n, dtype, k, pad=pads[k][0], shift=pads[k][1])[0] for k in (0, 1))
    w, c = vector(n, F32, 2), vector(n, F32, 3, 0.0)
    for rms in (False, True):
        (y, y_room), (h, h_room) = (rows(b, n, dtype, 0, pad=pads[k][0], shift=pads[k][1]) for k in (2, 3))
        y, h, mean, rstd = pamm.norm_forward(x, w, c, residual=r, rms=rms, Y=y, H=h)
        want = plain64.norm_forward(x, w, c, r, 1e-5, rms)
        by, bh, _, _ = plain64.norm_forward_bounds(x, w, c, r, 1e-5, rms)
        assert plain64.within(y, want[0], plain64.stored(by, want[0], dtype)) <= 1.0 and untouched(y, y_room, *pads[2])
        assert plain64.within(h, want[1], plain64.stored(bh, want[1], dtype)) <= 1.0 and untouched(h, h_room, *pads[3])
        dy, dh = (rows(b, n, dtype, 10 + k, 1e-2, *pads[k])[0] for k in (1, 3))
        dx, dx_room = rows(b, n, dtype, 0, pad=pads[2][0], shift=pads[2][1])
        dx, dw, dc = pamm.norm_backward(dy, h, mean, rstd, w, bias=True, dH=dh, dX=dx)
        gx, gw, gc = plain64.norm_backward(dy, h, mean, rstd, w, dh, rms)
        bx, bw, bc = plain64.norm_backward_bounds(dy, h, mean, rstd, w, dh, rms)
        assert plain64.within(dx, gx, plain64.stored(bx, gx, dtype)) <= 1.0 and untouched(dx, dx_room, *pads[2])
        assert plain64.within(dw, gw, plain64.stored(bw, gw, F32)) <= 1.0 and plain64.within(dc, gc, plain64.stored(bc, gc, F32)) <= 1.0
