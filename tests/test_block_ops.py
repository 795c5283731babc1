"""Host-side checks of the operators around the projection: refusals, scratch sizes, rotary frequencies and the 64-bit
statements the GPU tests compare with.  No GPU is used."""
import ctypes
import math

import pytest
import torch

from paper_2506_02939_b200 import build as pamm_build

pamm_build.build()
from paper_2506_02939_b200 import pamm  # noqa: E402
from tests import plain64  # noqa: E402

FAKE, ODD, NULL = 0x1000, 0x1001, None       # never dereferenced: checks come first
BAD, UNSUP, WS = pamm.ERR_INVALID_ARG, pamm.ERR_UNSUPPORTED, pamm.ERR_WORKSPACE


def norm_forward(kind=0, X=FAKE, ldx=8, R=NULL, ldr=0, b=4, n=8, dt=0, w=FAKE, c=NULL, w_dt=0, eps=1e-5, Y=FAKE + 4096, ldy=8, H=NULL,
                 ldh=0, mean=FAKE, rstd=FAKE):
    return pamm._lib.pamm_norm_forward(kind, X, ldx, R, ldr, b, n, dt, w, c, w_dt, eps, Y, ldy, H, ldh, mean, rstd, None)


def test_norm_forward_refusals():
    for kw, code in [(dict(X=NULL), BAD), (dict(Y=NULL), BAD), (dict(b=-1), BAD), (dict(n=0), BAD), (dict(n=40000, ldx=40000, ldy=40000), UNSUP),
                     (dict(ldx=7), BAD), (dict(ldy=7), BAD), (dict(R=FAKE, ldr=7), BAD), (dict(H=FAKE, ldh=7), BAD), (dict(dt=2), UNSUP),
                     (dict(w_dt=5), UNSUP), (dict(kind=2), UNSUP), (dict(eps=-1.0), BAD), (dict(eps=math.nan), BAD), (dict(X=ODD), BAD),
                     (dict(w=FAKE + 2), BAD), (dict(c=ODD), BAD), (dict(mean=FAKE + 2), BAD), (dict(H=FAKE + 4096, ldh=8), BAD),
                     (dict(b=1 << 31), BAD)]:
        assert norm_forward(**kw) == code, kw
    assert norm_forward(b=0, X=NULL, Y=NULL) == pamm.OK


def test_norm_backward_refusals():
    def call(kind=0, dY=FAKE, lddy=8, X=FAKE, ldx=8, mean=FAKE, rstd=FAKE, b=4, n=8, dt=0, w=FAKE, w_dt=0, dH=NULL, lddh=0, dX=FAKE, lddx=8,
             dw=FAKE, dc=NULL, dw_dt=0, ws=FAKE, size=1 << 20):
        return pamm._lib.pamm_norm_backward(kind, dY, lddy, X, ldx, mean, rstd, b, n, dt, w, w_dt, dH, lddh, dX, lddx, dw, dc, dw_dt, ws, size, None)

    for kw, code in [(dict(dY=NULL), BAD), (dict(X=NULL), BAD), (dict(dX=NULL), BAD), (dict(mean=NULL), BAD), (dict(rstd=NULL), BAD),
                     (dict(lddy=7), BAD), (dict(ldx=7), BAD), (dict(lddx=7), BAD), (dict(dH=FAKE, lddh=7), BAD), (dict(b=-1), BAD),
                     (dict(n=0), BAD), (dict(n=32769, lddy=32769, ldx=32769, lddx=32769), UNSUP), (dict(dt=3), UNSUP), (dict(dw_dt=3), UNSUP),
                     (dict(w_dt=3), UNSUP), (dict(kind=-1), UNSUP), (dict(dw=FAKE + 2), BAD), (dict(dc=FAKE), BAD), (dict(ws=NULL), WS),
                     (dict(ws=FAKE + 16), WS), (dict(size=16), WS), (dict(dY=FAKE + 2), BAD), (dict(dw=NULL, dc=FAKE, ws=NULL), WS)]:
        assert call(**kw) == code, kw
    assert call(b=0, dw=NULL, dY=NULL, X=NULL, dX=NULL, ws=NULL) == pamm.OK


def test_rotary_refusals():
    def call(X=FAKE, Y=FAKE + 4096, xs=(64, 32, 8), ys=(64, 32, 8), batch=1, seq=2, heads=4, rotated=4, d=8, rot=8, dt=0, pairs=0, table=FAKE,
             rows=16, pos=NULL, pos_dt=0, first=0):
        return pamm._lib.pamm_rotary(X, *xs, Y, *ys, batch, seq, heads, rotated, d, rot, dt, pairs, 0, table, rows, pos, pos_dt, 0, 1, first, None)

    for kw, code in [(dict(X=NULL), BAD), (dict(Y=NULL), BAD), (dict(table=NULL), BAD), (dict(rotated=5), BAD), (dict(rotated=-1), BAD),
                     (dict(d=0), BAD), (dict(rot=7), BAD), (dict(rot=0), BAD), (dict(rot=10), BAD), (dict(d=600, rot=514), UNSUP),
                     (dict(dt=2), UNSUP), (dict(pairs=2), UNSUP), (dict(first=15), BAD), (dict(first=-1), BAD), (dict(rows=0), BAD),
                     (dict(pos=FAKE + 2), BAD), (dict(pos=FAKE + 4, pos_dt=1), BAD), (dict(pos=FAKE, pos_dt=2), UNSUP), (dict(X=ODD), BAD),
                     (dict(Y=FAKE, ys=(64, 32, 16)), BAD), (dict(batch=-1), BAD), (dict(batch=1 << 20, seq=1 << 20), UNSUP)]:
        assert call(**kw) == code, kw
    assert call(batch=0, X=NULL, Y=NULL) == pamm.OK and call(seq=0) == pamm.OK and call(heads=0, rotated=0) == pamm.OK
    for rot, base, kind, factor, trained, slow, fast, code in [
            (7, 1e4, 0, 1, 0, 1, 32, BAD), (0, 1e4, 0, 1, 0, 1, 32, BAD), (8, 0.0, 0, 1, 0, 1, 32, BAD), (8, 1e4, 4, 1, 0, 1, 32, UNSUP),
            (8, 1e4, 1, 0.5, 0, 1, 32, BAD), (8, 1e4, 3, 2, 0, 1, 32, BAD), (8, 1e4, 3, 2, 64, 32, 1, BAD), (514, 1e4, 0, 1, 0, 1, 32, UNSUP),
            (8, math.nan, 0, 1, 0, 1, 32, BAD), (8, 1e4, 2, math.inf, 0, 1, 32, BAD)]:
        with pytest.raises(pamm.PammError) as e:
            pamm.rotary_frequencies(rot, base, kind, factor, trained, slow, fast)
        assert e.value.code == code, (rot, base, kind)


def test_clip_refusals():
    def call(entry=(FAKE, 2, 8, 8, 0), out=None, count=1, limit=1.0, norm=FAKE, ws=FAKE, size=1 << 20):
        a = (ctypes.c_int64 * 5)(*entry)
        o = None if out is None else (ctypes.c_int64 * 5)(*out)
        return pamm._lib.pamm_clip_grad_norm(ctypes.addressof(a), None if o is None else ctypes.addressof(o), count, limit, norm, ws, size, None)

    for kw, code in [(dict(entry=(0, 2, 8, 8, 0)), BAD), (dict(entry=(ODD, 2, 8, 8, 0)), BAD), (dict(entry=(FAKE, 2, 8, 7, 0)), BAD),
                     (dict(entry=(FAKE, 2, 8, 8, 2)), UNSUP), (dict(entry=(FAKE, -1, 8, 8, 0)), BAD), (dict(count=-1), BAD), (dict(limit=-1.0), BAD),
                     (dict(limit=math.nan), BAD), (dict(norm=NULL), BAD), (dict(ws=NULL), WS), (dict(size=8), WS), (dict(ws=FAKE + 8), WS),
                     (dict(out=(FAKE, 8, 2, 2, 0)), BAD), (dict(out=(FAKE, 2, 8, 8, 7)), UNSUP), (dict(entry=(FAKE, 1 << 30, 1 << 30, 1 << 30, 0)), BAD)]:
        assert call(**kw) == code, kw


def test_scratch_sizes():
    w = pamm.workspace_bytes(pamm.WS_NORM_BACKWARD, 65536, 2048, 1, 1, pamm.BF16)
    assert w % 256 == 0 and 2 * 2048 * 4 <= w <= 16 << 20
    assert 0 < pamm.workspace_bytes(pamm.WS_NORM_BACKWARD, 0, 8, 1, 1, pamm.F32) <= w
    assert 0 < pamm.workspace_bytes(pamm.WS_GRAD_NORM, 0, 0, 0, 0, pamm.F32) <= 1 << 20
    for b, n in ((-1, 8), (4, 0), (4, 40000)):
        with pytest.raises(pamm.PammError):
            pamm.workspace_bytes(pamm.WS_NORM_BACKWARD, b, n, 1, 1, pamm.F32)


def test_python_refusals():
    x = torch.zeros((4, 8))
    with pytest.raises(ValueError):
        pamm.norm_forward(x)                                  # not on a device
    with pytest.raises(TypeError):
        pamm.norm_forward(x.half())
    with pytest.raises(TypeError):
        pamm.grad_norm([x])
    with pytest.raises(ValueError):
        pamm.rotary(x, x)
    with pytest.raises(ValueError):
        pamm.rotary(x.view(2, 2, 8), x)


def test_frequencies():
    rot, base, factor, trained = 64, 10000.0, 8.0, 2048
    plain, one = pamm.rotary_frequencies(rot, base)
    assert one == 1.0 and torch.allclose(plain, torch.tensor(plain64.rotary_frequencies(rot, base), dtype=torch.float64), rtol=1e-14)
    linear, one = pamm.rotary_frequencies(rot, base, pamm.ROTARY_LINEAR, factor)
    assert one == 1.0 and torch.allclose(linear, plain / factor, rtol=1e-14)
    wide, one = pamm.rotary_frequencies(rot, base, pamm.ROTARY_BASE, factor)
    assert one == 1.0 and wide[0] == plain[0] and abs(wide[-1] * factor / plain[-1] - 1) < 1e-12 and (wide <= plain).all()
    parts, amplitude = pamm.rotary_frequencies(rot, base, pamm.ROTARY_PARTS, factor, trained, 1.0, 32.0)
    turns = trained * plain / (2 * math.pi)
    assert torch.equal(parts[turns >= 32], plain[turns >= 32])
    assert torch.allclose(parts[turns <= 1], plain[turns <= 1] / factor, rtol=1e-14)
    mid = (turns > 1) & (turns < 32)
    keep = (turns[mid] - 1) / 31
    assert mid.any() and torch.allclose(parts[mid], keep * plain[mid] + (1 - keep) * plain[mid] / factor, rtol=1e-12)
    assert abs(amplitude - (0.1 * math.log(factor) + 1)) < 1e-15
    assert torch.equal(pamm.rotary_frequencies(rot, base, pamm.ROTARY_PARTS, 1.0, trained)[0], plain)
    assert len(pamm.rotary_frequencies(2, base, pamm.ROTARY_BASE, 4.0)[0]) == 1


@pytest.mark.parametrize("rms", [False, True])
def test_the_64_bit_norm_gradient_against_differences(rms):
    g = torch.Generator().manual_seed(1)
    x, dy, dh, v = (torch.randn((3, 10), generator=g, dtype=torch.float64) for _ in range(4))
    w, c, vw = (torch.randn(10, generator=g, dtype=torch.float64) for _ in range(3))
    _, _, mean, rstd = plain64.norm_forward(x, w, c, rms=rms)
    dx, dw, dc = plain64.norm_backward(dy, x, mean, rstd, w, dh, rms)

    def loss(x, w, c):
        y, h, _, _ = plain64.norm_forward(x, w, c, rms=rms)
        return float((dy * y).sum() + (dh * h).sum())

    t = 1e-5
    assert abs((loss(x + t * v, w, c) - loss(x - t * v, w, c)) / (2 * t) - float((dx * v).sum())) < 1e-6
    assert abs((loss(x, w + t * vw, c) - loss(x, w - t * vw, c)) / (2 * t) - float((dw * vw).sum())) < 1e-6
    assert abs((loss(x, w, c + t * vw) - loss(x, w, c - t * vw)) / (2 * t) - float((dc * vw).sum())) < 1e-6


def test_the_largest_rotary_row_and_one_beyond():
    def call(heads, d, batch=0):
        return pamm._lib.pamm_rotary(FAKE, 0, 0, d, FAKE, 0, 0, d, batch, 1, heads, heads, d, 2, 0, 0, 0, FAKE, 4, None, 0, 0, 0, 0, None)

    for heads, d in ((1, 2 ** 24), (2 ** 23, 2), (2 ** 12, 2 ** 12)):
        assert call(heads, d) == pamm.OK                  # of no sequence: nothing is launched
        assert call(heads, d + 1, 1) == call(heads, d + 1) == pamm.ERR_UNSUPPORTED
    assert call(2 ** 24 + 1, 2) == pamm.ERR_UNSUPPORTED


def test_a_rotary_table_is_computed_on_its_own_device(monkeypatch):
    """With stand-ins for a second device: the launch happens while the table's device is the current one."""
    current, launched = [0], []

    class Device:
        def __init__(self, device):
            self.index = torch.device(device).index

        def __enter__(self):
            self.before, current[0] = current[0], self.index

        def __exit__(self, *_):
            current[0] = self.before

    class Table:
        shape, dtype, device, is_cuda = (5, 8), torch.float32, torch.device("cuda", 1), True
        is_contiguous, data_ptr = (lambda self: True), (lambda self: FAKE)

    class Library:
        def pamm_rotary_table(self, *args):
            launched.append((current[0], args[-1]))
            return pamm.OK

    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(pamm, "_lib", Library())
    monkeypatch.setattr(pamm, "_stream", lambda stream: ("the stream of", current[0]))
    pamm.rotary_table(5, torch.ones(4, dtype=torch.float64), out=Table())
    assert launched == [(1, ("the stream of", 1))] and current == [0]
