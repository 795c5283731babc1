"""Rotary positions against 64-bit statements, element by element."""
import math

import numpy as np
import pytest
import torch

from paper_2506_02939_b200 import build as pamm_build

pamm_build.build()
from paper_2506_02939_b200 import pamm  # noqa: E402
from tests import plain64  # noqa: E402

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def normal(shape, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def table_of(rot, length=64, **kw):
    return pamm.rotary_table(length, *pamm.rotary_frequencies(rot, **kw))


def check(got, x, table, positions, rotated, rot, interleaved, transposed):
    rows = table[positions]
    want, size = plain64.rotary(x, rows[..., :rot // 2], rows[..., rot // 2:], rotated, rot, interleaved, transposed)
    assert plain64.within(got, want, plain64.stored(3 * plain64.U * size, want, x.dtype)) <= 1.0
    rest = torch.ones_like(got, dtype=torch.bool)
    rest[:, :, :rotated, :rot] = False
    assert torch.equal(got[rest], x[rest])           # what is not turned passes through bit for bit


SHAPES = [(1, 1, 1, 2, 2), (1, 3, 2, 8, 4), (2, 5, 3, 10, 6), (3, 17, 4, 64, 64), (2, 9, 5, 80, 20), (1, 33, 48, 128, 128), (4, 1, 12, 128, 64),
          (2, 7, 3, 256, 256), (2, 6, 1, 40, 40), (1, 4, 2, 512, 512), (1, 2, 70, 96, 48), (2, 3, 3, 33, 32)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("batch,seq,heads,d,rot", SHAPES)
def test_all_shapes(batch, seq, heads, d, rot, interleaved, dtype):
    table = table_of(rot)
    for k, (rotated, transposed, given) in enumerate([(heads, False, None), (heads, True, torch.int64), ((heads + 1) // 2, False, torch.int32),
                                                      (0, False, None)]):
        x = normal((batch, seq, heads, d), dtype, 10 * k + d)
        g = torch.Generator().manual_seed(k)
        pos = None if given is None else torch.randint(0, 64, (batch, seq), generator=g).to(given).cuda()
        where = torch.arange(seq, device="cuda").expand(batch, -1) + 2 if pos is None else pos.long()
        got = pamm.rotary(x, table, pos, rotated=rotated, interleaved=interleaved, transposed=transposed, first=2)
        check(got, x, table, where, rotated, rot, interleaved, transposed)
        inside = x.clone()
        assert pamm.rotary(inside, table, pos, rotated=rotated, interleaved=interleaved, transposed=transposed, first=2, out=inside) is inside
        assert torch.equal(inside, got)
    assert pamm.last_device_status() == pamm.OK


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("interleaved", [False, True])
def test_strides(dtype, interleaved):
    table = table_of(64)
    batch, seq, heads, d = 2, 11, 6, 64
    where = torch.arange(seq, device="cuda").expand(batch, -1)
    fused = normal((batch * seq, heads * d + 8), dtype, 1)                                    # padded rows of [Q|K|V]
    room = normal((batch, heads, seq, d), dtype, 2)                                           # heads before tokens
    odd = normal((batch * seq * heads * d + 1,), dtype, 3)[1:].view(batch, seq, heads, d)     # off the 16-byte grid
    gap = normal((batch, seq, heads, d + 3), dtype, 4)[..., :d]
    one = normal((1, 1, heads, d), dtype, 5).expand(batch, seq, heads, d)                     # broadcast input
    back = normal((batch, seq, heads, d), dtype, 6).flip(1)
    for x in (fused.view(batch, seq, -1)[:, :, 8:].unflatten(2, (heads, d)), room.transpose(1, 2), odd, gap, one, back):
        got = pamm.rotary(x, table, rotated=4, interleaved=interleaved)
        check(got, x, table, where, 4, 64, interleaved, False)
        wide = torch.full((batch, seq, heads + 1, d + 5), float("nan"), dtype=dtype, device="cuda")
        pamm.rotary(x, table, rotated=4, interleaved=interleaved, out=wide[:, :, 1:, 2:2 + d])
        assert torch.equal(wide[:, :, 1:, 2:2 + d], got)
        assert torch.isnan(wide[:, :, 0]).all() and torch.isnan(wide[..., :2]).all() and torch.isnan(wide[..., 2 + d:]).all()
    x = fused.view(batch, seq, -1)[:, :, 8:].unflatten(2, (heads, d))
    before, want = fused.clone(), pamm.rotary(x, table, rotated=3, interleaved=interleaved)
    pamm.rotary(x, table, rotated=3, interleaved=interleaved, out=x)
    assert torch.equal(x, want) and torch.equal(fused[:, :8], before[:, :8])
    # tokens without a batch; positions of every second entry, shared by the sequences
    flat = x.reshape(batch * seq, heads, d)
    assert torch.equal(pamm.rotary(flat[:seq], table, interleaved=interleaved), pamm.rotary(x[:1], table, interleaved=interleaved)[0])
    many = torch.arange(60, device="cuda")
    assert torch.equal(pamm.rotary(x, table, many[10:10 + 2 * seq:2], interleaved=interleaved),
                       pamm.rotary(x, table, many[10:10 + 2 * seq:2].expand(batch, -1).contiguous(), interleaved=interleaved))


@pytest.mark.parametrize("interleaved", [False, True])
def test_turning_back_and_relative_positions(interleaved):
    x = normal((1, 40, 3, 64), F32, 1)
    table = table_of(64)
    there = pamm.rotary(x, table, interleaved=interleaved)
    back = pamm.rotary(there, table, interleaved=interleaved, transposed=True)
    size = x.double().abs().max()
    assert float((back - x).abs().max()) <= 20 * plain64.U * float(size)
    # <q at p, k at p - 3> depends on the distance alone
    q, k = normal((64,), F32, 2).expand(1, 40, 1, 64), normal((64,), F32, 3).expand(1, 40, 1, 64)
    a, b = pamm.rotary(q, table, interleaved=interleaved).double(), pamm.rotary(k, table, interleaved=interleaved).double()
    dots = (a[0, 3:, 0] * b[0, :-3, 0]).sum(-1)
    room = 64 * 10 * plain64.U * float(q.double().abs().max() * k.double().abs().max())
    assert float((dots - dots[0]).abs().max()) <= room


def test_gradient_against_the_formula_and_differences():
    """The turn is linear, so that one difference is exact: <dy, R (x + v)> - <dy, R x> = <R^T dy, v>."""
    table = table_of(32, **dict(scaling=pamm.ROTARY_PARTS, factor=4.0, trained_length=16))
    x, v, dy = (normal((2, 8, 3, 48), F32, s) for s in (1, 2, 3))
    where = torch.arange(8, device="cuda").expand(2, -1)
    for interleaved in (False, True):
        dx = pamm.rotary(dy, table, rotated=2, interleaved=interleaved, transposed=True)
        rows = table[where]
        turn = [plain64.rotary(t.double(), rows[..., :16], rows[..., 16:], 2, 32, interleaved, False)[0] for t in (x.double() + v.double(), x)]
        slope = float((dy.double() * (turn[0] - turn[1])).sum())
        want = float((dx.double() * v.double()).sum())
        assert abs(slope - want) <= 6 * plain64.U * float((dx.double() * v.double()).abs().sum() * 2)


@pytest.mark.parametrize("rot", [2, 20, 128, 512])
def test_table_against_64_bits(rot):
    for first, length, base in ((0, 70, 10000.0), (1_000_000, 33, 500000.0), (2 ** 33, 5, 1e6)):
        freq, amplitude = pamm.rotary_frequencies(rot, base)
        want = np.array(plain64.rotary_frequencies(rot, base))
        assert amplitude == 1.0 and np.allclose(freq.numpy(), want, rtol=1e-14, atol=0)
        table = pamm.rotary_table(length, freq, first=first).cpu().double().numpy()
        angle = (first + np.arange(length, dtype=np.float64))[:, None] * freq.numpy()
        # one rounding to fp32, and the angle's own in 64 bits
        room = 2.0 ** -25 + angle.max() * 2.0 ** -52 + 1e-15
        assert np.abs(table[:, :rot // 2] - np.cos(angle)).max() <= room
        assert np.abs(table[:, rot // 2:] - np.sin(angle)).max() <= room


def test_a_position_outside_the_table_is_reported_and_passes_through():
    table = table_of(64, 16)
    x = normal((1, 5, 2, 64), BF16, 1)
    pos = torch.tensor([[0, 16, 3, -1, 2 ** 40]], device="cuda")
    assert pamm.last_device_status() == pamm.OK
    for interleaved in (False, True):
        got = pamm.rotary(x, table, pos, interleaved=interleaved)
        assert pamm.last_device_status() == pamm.ERR_BAD_INDEX and pamm.last_device_status() == pamm.OK
        assert torch.equal(got[:, [1, 3, 4]], x[:, [1, 3, 4]])
        fine = pamm.rotary(x[:, [0, 2]], table, torch.tensor([[0, 3]], device="cuda"), interleaved=interleaved)
        assert torch.equal(got[:, [0, 2]], fine)


def test_empty_calls():
    table = table_of(8)
    for shape in ((0, 4, 2, 8), (2, 0, 2, 8), (2, 4, 0, 8)):
        assert pamm.rotary(torch.empty(shape, device="cuda"), table).shape == shape
    assert pamm.rotary_table(0, pamm.rotary_frequencies(8)[0]).shape == (0, 8)


def test_offsets_beyond_32_bits():
    d, far = 64, 2 ** 30 + 8
    table = table_of(d, 2000)
    room = torch.zeros(2 * far + 2 * d, dtype=BF16, device="cuda")
    x = torch.as_strided(room, (3, 2, d), (far, d, 1))
    near = normal((3, 2, d), BF16, 1)
    x.copy_(near)
    pamm.rotary(x, table, out=x)
    assert torch.equal(x, pamm.rotary(near, table))
    # a table of more than 2^31 entries
    big = torch.empty((2 ** 25 + 3, d), dtype=F32, device="cuda")
    assert big.numel() > 2 ** 31
    pamm.rotary_table(2 ** 25 + 3, pamm.rotary_frequencies(d)[0], out=big)
    last = torch.full((3,), 2 ** 25 + 2, device="cuda")
    small = pamm.rotary_table(1, pamm.rotary_frequencies(d)[0], first=2 ** 25 + 2)
    assert torch.equal(big[-1:], small)
    assert torch.equal(pamm.rotary(near, big, last), pamm.rotary(near, small, torch.zeros(3, dtype=torch.int32, device="cuda")))


def test_on_another_stream_in_a_graph_and_prepared():
    table, x = table_of(64), normal((2, 16, 6, 64), BF16, 1)
    want = pamm.rotary(x, table, rotated=4)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = pamm.rotary(x, table, rotated=4, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = pamm.rotary(x, table, rotated=4)
    got.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    out = torch.zeros_like(x)
    pamm.prepared(pamm.rotary, x, table, rotated=4, out=out)()
    assert torch.equal(out, want)


def test_scaled_amplitude():
    freq, amplitude = pamm.rotary_frequencies(64, scaling=pamm.ROTARY_PARTS, factor=8.0, trained_length=2048)
    assert abs(amplitude - (0.1 * math.log(8.0) + 1)) < 1e-15
    table = pamm.rotary_table(4, freq, amplitude)
    assert torch.allclose(table[0, :32], torch.tensor(amplitude, dtype=F32, device="cuda"), rtol=1e-7, atol=0) and not table[0, 32:].any()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("heads,rotated", [(1, 1), (1, 0), (2, 1)])
def test_heads_of_the_largest_size_element_by_element(heads, rotated, interleaved, dtype):
    d = 2 ** 24 // heads
    table = pamm.rotary_table(3, *pamm.rotary_frequencies(2))
    x = torch.randn((heads * d + 1,), device="cuda").to(dtype)[1:].view(1, heads, d)           # off every wider grid
    got = pamm.rotary(x, table, rotated=rotated, interleaved=interleaved, first=2)
    assert torch.equal(got[..., 2:], x[..., 2:]) and torch.equal(got[:, rotated:], x[:, rotated:])
    want = pamm.rotary(x[..., :2].contiguous(), table, rotated=rotated, interleaved=interleaved, first=2)
    assert torch.equal(got[..., :2], want)
