"""Dropout from a counter-based generator: the mask word by word, the values element by element."""
import math

import numpy as np
import pytest
import torch

from paper_2506_02939_b200 import build as pamm_build

pamm_build.build()
from paper_2506_02939_b200 import pamm  # noqa: E402
from tests import attention64  # noqa: E402

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def normal(shape, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def statement(x, p, seed, offset, r=None):
    kept = torch.from_numpy(attention64.words(x.numel(), seed, offset) >= math.floor(p * 2 ** 32)).view(x.shape)
    y = torch.where(kept, x.detach().cpu().double() / (1.0 - p) if p < 1 else torch.zeros(x.shape, dtype=torch.float64), 0.0)
    return y if r is None else y + r.detach().cpu().double(), y


def check(got, x, p, seed, offset, r=None):
    want, y = statement(x, p, seed, offset, r)
    half = torch.finfo(x.dtype).eps / 2
    # the factor is rounded, the product, the sum, and the sum to its type
    err = 2 * 2.0 ** -24 * y.abs() + 2.0 ** -24 * want.abs()
    bound = err + half * (want.abs() + err) + 1e-37
    off = (got.detach().cpu().double() - want).abs()
    assert (off <= bound).all()
    if r is None:
        assert torch.equal(got.cpu() == 0, want == 0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("shape", [(1,), (3,), (4,), (5, 8), (7, 9), (2, 3, 31), (1, 4099), (33, 64), (64, 33)])
def test_shapes(shape, residual, dtype):
    x = normal(shape, dtype, 1)
    r = normal(shape, dtype, 2) if residual else None
    for p, seed, offset in ((0.1, 7, 0), (0.5, 2 ** 63 + 5, 2 ** 33 + 1), (0.0, 1, 2), (1.0, 1, 2), (1e-12, 3, 4)):
        check(pamm.dropout(x, p, seed, offset, residual=r), x, p, seed, offset, r)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_strided_rows_and_alignments(dtype):
    for rows, n, ld, shift in ((5, 24, 32, 0), (5, 24, 25, 0), (6, 7, 9, 1), (3, 64, 64, 1), (4, 16, 24, 8)):
        wide = normal((rows * ld + shift,), dtype, 3)
        x = wide[shift:].view(rows, ld)[:, :n]
        r = normal((rows, n), dtype, 4)
        out = torch.full((rows, ld), math.nan, dtype=dtype, device="cuda")
        got = pamm.dropout(x, 0.3, 11, 5, residual=r, Y=out[:, :n])
        check(got, x, 0.3, 11, 5, r)
        assert torch.isnan(out[:, n:]).all()
        check(pamm.dropout(x, 0.3, 11, 5), x, 0.3, 11, 5)


def test_in_place_and_dropped_places():
    for dtype in (F32, BF16):
        x = normal((50, 40), dtype, 5)
        r = normal((50, 40), dtype, 6)
        want = pamm.dropout(x, 0.4, 1, 2, residual=r)
        a, b = x.clone(), r.clone()
        assert torch.equal(pamm.dropout(a, 0.4, 1, 2, residual=r, Y=a), want) and torch.equal(pamm.dropout(x, 0.4, 1, 2, residual=b, Y=b), want)
        dropped = pamm.dropout(torch.ones_like(x), 0.4, 1, 2) == 0
        bad = x.masked_fill(dropped, math.nan)                # a dropped place is zero, whatever it held
        assert torch.equal(pamm.dropout(bad, 0.4, 1, 2, residual=r), want)
        assert not torch.isfinite(pamm.dropout(torch.full_like(x, math.inf), 0.4, 1, 2)[~dropped]).any()


def test_mask_statistics_and_independence():
    n = 1 << 22
    x = torch.ones(n, dtype=BF16, device="cuda")
    masks = [pamm.dropout(x, 0.25, seed, offset) == 0 for seed, offset in ((1, 0), (1, 1), (2, 0))]
    for m in masks:
        assert abs(float(m.float().mean()) - 0.25) < 5 * math.sqrt(0.25 * 0.75 / n)
    for i in range(3):
        for j in range(i):
            both = float((masks[i] & masks[j]).float().mean())
            assert abs(both - 0.0625) < 5 * math.sqrt(0.0625 * 0.9375 / n)


def test_counter_and_graphs():
    x, r = normal((33, 70), BF16, 7), normal((33, 70), BF16, 8)
    counter = torch.tensor([3], device="cuda")
    assert torch.equal(pamm.dropout(x, 0.2, 9, 10, counter=counter, residual=r), pamm.dropout(x, 0.2, 9, 13, residual=r))
    counter.fill_(-1)                                         # modulo 2^64
    assert torch.equal(pamm.dropout(x, 0.2, 9, 10, counter=counter), pamm.dropout(x, 0.2, 9, 9))
    counter.zero_()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y = pamm.dropout(x, 0.2, 9, 100, counter=counter, residual=r)
        counter += 1
    for i in range(3):
        g.replay()
        assert torch.equal(y, pamm.dropout(x, 0.2, 9, 100 + i, residual=r))
    out = torch.zeros_like(x)
    call = pamm.prepared(pamm.dropout, x, 0.2, 9, 100, residual=r, Y=out)
    call()
    assert torch.equal(out, pamm.dropout(x, 0.2, 9, 100, residual=r))


def test_elements_beyond_32_bits():
    """The last elements of more than 2^32 have blocks of their own."""
    n = (1 << 32) + 64
    x = torch.ones(n, dtype=BF16, device="cuda")
    tail = pamm.dropout(x, 0.5, 21, 1)[-64:].cpu()
    words = []
    for block in range((n - 64) // 4, n // 4):
        c, k = [block & 0xFFFFFFFF, block >> 32, 1, 0], [21, 0]
        for _ in range(10):
            a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
            c = [b >> 32 ^ c[1] ^ k[0], b & 0xFFFFFFFF, a >> 32 ^ c[3] ^ k[1], a & 0xFFFFFFFF]
            k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
        words += c
    assert np.array_equal(tail.float().numpy() != 0, np.array(words) >= 2 ** 31)


def test_empty_and_refusals():
    x = normal((4, 8), F32, 9)
    assert pamm.dropout(x[:0], 0.1, 1).shape == (0, 8)
    for error, call in [(pamm.PammError, lambda: pamm.dropout(x, -0.1, 1)), (pamm.PammError, lambda: pamm.dropout(x, 1.1, 1)),
                        (pamm.PammError, lambda: pamm.dropout(x, math.nan, 1)), (ValueError, lambda: pamm.dropout(x, 0.1, 1, residual=x[:2])),
                        (TypeError, lambda: pamm.dropout(x, 0.1, 1, residual=x.bfloat16())), (ValueError, lambda: pamm.dropout(x.t(), 0.1, 1)),
                        (ValueError, lambda: pamm.dropout(x.cpu(), 0.1, 1)), (TypeError, lambda: pamm.dropout(x.half(), 0.1, 1)),
                        (OverflowError, lambda: pamm.dropout(x, 0.1, 2 ** 64)), (OverflowError, lambda: pamm.dropout(x, 0.1, 1, -1)),
                        (ValueError, lambda: pamm.dropout(x, 0.1, 1, counter=torch.zeros(2, dtype=torch.int64, device="cuda"))),
                        (ValueError, lambda: pamm.dropout(x, 0.1, 1, counter=torch.zeros(1, device="cuda")))]:
        with pytest.raises(error):
            call()
