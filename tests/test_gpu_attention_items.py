"""Attention on the tensor cores where a block works on many items, and where the running maximum rises, at the wide heads too: against
64-bit statements, element by element."""
import math

import pytest
import torch

from paper_2506_02939_b200 import build as pamm_build

pamm_build.build()
from paper_2506_02939_b200 import pamm  # noqa: E402
from tests import attention64  # noqa: E402
from tests.test_gpu_attention import check, index, normal, parts  # noqa: E402

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_items_of_one_to_six_tiles_behind_each_other(causal, d):
    """Hundreds of items of mixed lengths, more than there are SMs: what a block hands from one to the next.  A sample of the sequences."""
    batch, seq, heads, kv = 40, 700, 8, 2
    lengths = [(700, 1, 129, 0, 640, 257, 128, 384, 65, 511)[(7 * i + i // 10) % 10] for i in range(batch)]
    Q, K, V = parts((batch, seq), heads, kv, d, BF16, 31)
    dO = normal(Q.shape, BF16, 32, 0.1)
    how = dict(causal=causal, lengths=index(lengths))
    O, lse = pamm.attention_forward(Q, K, V, **how)
    grads = pamm.attention_backward(dO, Q, K, V, O, lse, **how)
    assert pamm.last_device_status() == pamm.OK
    some = [0, 5, 13, 14, 22, 27, 31, 36, 38, 39]
    few = [lengths[i] for i in some]
    q, k, v, do, o, l = (t[some] for t in (Q, K, V, dO, O, lse))
    want, wl, e, el = attention64.forward(q, k, v, causal, few, rounded=True)
    assert attention64.share(o, want, e) <= 1.0 and attention64.share(l, wl, el) <= 1.0
    want, err = attention64.backward(do, q, k, v, o, l.masked_fill(l == -math.inf, 0.0), causal, few, rounded=True)
    for got, w, e in zip(grads, want, err):
        assert attention64.share(got[some], w, e) <= 1.0


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_packed_items_of_one_to_six_tiles_behind_each_other(causal, d):
    heads, kv = 8, 2
    starts = [3]
    for i in range(40):
        starts.append(starts[-1] + (700, 1, 129, 0, 640, 257, 128, 384, 65, 511)[(7 * i + i // 10) % 10])
    tokens = starts[-1] + 300
    Q, K, V = parts((tokens,), heads, kv, d, BF16, 33)
    dO = normal(Q.shape, BF16, 34, 0.1)
    how = dict(causal=causal, starts=index(starts))
    O, lse = pamm.attention_forward(Q, K, V, **how)
    grads = pamm.attention_backward(dO, Q, K, V, O, lse, **how)
    assert pamm.last_device_status() == pamm.OK
    for i in (0, 5, 13, 14, 22, 27, 31, 36, 38, 39):
        at = slice(starts[i], starts[i + 1])
        q, k, v, do, o, l = (*(t[at] for t in (Q, K, V, dO, O)), lse[:, at])
        want, wl, e, el = attention64.forward(q, k, v, causal, rounded=True)
        assert attention64.share(o, want, e) <= 1.0 and attention64.share(l, wl, el) <= 1.0
        want, err = attention64.backward(do, q, k, v, o, l, causal, rounded=True)
        for got, w, e in zip(grads, want, err):
            assert attention64.share(got[at], w, e) <= 1.0
    for t in (O, *grads):
        assert not t[:3].any() and not t[starts[-1]:].any()


@pytest.mark.parametrize("d", [40, 72, 96, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_maxima_that_rise_in_every_group_of_keys(causal, d):
    """Scores of up to +-170 that rise along the keys, by more than 2^8 from one 64 keys to the next, in rows of the one sign; in the rows of
    the other sign, between them, they fall."""
    seq, heads, kv = 400, 2, 1
    _, _, V = parts((1, seq), heads, kv, d, BF16, 35)
    sign = (torch.randint(0, 2, (1, seq, heads, 1), generator=torch.Generator(device="cuda").manual_seed(36), device="cuda") * 2 - 1).float()
    up = torch.linspace(0, 170, seq, device="cuda").view(1, seq, 1, 1)
    unit = (torch.arange(d, device="cuda") % 3 + 1.0) / 2
    size = float((unit * unit).sum()) / math.sqrt(d)
    Q, K = (sign * unit).to(BF16), (up / size * unit).to(BF16)
    check(Q, K, V, causal)
    check(Q, K + normal(K.shape, BF16, 37, 0.2), V, causal)
