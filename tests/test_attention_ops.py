"""Host-side checks of attention and dropout: refusals, scratch sizes, and the 64-bit statements the GPU tests compare with.  No GPU is
used."""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2506_02939_b200 import build as pamm_build

pamm_build.build()
from paper_2506_02939_b200 import pamm  # noqa: E402
from tests import attention64  # noqa: E402

FAKE, ODD, NULL = 0x1000, 0x1001, None       # never dereferenced: checks come first
BAD, UNSUP, WS = pamm.ERR_INVALID_ARG, pamm.ERR_UNSUPPORTED, pamm.ERR_WORKSPACE


def heads(data=FAKE, batch=512, token=64, head=8):
    return (ctypes.c_int64 * 4)(data or 0, batch, token, head)


def call(back=False, tensors=None, lse=FAKE, batch=2, seq=4, h=4, kv=2, d=8, dt=0, scale=1.0, lengths=NULL, starts=NULL, sequences=0, index=0,
         ws=FAKE, size=1 << 20, missing=None, **other):
    names = ("dO", "Q", "K", "V", "O") + ("dQ", "dK", "dV") if back else ("Q", "K", "V", "O")
    t = [heads(**other.get(n, {})) for n in names]
    a = [None if n == missing else ctypes.addressof(x) for n, x in zip(names, t)]
    sizes = (batch, seq, h, kv, d, dt, scale, 0, lengths, starts, sequences, index)
    if back:
        return pamm._lib.pamm_attention_backward(*a[:5], lse, *a[5:], *sizes, ws, size, None)
    return pamm._lib.pamm_attention_forward(*a, lse, *sizes, None)


@pytest.mark.parametrize("back", [False, True])
def test_attention_refusals(back):
    cases = [(dict(batch=-1), BAD), (dict(seq=-1), BAD), (dict(h=-1), BAD), (dict(kv=0), BAD), (dict(kv=3), BAD), (dict(kv=8), BAD), (dict(d=0), BAD),
             (dict(d=257), UNSUP), (dict(dt=2), UNSUP), (dict(scale=0.0), BAD), (dict(scale=-1.0), BAD), (dict(scale=math.nan), BAD),
             (dict(scale=math.inf), BAD), (dict(lse=FAKE + 2), BAD), (dict(lengths=FAKE, starts=FAKE, batch=1), BAD), (dict(lengths=FAKE + 2), BAD),
             (dict(lengths=FAKE + 4, index=1), BAD), (dict(lengths=FAKE, index=2), UNSUP), (dict(starts=FAKE, batch=2), BAD),
             (dict(starts=FAKE, batch=1, sequences=-1), BAD), (dict(starts=FAKE + 2, batch=1, sequences=1), BAD), (dict(batch=1 << 31), UNSUP),
             (dict(seq=1 << 31), UNSUP), (dict(batch=1 << 20, seq=1 << 20), UNSUP), (dict(batch=1 << 26, seq=1, h=64, kv=64), UNSUP),
             (dict(starts=FAKE, batch=1, sequences=(1 << 31) - 1), UNSUP), (dict(missing="Q"), BAD), (dict(Q=dict(data=0)), BAD), (dict(K=dict(data=ODD)), BAD),
             (dict(O=dict(data=ODD)), BAD)]
    if back:
        cases += [(dict(lse=NULL), BAD), (dict(ws=NULL), WS), (dict(ws=FAKE + 8), WS), (dict(size=16), WS), (dict(missing="dV"), BAD), (dict(dQ=dict(token=0)), BAD),
                  (dict(dK=dict(head=0)), BAD), (dict(dV=dict(batch=0)), BAD), (dict(dO=dict(data=0)), BAD)]
    else:
        cases += [(dict(O=dict(token=0)), BAD), (dict(O=dict(head=0)), BAD), (dict(O=dict(batch=0)), BAD)]
    for kw, code in cases:
        assert call(back, **kw) == code, kw
    for kw in (dict(batch=0), dict(seq=0), dict(h=0, kv=0)):
        assert call(back, **kw, Q=dict(data=0), ws=NULL) == pamm.OK


@pytest.mark.parametrize("back", [False, True])
def test_outputs_that_begin_where_another_tensor_does(back):
    apart = {n: dict(data=FAKE * (i + 2)) for i, n in enumerate(("dO", "Q", "K", "V", "O", "dQ", "dK", "dV"))}
    for one in ("dQ", "dK", "dV") if back else ("O",):
        for other in ("dO", "Q", "K", "V", "O", "dQ", "dK", "dV") if back else ("Q", "K", "V"):
            if one != other:
                assert call(back, **{**apart, one: apart[other]}) == BAD, (one, other)
        assert call(back, **{**apart, one: dict(data=FAKE)}) == BAD, one             # the log-sums, and the workspace


def test_dropout_refusals():
    def call(X=FAKE, ldx=8, R=NULL, ldr=0, b=4, n=8, dt=0, p=0.5, seed=1, offset=2, counter=NULL, Y=FAKE + 4096, ldy=8):
        return pamm._lib.pamm_dropout(X, ldx, R, ldr, b, n, dt, p, seed, offset, counter, Y, ldy, None)

    for kw, code in [(dict(X=NULL), BAD), (dict(Y=NULL), BAD), (dict(X=ODD), BAD), (dict(Y=ODD), BAD), (dict(R=ODD, ldr=8), BAD), (dict(ldx=7), BAD), (dict(ldy=7), BAD),
                     (dict(R=FAKE, ldr=7), BAD), (dict(b=-1), BAD), (dict(n=-1), BAD), (dict(dt=2), UNSUP), (dict(p=-0.1), BAD), (dict(p=1.5), BAD),
                     (dict(p=math.nan), BAD), (dict(counter=FAKE + 4), BAD), (dict(Y=FAKE, ldy=16), BAD), (dict(R=FAKE + 4096, ldr=16), BAD),
                     (dict(b=1 << 30, n=1 << 30, ldx=1 << 30, ldy=1 << 30), UNSUP)]:
        assert call(**kw) == code, kw
    assert call(b=0, X=NULL, Y=NULL) == pamm.OK and call(n=0, X=NULL, Y=NULL) == pamm.OK


def test_scratch_size():
    w = pamm.workspace_bytes(pamm.WS_ATTENTION_BACKWARD, 65536, 16, 1, 1, pamm.BF16)
    assert w >= 65536 * 16 * 4 and w % 256 == 0
    assert pamm.workspace_bytes(pamm.WS_ATTENTION_BACKWARD, 0, 0, 1, 1, pamm.F32) > 0
    for b, n in ((-1, 8), (4, -1), (1 << 40, 1 << 40)):
        with pytest.raises(pamm.PammError):
            pamm.workspace_bytes(pamm.WS_ATTENTION_BACKWARD, b, n, 1, 1, pamm.F32)


def test_python_refusals_without_a_device():
    x = torch.zeros((2, 3, 4, 8))
    for call in (lambda: pamm.attention_forward(x, x, x), lambda: pamm.attention_backward(x, x, x, x, x, x), lambda: pamm.dropout(x, 0.5, 1)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        pamm.dropout(x.half(), 0.5, 1)
    from paper_2506_02939_b200.autograd import Dropout, attention, dropout
    with pytest.raises(ValueError):
        Dropout(1.5)
    for kv in (0, 2, 5):
        with pytest.raises(ValueError):
            attention(x, kv)
    with pytest.raises(ValueError):
        dropout(x, 0.5, 1, residual=x[:1])


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("lengths,starts", [(None, None), ([5, 0], None), (None, [1, 3, 3, 6])])
def test_the_64_bit_gradient_against_differences(causal, lengths, starts):
    g = torch.Generator().manual_seed(1)
    tokens, d, scale = ((7,) if starts else (2, 6)), 4, 0.7
    Q, dO, v = (torch.randn((*tokens, 4, d), generator=g, dtype=torch.float64) for _ in range(3))
    K, V, vk, vv = (torch.randn((*tokens, 2, d), generator=g, dtype=torch.float64) for _ in range(4))
    O, lse, _, _ = attention64.forward(Q, K, V, causal, lengths, starts, scale)
    (dQ, dK, dV), _ = attention64.backward(dO, Q, K, V, O, lse.masked_fill(lse == -math.inf, 0.0), causal, lengths, starts, scale)

    def loss(q, k, w):
        return float((attention64.forward(q, k, w, causal, lengths, starts, scale)[0] * dO).sum())

    t = 1e-5
    assert abs((loss(Q + t * v, K, V) - loss(Q - t * v, K, V)) / (2 * t) - float((dQ * v).sum())) < 1e-6
    assert abs((loss(Q, K + t * vk, V) - loss(Q, K - t * vk, V)) / (2 * t) - float((dK * vk).sum())) < 1e-6
    assert abs((loss(Q, K, V + t * vv) - loss(Q, K, V - t * vv)) / (2 * t) - float((dV * vv).sum())) < 1e-6


def test_the_generator_by_hand():
    """Word 0 for counter and key zero, and for all ones, are the published known answers of the ten-round generator."""
    assert [int(w) for w in attention64.words(4, 0, 0)] == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    w = attention64.words(1 << 12, 12345, 6789)
    assert w.dtype == np.uint64 and len(set(w.tolist())) > 4000 and abs(float(w.mean()) / 2 ** 32 - 0.5) < 0.02
