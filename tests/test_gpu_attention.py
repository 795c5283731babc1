"""Attention, forward and backward, against 64-bit statements, element by element."""
import math

import pytest
import torch

from paper_2506_02939_b200 import build as pamm_build

pamm_build.build()
from paper_2506_02939_b200 import pamm  # noqa: E402
from tests import attention64  # noqa: E402

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def normal(shape, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def parts(tokens, heads, kv, d, dtype, seed, scale=1.5):
    return normal((*tokens, heads + 2 * kv, d), dtype, seed, scale).split((heads, kv, kv), -2)


def index(values, dtype=torch.int32):
    return None if values is None else torch.tensor(values, dtype=dtype, device="cuda")


def check(Q, K, V, causal, lengths=None, starts=None, scale=None, dO=None, index_type=torch.int32, outputs=None, clean=None):
    """Forward and backward against the statement; ``clean``: the inputs without what lies in rows that no sequence has."""
    how = dict(causal=causal, lengths=index(lengths, index_type), starts=index(starts, index_type), scale=scale)
    rounded = Q.dtype == BF16
    dO = normal(Q.shape, Q.dtype, 99, 0.1) if dO is None else dO
    given = outputs or {}
    O, lse = pamm.attention_forward(Q, K, V, **how, **{k: v for k, v in given.items() if k in ("O", "lse")})
    q, k, v, do = (Q, K, V, dO) if clean is None else clean
    wO, wL, eO, eL = attention64.forward(q, k, v, causal, lengths, starts, scale, rounded)
    assert attention64.share(O, wO, eO) <= 1.0
    assert attention64.share(lse, wL, eL) <= 1.0
    grads = pamm.attention_backward(dO, Q, K, V, O, lse, **how, **{k: v for k, v in given.items() if k in ("dQ", "dK", "dV")})
    want, err = attention64.backward(do, q, k, v, O, lse.masked_fill(lse == -math.inf, 0.0), causal, lengths, starts, scale, rounded)
    for got, w, e in zip(grads, want, err):
        assert attention64.share(got, w, e) <= 1.0
    assert pamm.last_device_status() == pamm.OK
    return (O, lse, *grads)


SIZES = [(1, 1, 1, 1, 64), (2, 2, 2, 1, 128), (3, 17, 4, 2, 64), (1, 63, 2, 2, 128), (2, 64, 3, 1, 64), (1, 65, 2, 1, 80), (1, 127, 1, 1, 128), (2, 128, 2, 2, 128),
         (1, 129, 6, 2, 40), (1, 200, 2, 1, 96), (1, 255, 1, 1, 64), (1, 256, 2, 1, 128), (2, 257, 2, 2, 128), (1, 300, 5, 5, 8), (1, 385, 4, 1, 128),
         (1, 513, 2, 1, 64), (1, 700, 1, 1, 128), (70, 3, 2, 1, 16)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("batch,seq,heads,kv,d", SIZES)
def test_sizes(batch, seq, heads, kv, d, causal, dtype):
    check(*parts((batch, seq), heads, kv, d, dtype, seq + d), causal)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("d", [1, 2, 7, 20, 33, 72, 100, 136, 160, 200, 256])
def test_head_widths(d, dtype):
    check(*parts((2, 70), 2, 1, d, dtype, d), True)
    check(*parts((1, 130), 1, 1, d, dtype, d), False)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d", [64, 128, 20])
def test_padded_rows_with_anything_in_them(d, causal, dtype):
    batch, seq, heads, kv = 7, 300, 4, 2
    lengths = [0, 1, 64, 128, 129, 299, 300]
    Q, K, V = parts((batch, seq), heads, kv, d, dtype, 3)
    dO = normal(Q.shape, dtype, 4, 0.1)
    clean = [t.clone() for t in (Q, K, V, dO)]
    for t, junk in ((Q, math.nan), (K, math.inf), (V, math.nan), (dO, -math.inf)):
        for b, n in enumerate(lengths):
            t[b, n:] = junk
    for c in clean:
        for b, n in enumerate(lengths):
            c[b, n:] = 0.0
    outputs = {k: torch.full(s, math.nan, dtype=t, device="cuda") for k, s, t in (
        ("O", Q.shape, dtype), ("lse", (batch, heads, seq), F32), ("dQ", Q.shape, dtype), ("dK", K.shape, dtype), ("dV", V.shape, dtype))}
    O, lse, dQ, dK, dV = check(Q, K, V, causal, lengths=lengths, dO=dO, outputs=outputs, clean=clean, index_type=torch.int64)
    for b, n in enumerate(lengths):
        assert (lse[b, :, n:] == -math.inf).all()
        for t in (O, dQ, dK, dV):
            assert (t[b, n:] == 0).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("starts", [[0, 5], [3, 3, 4, 4, 70, 198, 330, 341], [0], [0] * 40 + [1, 2, 3, 130, 259, 259], [0, 128, 256, 384], [7, 300, 300, 301],
                                    list(range(0, 401, 8)), [0, 255, 256, 512]])
def test_packed_sequences(starts, causal, dtype):
    tokens, heads, kv, d = starts[-1] + 9, 4, 2, 64
    Q, K, V = parts((tokens,), heads, kv, d, dtype, 5)
    dO = normal(Q.shape, dtype, 6, 0.1)
    clean = [t.clone() for t in (Q, K, V, dO)]
    for t in (Q, K, V, dO):
        t[:starts[0]] = math.nan
        t[starts[-1]:] = math.nan
    for c in clean:
        c[:starts[0]] = 0.0
        c[starts[-1]:] = 0.0
    O, lse, dQ, dK, dV = check(Q, K, V, causal, starts=starts, dO=dO, clean=clean)
    for t in (O, dQ, dK, dV):
        assert (t[:starts[0]] == 0).all() and (t[starts[-1]:] == 0).all()


def test_a_neighbour_with_nan_stays_a_neighbour():
    """Packed sequences share tiles: what one of them holds reaches no other."""
    starts, d = [0, 40, 90, 300], 64
    for dtype in (BF16, F32):
        Q, K, V = parts((300,), 2, 1, d, dtype, 7)
        for t in (Q, K, V):
            t[40:90] = math.nan
        O, lse = pamm.attention_forward(Q, K, V, starts=index(starts))
        dQ, dK, dV = pamm.attention_backward(torch.ones_like(O), Q, K, V, O, lse, starts=index(starts))
        for t in (O, dQ, dK, dV):
            assert torch.isfinite(t[:40]).all() and torch.isfinite(t[90:]).all() and torch.isnan(t[40:90]).any()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("d", [64, 128])
def test_orders_strides_and_alignments(d, dtype):
    batch, seq, heads, kv = 2, 150, 4, 2

    def by_head(t):                                          # memory by head, then token
        return t.transpose(1, 2).contiguous().transpose(1, 2)

    def shifted(t, by):                                      # rows off the 16-byte grid
        flat = torch.zeros(t.numel() + by, dtype=t.dtype, device="cuda")
        flat[by:] = t.flatten()
        return flat[by:].view(t.shape)

    def spaced(t):                                           # rows further apart
        wide = torch.full((*t.shape[:-1], d + 8), math.nan, dtype=t.dtype, device="cuda")
        wide[..., :d] = t
        return wide[..., :d]

    Q, K, V = (t.contiguous() for t in parts((batch, seq), heads, kv, d, dtype, 8))
    dO = normal(Q.shape, dtype, 9, 0.1)
    plain = check(Q, K, V, True, dO=dO)
    for form in (by_head, spaced, lambda t: shifted(t, 1), lambda t: shifted(t, 8), lambda t: t.transpose(0, 1).contiguous().transpose(0, 1)):
        outputs = dict(O=form(torch.zeros_like(Q)), dQ=form(torch.zeros_like(Q)), dK=form(torch.zeros_like(K)), dV=form(torch.zeros_like(V)))
        got = check(form(Q), form(K), form(V), True, dO=form(dO), outputs=outputs)
        assert got[0].data_ptr() == outputs["O"].data_ptr()
        if dtype == F32:                                     # one way of computing, whatever the order in memory
            for a, b in zip(got, plain):
                assert torch.equal(a, b)
    # one key and value for all heads and sequences, by strides of zero
    k1, v1 = K[:1, :, :1].expand(batch, seq, heads, d), V[:1, :, :1].expand(batch, seq, heads, d)
    check(Q, k1, v1, False, dO=dO[:, :, :1].expand(Q.shape))


def test_offsets_beyond_32_bits():
    token = 1 << 24                                          # elements from token to token: 300 of them pass 2^32
    memory = torch.empty(260 * token, dtype=BF16, device="cuda")
    Z = memory.as_strided((260, 3, 64), (token, 64, 1))
    Z.copy_(normal((260, 3, 64), BF16, 10))
    small = Z.contiguous()
    out = memory.as_strided((260, 1, 64), (token, 64, 1), 1024)
    outs = [memory.as_strided((260, 1, 64), (token, 64, 1), 2048 + 64 * i) for i in range(3)]
    O, lse = pamm.attention_forward(*Z.split(1, -2), causal=True, O=out)
    o2, l2 = pamm.attention_forward(*small.split(1, -2), causal=True)
    assert torch.equal(O, o2) and torch.equal(lse, l2)
    dO = normal(o2.shape, BF16, 11)
    got = pamm.attention_backward(dO, *Z.split(1, -2), O, lse, causal=True, dQ=outs[0], dK=outs[1], dV=outs[2])
    for a, b in zip(got, pamm.attention_backward(dO, *small.split(1, -2), o2, l2, causal=True)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_scores_of_every_size(dtype):
    """Large scores, one key that takes everything, equal scores, a given scale."""
    Q, K, V = parts((1, 200), 2, 1, 64, dtype, 12, 6.0)
    check(Q, K, V, True)
    Q, K, V = parts((1, 200), 2, 1, 64, dtype, 13)
    K[:, 100] *= 40.0
    check(Q, K, V, False)
    check(torch.zeros_like(Q), K, V, True)
    check(Q, K, V, True, scale=0.01)
    check(Q, K, V, False, scale=3.0)
    grow = torch.linspace(0, 30, 200, device="cuda").to(dtype).view(1, 200, 1, 1)          # the running maximum rises in every tile
    check(torch.ones_like(Q) * 4, (grow * torch.ones_like(K)) / 8, V, False)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_repeats_are_equal_to_the_bit(dtype):
    Q, K, V = parts((3, 600), 6, 2, 128, dtype, 14)
    dO = normal(Q.shape, dtype, 15)
    first = None
    for _ in range(3):
        O, lse = pamm.attention_forward(Q, K, V, causal=True)
        now = (O, lse, *pamm.attention_backward(dO, Q, K, V, O, lse, causal=True))
        assert first is None or all(torch.equal(a, b) for a, b in zip(now, first))
        first = now


def test_bad_entries_are_reported_and_stay_in_bounds():
    Q, K, V = parts((4, 150), 2, 1, 64, BF16, 16)
    want, _ = pamm.attention_forward(Q, K, V, lengths=index([0, 150, 150, 20]))
    assert pamm.last_device_status() == pamm.OK
    O, lse = pamm.attention_forward(Q, K, V, lengths=index([-5, 151, 2 ** 31 - 1, 20]))
    assert pamm.last_device_status() == pamm.ERR_BAD_INDEX and torch.equal(O, want)
    pamm.attention_backward(O, Q, K, V, O, lse, lengths=index([-5, 151, 2 ** 31 - 1, 20]))
    assert pamm.last_device_status() == pamm.ERR_BAD_INDEX
    Q, K, V = parts((150,), 2, 1, 64, BF16, 17)
    for starts in ([0, 100, 50, 150], [-7, 20, 400], [150, 0], [2 ** 40, -2 ** 40]):
        O, lse = pamm.attention_forward(Q, K, V, starts=index(starts, torch.int64))
        assert pamm.last_device_status() == pamm.ERR_BAD_INDEX
        pamm.attention_backward(O, Q, K, V, O, lse, starts=index(starts, torch.int64))
        assert pamm.last_device_status() == pamm.ERR_BAD_INDEX


def test_empty_calls():
    for shape, kv in (((0, 5, 2, 64), 1), ((3, 0, 2, 64), 1), ((0, 2, 64), 1)):
        Q = torch.zeros(shape, dtype=BF16, device="cuda")
        K = torch.zeros((*shape[:-2], kv, 64), dtype=BF16, device="cuda")
        O, lse = pamm.attention_forward(Q, K, K)
        assert O.shape == Q.shape and lse.numel() == 0
        assert [t.shape for t in pamm.attention_backward(O, Q, K, K, O, lse)] == [Q.shape, K.shape, K.shape]


def test_streams_graphs_and_prepared_calls():
    Q, K, V = parts((2, 300), 4, 2, 128, BF16, 18)
    dO = normal(Q.shape, BF16, 19)
    O, lse = pamm.attention_forward(Q, K, V, causal=True)
    grads = pamm.attention_backward(dO, Q, K, V, O, lse, causal=True)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    o2, l2 = pamm.attention_forward(Q, K, V, causal=True, stream=side)
    g2 = pamm.attention_backward(dO, Q, K, V, o2, l2, causal=True, stream=side)
    side.synchronize()
    assert torch.equal(O, o2) and all(torch.equal(a, b) for a, b in zip(grads, g2))
    # two graphs in flight at once: each has its own workspace
    graphs, outs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            o, l = pamm.attention_forward(Q, K, V, causal=True)
            outs.append((o, l, *pamm.attention_backward(dO, Q, K, V, o, l, causal=True)))
        graphs.append(g)
    for _ in range(3):
        for g, s in zip(graphs, (side, torch.cuda.Stream())):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for out in outs:
        assert all(torch.equal(a, b) for a, b in zip(out, (O, lse, *grads)))
    o3, l3 = torch.zeros_like(O), torch.zeros_like(lse)
    call = pamm.prepared(pamm.attention_forward, Q, K, V, causal=True, O=o3, lse=l3)
    g3 = [torch.zeros_like(t) for t in grads]
    back = pamm.prepared(pamm.attention_backward, dO, Q, K, V, o3, l3, causal=True, dQ=g3[0], dK=g3[1], dV=g3[2])
    for _ in range(2):
        call()
        back()
    assert torch.equal(o3, O) and torch.equal(l3, lse) and all(torch.equal(a, b) for a, b in zip(g3, grads))


def test_python_refusals():
    Q, K, V = parts((2, 20), 4, 2, 64, BF16, 20)
    O, lse = pamm.attention_forward(Q, K, V)
    for error, call in [
            (ValueError, lambda: pamm.attention_forward(Q, K[:, :, :1].expand(2, 20, 3, 64), V)), (ValueError, lambda: pamm.attention_forward(Q, K, V[:, :10])),
            (TypeError, lambda: pamm.attention_forward(Q, K.float(), V)), (TypeError, lambda: pamm.attention_forward(Q.half(), K.half(), V.half())),
            (ValueError, lambda: pamm.attention_forward(Q.cpu(), K, V)), (ValueError, lambda: pamm.attention_forward(Q[0, 0], K[0, 0], V[0, 0])),
            (ValueError, lambda: pamm.attention_forward(Q, K, V, lengths=index([1, 2, 3]))), (TypeError, lambda: pamm.attention_forward(Q, K, V, lengths=torch.ones(2, device="cuda"))),
            (ValueError, lambda: pamm.attention_forward(Q, K, V, lengths=torch.ones(2, dtype=torch.int32))), (ValueError, lambda: pamm.attention_forward(Q, K, V, starts=index([0, 20]))),
            (ValueError, lambda: pamm.attention_forward(Q[0], K[0], V[0], starts=index([0, 20]), lengths=index([5]))),
            (ValueError, lambda: pamm.attention_forward(Q, K, V, O=torch.zeros((2, 20, 1, 64), dtype=BF16, device="cuda").expand(2, 20, 4, 64))),
            (ValueError, lambda: pamm.attention_forward(Q.transpose(2, 3), K.transpose(2, 3), V.transpose(2, 3))), (ValueError, lambda: pamm.attention_backward(O, Q, K, V, O, lse[:1])),
            (ValueError, lambda: pamm.attention_backward(O, Q, K, V, O, lse.transpose(0, 1))), (ValueError, lambda: pamm.attention_backward(O[:, :5], Q, K, V, O, lse)),
            (pamm.PammError, lambda: pamm.attention_forward(Q, K, V, scale=0.0)), (pamm.PammError, lambda: pamm.attention_forward(Q, K, V, scale=math.nan)),
            (pamm.PammError, lambda: pamm.attention_forward(Q, K, V, scale=-1.0)), (pamm.PammError, lambda: pamm.attention_forward(Q, K, V, scale=math.inf)),
            (pamm.PammError, lambda: pamm.attention_forward(*parts((2, 3), 1, 1, 257, BF16, 1))),
            (pamm.PammError, lambda: pamm.attention_backward(O, Q, K, V, O, lse, workspace=torch.empty(16, dtype=torch.uint8, device="cuda")))]:
        with pytest.raises(error):
            call()
    assert torch.equal(pamm.attention_forward(Q, K, V)[0], O)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_many_sequences_without_a_token(causal, d):
    """Blocks meet long runs of tiles with nothing to compute, between short and long ones."""
    batch, seq, heads, kv = 400, 700, 2, 1
    lengths = [(0, 0, 0, 0, 1, 0, 0, 130, 0, 0, 0, 700)[i % 12] for i in range(batch)]
    Q, K, V = parts((batch, seq), heads, kv, d, BF16, 21)
    dO = normal(Q.shape, BF16, 22, 0.1)
    O, lse = pamm.attention_forward(Q, K, V, causal=causal, lengths=index(lengths))
    grads = pamm.attention_backward(dO, Q, K, V, O, lse, causal=causal, lengths=index(lengths))
    assert pamm.last_device_status() == pamm.OK
    some = [i for i, n in enumerate(lengths) if n]
    q, k, v, g = (t[some].contiguous() for t in (Q, K, V, dO))
    few = index([lengths[i] for i in some])
    o, l = pamm.attention_forward(q, k, v, causal=causal, lengths=few)
    for a, b in zip((O, lse, *grads), (o, l, *pamm.attention_backward(g, q, k, v, o, l, causal=causal, lengths=few))):
        assert torch.equal(a[some], b)
    none = [i for i, n in enumerate(lengths) if not n]
    assert not any(t[none].any() for t in (O, *grads)) and (lse[none] == -math.inf).all()
    # packed: short documents, and a tail that belongs to none of them, with many heads
    starts = [0, 1, 2, 3, 140, 141, 900]
    Q, K, V = parts((5000,), 24, 12, d, BF16, 23)
    O, lse = pamm.attention_forward(Q, K, V, causal=causal, starts=index(starts))
    grads = pamm.attention_backward(Q, Q, K, V, O, lse, causal=causal, starts=index(starts))
    assert pamm.last_device_status() == pamm.OK
    o, l = pamm.attention_forward(Q[:900], K[:900], V[:900], causal=causal, starts=index(starts))
    for a, b in zip((O, *grads), (o, *pamm.attention_backward(Q[:900], Q[:900], K[:900], V[:900], o, l, causal=causal, starts=index(starts)))):
        assert torch.equal(a[:900], b) and not a[900:].any()
