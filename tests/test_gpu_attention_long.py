"""Attention whose items of work take long: waits that span an item end with it, however long the context or the run of empty
sequences."""
import math

import pytest
import torch

from paper_2506_02939_b200 import build as pamm_build

pamm_build.build()
from paper_2506_02939_b200 import pamm  # noqa: E402
from tests.attention64 import U  # noqa: E402

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def test_a_wait_lasts_as_long_as_there_is_progress():
    assert pamm.last_device_status() == pamm.OK
    pamm.selftest_progress_wait()
    assert pamm.last_device_status() == pamm.OK


def sparse(shape, seed, count):
    """Ones of either sign in `count` random rows of every column, in the first and in the last one too."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    rows, cols = math.prod(shape[:-1]), shape[-1]
    t = torch.zeros((rows, cols), device="cuda")
    at = torch.randint(0, rows, (count, cols), generator=g, device="cuda")
    at[0], at[1] = 0, rows - 1
    t.scatter_(0, at, torch.randint(0, 2, (count, cols), generator=g, device="cuda") * 2.0 - 1.0)
    return t.view(shape).to(BF16)


def test_many_query_heads_over_one_in_a_long_context():
    """A tile of keys meets 1024 tiles of each of 32 heads: 45 ms an item.  With scores of 0 every probability is 2^-17, as a bf16 operand
    exactly, and the sums of a hundred ones are exact whatever their order: a step that is lost shows."""
    tokens, heads, d = 1 << 17, 32, 64
    zero = torch.zeros((tokens, 1, d), dtype=BF16, device="cuda")
    q = torch.randint(-1, 2, (tokens, heads, d), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(BF16)
    V = sparse((tokens, 1, d), 2, 100)
    O, lse = pamm.attention_forward(q, zero, V)
    assert pamm.last_device_status() == pamm.OK
    assert torch.equal(O, (V.double().sum(0, keepdim=True) / tokens).to(BF16).expand_as(O))
    assert ((lse.double() - math.log(tokens)).abs() <= 4 * U * math.log(tokens)).all()
    # values of one and minus one in column 0: O and delta are 0, dS is the gradient's column 0 with the key's sign
    sign = (torch.arange(tokens, device="cuda") % 2 * 2 - 1).to(BF16)
    V = zero.clone()
    V[:, 0, 0] = sign
    dO, K = sparse((tokens, heads, d), 3, 100), sparse((tokens, 1, d), 4, 100)
    first = dO[..., 0].double()
    for Q, k in ((q, zero), (torch.zeros_like(q), K)):
        O, lse = pamm.attention_forward(Q, k, V)
        dQ, dK, dV = pamm.attention_backward(dO, Q, k, V, O, lse)
        assert pamm.last_device_status() == pamm.OK and not O.any()
        assert torch.equal(dV, (dO.double().sum((0, 1)) / tokens).to(BF16).expand_as(dV))
        want = torch.einsum("ih,ihd->d", first, Q.double()) / tokens / 8
        assert torch.equal(dK.double(), (sign.double()[:, None] * want)[:, None])
        want = (sign.double()[:, None] * k[:, 0].double()).sum(0) / tokens / 8
        assert torch.equal(dQ.double(), first[..., None] * want)


def test_a_million_empty_sequences_between_two():
    """Blocks look at thousands of items without a token, one after another, while their other warps wait."""
    batch, seq, heads, d = 1 << 20, 2, 4, 8
    lengths = torch.zeros(batch, dtype=torch.int32, device="cuda")
    lengths[0], lengths[-1] = 2, 1
    Z = torch.full((batch, seq, heads + 2, d), math.nan, dtype=BF16, device="cuda")
    some = torch.randn((2, seq, heads + 2, d), generator=torch.Generator(device="cuda").manual_seed(2), device="cuda").to(BF16)
    Z[0], Z[-1] = some[0], some[1]
    Q, K, V = Z.split((heads, 1, 1), -2)
    O, lse = pamm.attention_forward(Q, K, V, lengths=lengths)
    grads = pamm.attention_backward(Q, Q, K, V, O, lse, lengths=lengths)
    assert pamm.last_device_status() == pamm.OK
    q, k, v = some.split((heads, 1, 1), -2)
    few = lengths[[0, -1]].contiguous()
    o, l = pamm.attention_forward(q, k, v, lengths=few)
    for a, b in zip((O, lse, *grads), (o, l, *pamm.attention_backward(q, q, k, v, o, l, lengths=few))):
        assert torch.equal(a[[0, -1]], b)
        assert (a[1:-1] == (-math.inf if a is lse else 0.0)).all()


def test_falling_starts_are_reported_and_stay_in_bounds():
    tokens, heads, d, guard = 150, 3, 64, 4096
    Q, K, V = torch.randn((tokens, heads + 2, d), generator=torch.Generator(device="cuda").manual_seed(5), device="cuda").to(BF16).split((heads, 1, 1), -2)

    def guarded(shape, dtype=BF16):
        n = math.prod(shape)
        whole = torch.full((n + 2 * guard,), 3.0, dtype=dtype, device="cuda")
        return whole, whole[guard:guard + n].view(shape)

    rows = {"O": (tokens, heads, d), "dQ": (tokens, heads, d), "dK": (tokens, 1, d), "dV": (tokens, 1, d)}
    for dtype in (BF16, torch.float32):
        q, k, v = (t.to(dtype) for t in (Q, K, V))
        for starts in ([0, 100, 50, 150], [150, 0], [0, 150, 0, 150, 0, 150], [120, 30, 31, 20, 150], list(range(150, -1, -1))):
            out = {n: guarded(s, dtype) for n, s in rows.items()}
            out["lse"] = guarded((heads, tokens), torch.float32)
            s = torch.tensor(starts, device="cuda")
            O, lse = pamm.attention_forward(q, k, v, starts=s, O=out["O"][1], lse=out["lse"][1])
            assert pamm.last_device_status() == pamm.ERR_BAD_INDEX, starts
            pamm.attention_backward(q, q, k, v, O, lse, starts=s, **{n: out[n][1] for n in ("dQ", "dK", "dV")})
            assert pamm.last_device_status() == pamm.ERR_BAD_INDEX, starts
            for whole, _ in out.values():
                assert (whole[:guard] == 3.0).all() and (whole[-guard:] == 3.0).all()
        sound = torch.tensor([0, 50, 150], device="cuda")
        a, b = pamm.attention_forward(q, k, v, starts=sound)[0], pamm.attention_forward(q[50:], k[50:], v[50:])[0]
        assert pamm.last_device_status() == pamm.OK and torch.equal(a[50:], b)
