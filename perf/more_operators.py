"""The operators behind the fused Q|K|V projection that a training step needs: what is measured, and their plain forms.

``attention``  softmax attention of the fused row [Q|K|V], forward (output and the rows' log-sums) and backward, which makes
               the probabilities anew: whole, padded and packed batches, causal or not, heads that share keys and values
``dropout``    dropout with a residual, whose mask comes from a counter-based generator and is never stored; the backward pass
               is the same call on the gradient
"""
import math
import random

import torch

own = False

BF16, F32 = "bf16", "f32"
_DT = {BF16: torch.bfloat16, F32: torch.float32}
_SIZE = {BF16: 2, F32: 4}


def listed():
    return [
        # eight short prompts looked at between training steps: latency
        dict(name="attention fwd, short", op="attention", back=False, batch=8, seq=17, heads=16, kv=16, d=128, causal=True,
             layout="whole", mix=0, dt=BF16),
        # a 1B-sized layer's training batch: 64 x 1024 tokens, 16 heads of 128
        dict(name="attention fwd, training", op="attention", back=False, batch=64, seq=1024, heads=16, kv=16, d=128, causal=True,
             layout="whole", mix=0, dt=BF16),
        # a small fp32 layer's padded batch: 8 x 256 tokens, 8 heads of 64
        dict(name="attention fwd, fp32 padded", op="attention", back=False, batch=8, seq=256, heads=8, kv=8, d=64, causal=True,
             layout="padded", mix=1, dt=F32),
        # packed documents of odd lengths, from one token on, both directions visible, as an encoder has them
        dict(name="attention fwd, packed", op="attention", back=False, batch=41, seq=901, heads=12, kv=12, d=64, causal=False,
             layout="packed", mix=2, dt=BF16),
        # a long-context layer: 2 x 8192 tokens, 32 heads over 8 of keys and values
        dict(name="attention fwd, long", op="attention", back=False, batch=2, seq=8192, heads=32, kv=8, d=128, causal=True,
             layout="whole", mix=0, dt=BF16),
        # the gradients of the same: the small fp32 batch,
        dict(name="attention bwd, fp32 padded", op="attention", back=True, batch=8, seq=256, heads=8, kv=8, d=64, causal=True,
             layout="padded", mix=1, dt=F32),
        # packed documents with heads of 80 that share keys and values,
        dict(name="attention bwd, packed", op="attention", back=True, batch=29, seq=777, heads=12, kv=4, d=80, causal=True,
             layout="packed", mix=3, dt=BF16),
        # the training batch,
        dict(name="attention bwd, training", op="attention", back=True, batch=64, seq=1024, heads=16, kv=16, d=128, causal=True,
             layout="whole", mix=0, dt=BF16),
        # and the long context
        dict(name="attention bwd, long", op="attention", back=True, batch=2, seq=8192, heads=32, kv=8, d=128, causal=True,
             layout="whole", mix=0, dt=BF16),
        # a small batch's residual dropout: latency
        dict(name="dropout, few tokens", op="dropout", back=False, b=8, n=2048, p=0.1, add=True, dt=BF16),
        # a 1B-sized layer's residual dropout: 64 x 1024 tokens
        dict(name="dropout, residual", op="dropout", back=False, b=65536, n=2048, p=0.1, add=True, dt=BF16),
        # the gradient's dropout where neither the rows nor their number are even, fp32
        dict(name="dropout bwd, odd", op="dropout", back=True, b=4099, n=1999, p=0.25, add=False, dt=F32),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    if rng.random() < 0.3:
        n = _log(rng, 16, 16384)
        if rng.random() < 0.6:
            n = (n + 63) // 64 * 64
        back = rng.random() < 0.5
        return dict(op="dropout", back=back, b=_log(rng, 1, min(65536, 130_000_000 // n)), n=n, p=rng.choice((0.05, 0.1, 0.2, 0.5)),
                    add=not back and rng.random() < 0.7, dt=rng.choice((BF16, BF16, F32)))
    dt = rng.choice((BF16, BF16, BF16, F32))
    d = rng.choice((40, 64, 80, 96, 128, 128))
    kv = rng.choice((1, 2, 4, 8, 12, 16))
    heads = kv * rng.choice([g for g in (1, 1, 2, 3, 4, 8) if g * kv <= 32])
    back = rng.random() < 0.5
    seq = _log(rng, 4 if back else 1, 8192 if dt == BF16 else 2048)      # a token that sees itself alone has no gradient to Q and K
    pairs = (2 << 30) if dt == BF16 else (1 << 27)                 # of all heads and sequences, at most
    batch = _log(rng, 1, max(1, min(64, pairs // (heads * seq * seq), 100_000_000 // ((heads + 2 * kv) * d * seq))))
    return dict(op="attention", back=back, batch=batch, seq=seq, heads=heads, kv=kv, d=d, causal=rng.random() < 0.7,
                layout=rng.choice(("whole", "padded", "packed")), mix=rng.randint(0, 1 << 20), dt=dt)


def _lengths(case):
    """The sequences' lengths: full ones, tails of up to a third left out, or packed ones between one token and ``seq``."""
    batch, seq, rng = case["batch"], case["seq"], random.Random(case["mix"])
    if case["layout"] == "whole":
        return [seq] * batch
    if case["layout"] == "padded":
        return [seq - rng.randint(0, seq // 3) for _ in range(batch)]
    return [seq] + [max(1, round(seq * rng.random() ** 1.5)) for _ in range(batch - 1)]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, scale=1.0, dt=F32):
        return torch.randn(shape, generator=g, device="cuda").mul_(scale).to(_DT[dt])

    if case["op"] == "dropout":
        b, n, dt = case["b"], case["n"], case["dt"]
        return dict(case=case, x=normal(b, n, scale=1e-3 if case["back"] else 1.0, dt=dt), r=normal(b, n, dt=dt) if case["add"] else None,
                    seed=random.Random(seed).getrandbits(62), offset=seed % 1000)
    lengths, heads, kv, d, dt = _lengths(case), case["heads"], case["kv"], case["d"], case["dt"]
    packed = case["layout"] == "packed"
    tokens = (sum(lengths) + 3,) if packed else (case["batch"], case["seq"])         # packed: a few rows behind the last sequence
    z = torch.randn((*tokens, heads + 2 * kv, d), generator=g, device="cuda")
    z[..., :heads, :].mul_(2.0)                                    # scores with a standard deviation of two: some keys stand out
    state = dict(case=case, z=z.to(_DT[dt]), lengths=None, starts=None)
    if packed:
        state["starts"] = torch.tensor([0] + lengths, device="cuda").cumsum(0).to(torch.int32)
    elif case["layout"] == "padded":
        state["lengths"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    if case["back"]:
        o, lse = _forward(state)
        state.update(o=o, lse=lse, do=normal(*tokens, heads, d, scale=1e-3, dt=dt))
    return state


def run(state):
    case = state["case"]
    if case["op"] == "dropout":
        return _dropout(state)
    if own:
        from paper_2506_02939_b200 import pamm
        q, k, v = state["z"].split((case["heads"], case["kv"], case["kv"]), -2)
        how = dict(causal=case["causal"], lengths=state["lengths"], starts=state["starts"])
        if case["back"]:
            dq, dk, dv = pamm.attention_backward(state["do"], q, k, v, state["o"], state["lse"], **how)
            return dict(dq=dq, dk=dk, dv=dv)
        o, lse = pamm.attention_forward(q, k, v, **how)
        return dict(o=o, lse=lse)
    if case["back"]:
        return _backward(state)
    o, lse = _forward(state)
    return dict(o=o, lse=lse)


def _batched(state):
    """Q, K and V as (batch, kv heads, ..., positions, d) in fp32, which scores count, and how rows come back: packed sequences are laid
    out side by side, each as long as the longest."""
    case, z = state["case"], state["z"]
    heads, kv, d, seq = case["heads"], case["kv"], case["d"], case["seq"]
    at = torch.arange(seq, device=z.device)
    if state["starts"] is not None:
        starts = state["starts"].long()
        lengths = starts[1:] - starts[:-1]
        where = (starts[:-1, None] + at).clamp(max=z.shape[0] - 1)
    else:
        lengths = torch.full((z.shape[0],), seq, device=z.device) if state["lengths"] is None else state["lengths"].long()
        where = None
    known = at < lengths[:, None]                                  # (batch, positions)
    allowed = known[:, :, None] & known[:, None, :]
    if case["causal"]:
        allowed = allowed & (at[:, None] >= at)
    allowed = allowed[:, None, None]

    def by_head(t, count):             # (…, count heads, d) -> (batch, kv, count / kv, positions, d)
        t = t if where is None else t[where]
        return t.float().view(t.shape[0], seq, kv, count // kv, d).permute(0, 2, 3, 1, 4)

    def by_token(t, dt):               # and back, rows of no sequence zero
        t = t.permute(0, 3, 1, 2, 4).flatten(2, 3)
        t = torch.where(known[:, :, None, None], t, 0.0).to(dt)
        if where is None:
            return t
        out = t.new_zeros((z.shape[0], *t.shape[2:]))
        out[where[known]] = t[known]
        return out

    def row_numbers(t):                # (batch, kv, group, positions) -> (batch, heads, positions), or (heads, tokens) of packed ones
        t = t.flatten(1, 2).masked_fill(~known[:, None], -math.inf)
        if where is None:
            return t
        out = t.new_full((heads, z.shape[0]), -math.inf)
        out[:, where[known]] = t.transpose(0, 1)[:, known]
        return out

    def rows_of(t):                    # its inverse
        if where is not None:
            t = t[:, where].transpose(0, 1)
        return t.reshape(t.shape[0], kv, heads // kv, seq)

    q, k, v = z.split((heads, kv, kv), -2)
    return by_head(q, heads), by_head(k, kv), by_head(v, kv), allowed, by_head, by_token, row_numbers, rows_of


def _forward(state):
    q, k, v, allowed, _, by_token, row_numbers, _ = _batched(state)
    s = torch.matmul(q, k.transpose(-1, -2)).mul_(1.0 / math.sqrt(q.shape[-1])).masked_fill_(~allowed, -math.inf)
    top = s.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = s.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total == 0.0, 1.0, total)
    return by_token(o, state["z"].dtype), row_numbers((top + total.log()).squeeze(-1))


def _backward(state):
    q, k, v, allowed, by_head, by_token, _, rows_of = _batched(state)
    heads, dt, scale = state["case"]["heads"], state["z"].dtype, 1.0 / math.sqrt(q.shape[-1])
    o, do = by_head(state["o"], heads), by_head(state["do"], heads)
    do = torch.where(allowed.any(-1, keepdim=True), do, 0.0)
    p = torch.matmul(q, k.transpose(-1, -2)).mul_(scale).sub_(rows_of(state["lse"]).unsqueeze(-1)).exp_().masked_fill_(~allowed, 0.0)
    dv = torch.matmul(p.transpose(-1, -2), do).sum(2, keepdim=True)
    ds = p.mul_(torch.matmul(do, v.transpose(-1, -2)).sub_((o * do).sum(-1, keepdim=True)))
    dq = torch.matmul(ds, k).mul_(scale)
    dk = torch.matmul(ds.transpose(-1, -2), q).sum(2, keepdim=True).mul_(scale)
    return dict(dq=by_token(dq, dt), dk=by_token(dk, dt), dv=by_token(dv, dt))


def _random_words(count, seed, offset, device):
    """``count`` words of 32 bits, as int64: Philox 4x32 with ten rounds (Salmon et al., 2011); word e is entry e % 4 of the block of
    counter (e / 4, offset), 64 bits each, under the key ``seed``."""
    low = 0xFFFFFFFF
    block = torch.arange((count + 3) // 4, device=device)
    c0, c1, c2, c3 = block & low, block >> 32, torch.full_like(block, offset & low), torch.full_like(block, offset >> 32)
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57                  # modulo 2^64
        c0, c1, c2, c3 = (p1 >> 32) & low ^ c1 ^ k0, p1 & low, (p0 >> 32) & low ^ c3 ^ k1, p0 & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return torch.stack((c0, c1, c2, c3), 1).flatten()[:count]


def _dropout(s):
    case, x, r = s["case"], s["x"], s["r"]
    if own:
        from paper_2506_02939_b200 import pamm
        return pamm.dropout(x, case["p"], s["seed"], s["offset"], residual=r)
    kept = _random_words(x.numel(), s["seed"], s["offset"], x.device).view(x.shape) >= int(case["p"] * 2.0 ** 32)
    y = torch.where(kept, x.float() * (1.0 / (1.0 - case["p"])), 0.0)
    return (y if r is None else y + r.float()).to(x.dtype)


def work(case):
    e = _SIZE[case["dt"]]
    if case["op"] == "dropout":
        values = case["b"] * case["n"]
        return dict(bytes=(3 if case["add"] else 2) * values * e, flops=(2 if case["add"] else 1) * values)
    lengths, heads, kv, d = _lengths(case), case["heads"], case["kv"], case["d"]
    tokens = sum(lengths)
    pairs = heads * sum(n * (n + 1) // 2 if case["causal"] else n * n for n in lengths)
    rows = (heads + 2 * kv) * d * e                                # of one token: Q, K, V
    if case["back"]:                                               # those, O, dO and the log-sum read; dQ, dK, dV written
        return dict(bytes=tokens * (2 * rows + 2 * heads * d * e + 4 * heads), flops=10 * d * pairs)
    return dict(bytes=tokens * (rows + heads * d * e + 4 * heads), flops=4 * d * pairs)


def exact(case, seed):
    """The operators' definitions in 64 bits."""
    s = prepare(case, seed)
    return _exact_dropout(case, s) if case["op"] == "dropout" else _exact_attention(case, s)


def _exact_attention(case, s):
    heads, kv, d, back = case["heads"], case["kv"], case["d"], case["back"]
    z, group, packed = s["z"], heads // kv, case["layout"] == "packed"
    o = torch.zeros((*z.shape[:-2], heads, d), dtype=torch.float64, device=z.device)
    lse = torch.full((heads, z.shape[0]) if packed else (z.shape[0], heads, case["seq"]), -math.inf, dtype=torch.float64, device=z.device)
    dz = torch.zeros(z.shape, dtype=torch.float64, device=z.device) if back else None
    first = 0
    for i, n in enumerate(_lengths(case)):
        rows = slice(first, first + n) if packed else (i, slice(0, n))
        first += n
        for h in range(kv):
            mine = slice(h * group, (h + 1) * group)
            q, k, v = (z[rows][:, a].double() for a in (mine, heads + h, heads + kv + h))
            a = torch.einsum("igd,jd->gij", q, k) / d ** 0.5
            if case["causal"]:
                a += torch.full((n, n), -math.inf, dtype=a.dtype, device=a.device).triu(1)
            where = (mine, slice(first - n, first)) if packed else (i, mine, slice(0, n))
            if not back:
                lse[where] = torch.logsumexp(a, -1)
                o[rows][:, mine] = torch.einsum("gij,jd->igd", torch.softmax(a, -1), v)
                continue
            p = torch.exp(a - s["lse"][where].double()[..., None])
            del a
            do, out = s["do"][rows][:, mine].double(), s["o"][rows][:, mine].double()
            dz[rows][:, heads + kv + h] = torch.einsum("gij,igd->jd", p, do)
            p *= torch.einsum("igd,jd->gij", do, v) - torch.einsum("igd,igd->gi", do, out)[..., None]
            p /= d ** 0.5
            dz[rows][:, mine] = torch.einsum("gij,jd->igd", p, k)
            dz[rows][:, heads + h] = torch.einsum("gij,igd->jd", p, q)
    if not back:
        return dict(o=o, lse=lse)
    dq, dk, dv = dz.split((heads, kv, kv), -2)
    return dict(dq=dq, dk=dk, dv=dv)


def _exact_dropout(case, s):
    x = s["x"].double().flatten()
    block, at = torch.arange(x.numel(), device=x.device) // 4, torch.arange(x.numel(), device=x.device) % 4

    def product(m, c):                 # upper and lower 32 bits of a 32-bit number times a constant, by halves of it
        a, b = c * (m >> 16), c * (m & 0xFFFF)
        a += b >> 16
        return a >> 16, ((a & 0xFFFF) << 16) + (b & 0xFFFF)

    word = [block % (1 << 32), block // (1 << 32), torch.full_like(block, s["offset"] % (1 << 32)), torch.full_like(block, s["offset"] // (1 << 32))]
    key = [s["seed"] % (1 << 32), s["seed"] // (1 << 32)]
    for _ in range(10):
        (h0, l0), (h1, l1) = product(0xD2511F53, word[0]), product(0xCD9E8D57, word[2])
        word = [h1.bitwise_xor_(word[1]).bitwise_xor_(key[0]), l1, h0.bitwise_xor_(word[3]).bitwise_xor_(key[1]), l0]
        key = [(key[0] + 0x9E3779B9) % (1 << 32), (key[1] + 0xBB67AE85) % (1 << 32)]
    drawn = torch.where(at < 2, torch.where(at == 0, word[0], word[1]), torch.where(at == 2, word[2], word[3]))
    y = torch.where(drawn < math.floor(case["p"] * 2.0 ** 32), 0.0, x / (1.0 - case["p"]))
    return y.view(s["x"].shape) if s["r"] is None else y.view(s["x"].shape) + s["r"].double()
