"""The operators around the fused Q|K|V projection that a training step needs: what is measured, and their plain forms.

``norm``    layer norm and its root-mean-square form, forward and backward, optionally with the residual addition
``rotary``  rotary positions on the heads of the fused row [Q|K|V], forward and transposed (the backward pass)
``clip``    the global norm over a list of gradients, and their clipping
"""
import math

import torch

own = False

BF16, F32 = "bf16", "f32"
_DT = {BF16: torch.bfloat16, F32: torch.float32}
_SIZE = {BF16: 2, F32: 4}
EPS = 1e-5


def listed():
    return [
        # eight tokens at a time through a model's norm, as when its answers are looked at between steps: latency
        dict(name="norm fwd, few tokens", op="norm", back=False, rms=True, b=8, n=2048, dt=BF16, wdt=BF16, bias=False, add=False),
        # the norm before the projection of a 1B-sized layer, with the residual addition: 64 x 1024 tokens
        dict(name="norm fwd, residual", op="norm", back=False, rms=True, b=65536, n=2048, dt=BF16, wdt=BF16, bias=False, add=True),
        # a small fp32 layer's training batch: 8 x 256 tokens, layer norm with bias
        dict(name="norm bwd, small", op="norm", back=True, rms=False, b=2048, n=512, dt=F32, wdt=F32, bias=True, add=False),
        # packed sequences of odd number and a width that leaves rows unaligned, fp32 weights beside bf16 activations
        dict(name="norm bwd, ragged", op="norm", back=True, rms=False, b=4099, n=1999, dt=BF16, wdt=F32, bias=True, add=False),
        # the wide layer's backward pass with the residual stream's gradient: 4 x 8192 tokens
        dict(name="norm bwd, residual", op="norm", back=True, rms=True, b=32768, n=4096, dt=BF16, wdt=BF16, bias=False, add=True),
        # one new token of each of eight sequences, 32 + 8 heads in a row of 48: latency, scattered positions
        dict(name="rotary, one token each", op="rotary", back=False, batch=8, seq=1, heads=48, rotated=40, d=128, rot=128,
             pairs="half", dt=BF16, whole=False, given=True, table=8192),
        # 64 x 1024 training tokens, 16 + 16 heads rotated out of a row of 48
        dict(name="rotary, training", op="rotary", back=False, batch=64, seq=1024, heads=48, rotated=32, d=128, rot=128,
             pairs="half", dt=BF16, whole=False, given=False, table=1024),
        # the gradient of a long-context layer's whole row, V passing through, adjacent pairs
        dict(name="rotary bwd, long", op="rotary", back=True, batch=4, seq=8192, heads=48, rotated=40, d=128, rot=128,
             pairs="adjacent", dt=BF16, whole=True, given=False, table=8192),
        # packed sequences in fp32, a quarter of an 80-wide head rotated
        dict(name="rotary, part of the head", op="rotary", back=False, batch=3, seq=517, heads=15, rotated=10, d=80, rot=20,
             pairs="adjacent", dt=F32, whole=False, given=True, table=4096),
        # a small fp32 model's gradients in place, below the limit, as in most steps: 8 layers of weights and norm vectors
        dict(name="clip, below the limit", op="clip", layers=8, n=512, m=1536, odd=0, dt=F32, out="place", over=False, bucket=False),
        # 192 gradients of odd sizes in two buckets, so that hardly any starts on a 16-byte boundary; above the limit
        dict(name="clip, odd sizes", op="clip", layers=48, n=767, m=1153, odd=3, dt=BF16, out="same", over=True, bucket=True),
        # a 1B-sized model's projection gradients in bf16, clipped into the optimizer's fp32 buffers
        dict(name="clip, large", op="clip", layers=16, n=2048, m=6144, odd=0, dt=BF16, out="f32", over=True, bucket=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _allowed(v):
    return v + 1 if v == 3072 else v


def draw(rng):
    op = rng.choice(("norm", "norm", "rotary", "clip"))
    dt = rng.choice((BF16, BF16, F32))
    if op == "norm":
        n = _allowed(_log(rng, 64, 16384))
        if rng.random() < 0.6:
            n = _allowed((n + 63) // 64 * 64)
        b = _allowed(_log(rng, 1, min(65536, 70_000_000 // n)))
        rms = rng.random() < 0.5
        return dict(op="norm", back=rng.random() < 0.5, rms=rms, b=b, n=n, dt=dt, wdt=rng.choice((dt, F32)),
                    bias=not rms and rng.random() < 0.8, add=rng.random() < 0.4)
    if op == "rotary":
        d = rng.choice((40, 64, 80, 96, 128, 256))
        rot = rng.choice((d, d, d // 2, d // 4))
        rotated = rng.randint(1, 40)
        heads = rotated + rng.randint(0, 8)
        tokens = _log(rng, 1, max(1, 100_000_000 // (heads * d)))
        batch = max(1, min(tokens, _log(rng, 1, 64)))
        seq = max(1, min(8192, tokens // batch))
        return dict(op="rotary", back=rng.random() < 0.5, batch=batch, seq=seq, heads=heads, rotated=rotated, d=d, rot=rot,
                    pairs=rng.choice(("half", "adjacent")), dt=dt, whole=rng.random() < 0.5, given=rng.random() < 0.5, table=8192)
    n, m = _allowed(_log(rng, 60, 4096)), _allowed(_log(rng, 60, 6144))
    bucket = rng.random() < 0.5
    layers = _log(rng, 1, max(1, min(64 if bucket else 15, 100_000_000 // (n * m))))
    over = rng.random() < 0.6
    return dict(op="clip", layers=layers, n=n, m=m, odd=rng.randint(0, 5), dt=dt, over=over, bucket=bucket,
                out=rng.choice(("same", "f32")) if over else "place")


def _gradients(case):
    """(type, rows, columns, row distance) of every gradient: a matrix and two vectors a layer and, with ``odd``, a matrix
    whose rows lie apart, as the framework lays out widths that are no multiple of 16 bytes."""
    layer = [(case["dt"], case["n"], case["m"], case["m"]), (F32, 1, case["n"], case["n"]), (F32, 1, case["m"], case["m"])]
    if case["odd"]:
        layer.append((case["dt"], case["odd"] * 7, 91, 96))
    return layer * case["layers"]


def _views(case, dts, make):
    """The gradients as views of the memory ``make(size, dt)`` gives, and that memory: one piece for each gradient or, with
    ``bucket``, one for each type.  ``dts``: the type that each gradient type is held in."""
    shapes = _gradients(case)
    if not case["bucket"]:
        memory = [make(rows * ld, dts[dt]) for dt, rows, _, ld in shapes]
        return [t.view(rows, ld)[:, :cols] for t, (_, rows, cols, ld) in zip(memory, shapes)], memory
    views, ends = [], {}
    sizes = {dt: sum(rows * ld for t, rows, _, ld in shapes if t == dt) for dt in (F32, BF16)}
    memory = {dt: make(size, dts[dt]) for dt, size in sizes.items() if size}
    for dt, rows, cols, ld in shapes:
        at = ends.get(dt, 0)
        views.append(memory[dt][at:at + rows * ld].view(rows, ld)[:, :cols])
        ends[dt] = at + rows * ld
    return views, list(memory.values())


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, scale=1.0, dt=F32):
        return torch.randn(shape, generator=g, device="cuda").mul_(scale).to(_DT[dt])

    if case["op"] == "norm":
        b, n, dt = case["b"], case["n"], case["dt"]
        state = dict(case=case)
        # a residual stream: rows of different size, a few channels far larger than the others
        channel = torch.exp(0.5 * torch.randn((n,), generator=g, device="cuda"))
        channel[torch.randint(0, n, (max(1, n // 256),), generator=g, device="cuda")] *= 8.0
        row = torch.exp(0.5 * torch.randn((b, 1), generator=g, device="cuda"))
        state["x"] = (normal(b, n).mul_(channel).mul_(row) + 0.1).to(_DT[dt])
        state["w"] = (1.0 + normal(n, scale=0.1)).to(_DT[case["wdt"]])
        state["c"] = normal(n, scale=0.1, dt=case["wdt"]) if case["bias"] else None
        if case["back"]:
            state["dy"] = normal(b, n, scale=1e-3, dt=dt)
            state["dh"] = normal(b, n, scale=1e-3, dt=dt) if case["add"] else None
            x = state["x"].float()
            mean = x.new_zeros((b,)) if case["rms"] else x.mean(1)
            var = (x - mean[:, None]).square().mean(1)
            state["mean"], state["rstd"] = None if case["rms"] else mean, torch.rsqrt(var + EPS)
        else:
            state["r"] = normal(b, n, scale=0.3, dt=dt) if case["add"] else None
        return state
    if case["op"] == "rotary":
        batch, seq, heads, d, rot = (case[k] for k in ("batch", "seq", "heads", "d", "rot"))
        z = normal(batch, seq, heads * d, scale=1e-3 if case["back"] else 1.0, dt=case["dt"])
        f = 10000.0 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot)
        angle = torch.arange(case["table"], device="cuda", dtype=torch.float64)[:, None] * f
        table = torch.cat((angle.cos(), angle.sin()), 1).float()       # [cos | sin] of every position, kept by the program
        given = torch.randint(0, case["table"], (batch, seq), generator=g, device="cuda") if case["given"] else None
        return dict(case=case, z=z.view(batch, seq, heads, d), table=table, positions=given)
    grads, memory = _views(case, {F32: F32, BF16: BF16}, lambda size, dt: normal(size, scale=1e-3, dt=dt))
    size = 1e-3 * math.sqrt(sum(t.numel() for t in grads))
    state = dict(case=case, grads=grads, memory=memory, out=None, limit=0.3 * size if case["over"] else 4.0 * size)
    if case["out"] != "place":
        state["out"], state["memory"] = _views(case, {F32: F32, BF16: F32 if case["out"] == "f32" else BF16},
                                               lambda size, dt: torch.zeros(size, dtype=_DT[dt], device="cuda"))
    return state


def run(state):
    return {"norm": _norm, "rotary": _rotary, "clip": _clip}[state["case"]["op"]](state)


def _norm(s):
    case = s["case"]
    if own:
        from paper_2506_02939_b200 import pamm
        if case["back"]:
            dx, dw, dc = pamm.norm_backward(s["dy"], s["x"], s["mean"], s["rstd"], s["w"], bias=case["bias"], dH=s["dh"])
            return dict(dx=dx, dw=dw, dc=dc)
        y, h, mean, rstd = pamm.norm_forward(s["x"], s["w"], s["c"], residual=s["r"], eps=EPS, rms=case["rms"])
        return dict(y=y, h=h if case["add"] else None, mean=mean, rstd=rstd)
    x, w = s["x"].float(), s["w"].float()
    n = x.shape[1]
    if case["back"]:
        dy = s["dy"].float()
        xh = (x if case["rms"] else x - s["mean"][:, None]) * s["rstd"][:, None]
        g = dy * w
        dx = g - xh * ((g * xh).sum(1, keepdim=True) / n)
        if not case["rms"]:
            dx = dx - g.sum(1, keepdim=True) / n
        dx = dx * s["rstd"][:, None]
        if s["dh"] is not None:
            dx = dx + s["dh"].float()
        wdt = s["w"].dtype
        return dict(dx=dx.to(s["x"].dtype), dw=(dy * xh).sum(0).to(wdt), dc=dy.sum(0).to(wdt) if case["bias"] else None)
    h = x if s["r"] is None else x + s["r"].float()
    mean = None if case["rms"] else h.sum(1) / n
    centred = h if mean is None else h - mean[:, None]
    rstd = 1.0 / torch.sqrt((centred * centred).sum(1) / n + EPS)
    y = centred * rstd[:, None] * w
    if s["c"] is not None:
        y = y + s["c"].float()
    dt = s["x"].dtype
    return dict(y=y.to(dt), h=h.to(dt) if case["add"] else None, mean=mean, rstd=rstd)


def _rotary(s):
    case, z = s["case"], s["z"]
    if own:
        from paper_2506_02939_b200 import pamm
        x = z if case["whole"] else z[:, :, :case["rotated"]]
        return pamm.rotary(x, s["table"], s["positions"], rotated=case["rotated"], rot_dim=case["rot"],
                           interleaved=case["pairs"] == "adjacent", transposed=case["back"])
    rot, half, rotated = case["rot"], case["rot"] // 2, case["rotated"]
    rows = s["table"][:case["seq"]][None] if s["positions"] is None else s["table"][s["positions"]]
    cos, sin = rows[:, :, None, :half], rows[:, :, None, half:]
    if case["back"]:
        sin = -sin
    x = z[:, :, :rotated].float()
    if case["pairs"] == "half":
        x1, x2 = x[..., :half], x[..., half:rot]
        turned = torch.cat((x1 * cos - x2 * sin, x2 * cos + x1 * sin, x[..., rot:]), -1)
    else:
        x1, x2 = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack((x1 * cos - x2 * sin, x2 * cos + x1 * sin), -1).flatten(-2)
        turned = torch.cat((turned, x[..., rot:]), -1)
    turned = turned.to(z.dtype)
    return torch.cat((turned, z[:, :, rotated:]), 2) if case["whole"] else turned


def _clip(s):
    grads, out = s["grads"], s["out"]
    if own:
        from paper_2506_02939_b200 import pamm
        return dict(norm=pamm.clip_grad_norm(grads, s["limit"], out=out), memory=s["memory"])
    total = torch.stack([g.float().square().sum() for g in grads]).sum().sqrt()
    coef = (s["limit"] / (total + 1e-6)).clamp(max=1.0)
    [t.copy_(g.float() * coef) for t, g in zip(grads if out is None else out, grads)]
    return dict(norm=total, memory=s["memory"])


def work(case):
    e = _SIZE[case["dt"]]
    if case["op"] == "norm":
        b, n, ew = case["b"], case["n"], _SIZE[case["wdt"]]
        stats = 4 * b * (1 if case["rms"] else 2)
        if case["back"]:
            matrices, vectors, per = (4 if case["add"] else 3), (3 if case["bias"] else 2), 13
        else:
            matrices, vectors, per = (4 if case["add"] else 2), (2 if case["bias"] else 1), 7
        return dict(bytes=matrices * b * n * e + vectors * n * ew + stats, flops=per * b * n)
    if case["op"] == "rotary":
        tokens = case["batch"] * case["seq"]
        values = tokens * (case["heads"] if case["whole"] else case["rotated"]) * case["d"]
        rows = min(case["table"], tokens) if case["given"] else case["seq"]
        return dict(bytes=2 * values * e + 4 * case["rot"] * rows + (8 * tokens if case["given"] else 0),
                    flops=3 * tokens * case["rotated"] * case["rot"])
    values = sum(rows * cols for _, rows, cols, _ in _gradients(case))
    read = sum(rows * cols * _SIZE[dt] for dt, rows, cols, _ in _gradients(case))
    write = {"place": 0, "same": read, "f32": 4 * values}[case["out"]]
    return dict(bytes=read + write, flops=(2 if case["out"] == "place" else 3) * values)


def exact(case, seed):
    """The operators' definitions in 64 bits."""
    s = prepare(case, seed)
    if case["op"] == "norm":
        return _exact_norm(case, s)
    if case["op"] == "rotary":
        z = s["z"].double()
        half = case["rot"] // 2
        where = torch.arange(case["seq"], device=z.device).expand(case["batch"], -1) if s["positions"] is None else s["positions"]
        turn = torch.complex(*(t.double() for t in s["table"][where].split(half, -1)))[:, :, None, :]
        if case["back"]:
            turn = turn.conj()
        k = torch.arange(half, device=z.device)
        first, second = (k, k + half) if case["pairs"] == "half" else (2 * k, 2 * k + 1)
        heads = z[:, :, :case["rotated"]]
        turned = torch.complex(heads.index_select(-1, first), heads.index_select(-1, second)) * turn
        heads.index_copy_(-1, first, turned.real.contiguous())
        heads.index_copy_(-1, second, turned.imag.contiguous())
        return z if case["whole"] else heads.contiguous()
    total = math.sqrt(math.fsum(float(torch.linalg.vector_norm(g.double())) ** 2 for g in s["grads"]))
    factor = min(1.0, s["limit"] / (total + 1e-6))
    if s["out"] is None:      # below the limit: what lies in the gradients' memory stays, the gaps between rows with it
        memory = [t.double() for t in s["memory"]]
        assert factor == 1.0
    else:
        views, memory = _views(case, {F32: F32, BF16: BF16}, lambda size, dt: torch.zeros(size, dtype=torch.float64, device="cuda"))
        for view, g in zip(views, s["grads"]):
            view.copy_(g).mul_(factor)
    return dict(norm=torch.tensor(total, dtype=torch.float64), memory=memory)


def _exact_norm(case, s):
    n = case["n"]
    h = s["x"].double() + (s["r"].double() if s.get("r") is not None else 0.0)
    w = s["w"].double()
    if not case["back"]:
        if case["rms"]:
            mean, square = None, torch.linalg.vector_norm(h, dim=1).square() / n
            unit = h
        else:
            square, mean = torch.var_mean(h, 1, correction=0)
            unit = h - mean.unsqueeze(1)
        rstd = (square + EPS).pow(-0.5)
        y = torch.einsum("ij,i,j->ij", unit, rstd, w)
        if s["c"] is not None:
            y += s["c"].double()
        return dict(y=y, h=h if case["add"] else None, mean=mean, rstd=rstd)
    rstd = s["rstd"].double()
    unit = torch.einsum("ij,i->ij", h if case["rms"] else h - s["mean"].double().unsqueeze(1), rstd)
    dy = s["dy"].double()
    dw = torch.einsum("ij,ij->j", dy, unit)
    dc = torch.einsum("ij->j", dy) if case["bias"] else None
    along = torch.einsum("ij,ij,j->i", dy, unit, w) / n
    dx = torch.addcmul(dy * w, unit, along.unsqueeze(1), value=-1.0)
    if not case["rms"]:
        dx -= (torch.mv(dy, w) / n).unsqueeze(1)
    dx *= rstd.unsqueeze(1)
    if s["dh"] is not None:
        dx += s["dh"].double()
    return dict(dx=dx, dw=dw, dc=dc)
