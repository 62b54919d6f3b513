"""Operators around the AirCache hot path that are timed and compared with their plain forms: the norm and rotation of
queries and keys (`air_rope`) and attention over a prompt (`air_prompt_attn`).

Tensors are indexed [B][head][token][d].  Fields of a case: op; dtype and d; hq query heads over hkv KV heads; `qkv`: the
tensors are views of one token-major buffer [B][token][hq + 2 hkv][d], as one projection leaves them, else each is
[B][head][token][d] in memory.

rope: `lens` tokens of every sequence of the batch (rows behind a shorter one are padding: position -1, left as they are);
rot: leading elements of a head that are rotated, `layout` half or interleaved; axes: pairs per position axis (one axis, or
three for images: time, row, column); norm: queries and keys are normalised per head first; factor: context extension of the
frequencies; start: position of the first token.

attn: q_lens / kv_lens of every sequence; the queries are the last q_len of the kv_len positions.  packed: the sequences lie
one behind the other along the token axis of a batch of one, else each in its row of a padded batch.
"""
from __future__ import annotations

import math

import torch

own = False  # True: `run` calls the library; False: the operators in elementary torch operations

THETA = 1e6


def _text(numbers):
    """A list of whole numbers as a case holds it."""
    return " ".join(map(str, numbers))


def _ints(text):
    return [int(x) for x in text.split()]


def _rope(name, lens, axes=(64,), **kw):
    return dict(dict(name=name, op="rope", dtype="bf16", d=128, hq=28, hkv=4, lens=_text(lens), rot=128, layout="half",
                     axes=_text(axes), norm=False, factor=1.0, start=0, qkv=True), **kw)


def _attn(name, q_lens, kv_lens, **kw):
    return dict(dict(name=name, op="attn", dtype="bf16", d=128, hq=28, hkv=4, q_lens=_text(q_lens), kv_lens=_text(kv_lens),
                     packed=False, qkv=False), **kw)


def listed():
    return [
        # One decoded token of a 7B geometry in front of the decode attention: launch latency.
        _rope("rope-token", [1], start=7432),
        # A decode step of 16 sequences far into their contexts, normalised heads.
        _rope("rope-batch-step", [1] * 16, norm=True, start=200_000, factor=8.0),
        # The prompt of one large image: positions of time, row and column, rows laid out for scoring and compaction.
        _rope("rope-image-7b", [7432], axes=[16, 24, 24]),
        # Two long prompts of a 72B geometry, half of every head rotated, neighbours paired, normalised, frequencies stretched.
        _rope("rope-long-72b", [16910, 16001], hq=64, hkv=8, rot=64, axes=[32], layout="interleaved", norm=True, factor=4.0),
        # Full-precision check of a small model: heads of 64 elements.
        _rope("rope-f32-d64", [656, 131], dtype="f32", d=64, hq=4, hkv=2, rot=64, axes=[32], qkv=False, norm=True),
        # One token over the whole prompt's cache, before compression or without it: bound by one pass over K and V.
        _attn("attn-token", [1], [7432]),
        # A step of eight sequences of differing lengths, small model with heads of 64 elements.
        _attn("attn-step-d64", [1] * 8, [7432, 1601, 257, 4000, 33, 901, 6000, 2500], d=64, hq=14, hkv=2),
        # Full-precision check of a small model: 656 tokens.
        _attn("attn-f32-d64", [656, 131], [656, 131], dtype="f32", d=64, hq=4, hkv=2),
        # The prompt of one large image, 7B geometry, read from the projection's packed output.
        _attn("attn-image-7b", [7432], [7432], qkv=True),
        # Sixteen prompts of differing lengths packed one behind the other.
        _attn("attn-packed-16", *[[2574, 2391, 2702, 2433, 2811, 2320, 2575, 2499, 2640, 2350, 2777, 2512, 2603, 2448, 2699, 2361]] * 2,
              packed=True, qkv=True),
        # A piece of 512 tokens of a long prompt over the keys before it, 72B geometry.
        _attn("attn-piece-72b", [512], [16910], hq=64, hkv=8),
        # Two long prompts of a 72B geometry: the largest.
        _attn("attn-long-72b", [16910, 16001], [16910, 16001], hq=64, hkv=8),
    ]


def _cost(case):
    w = work(case)
    return w["bytes"] / 4e12 + w["flops"] * (1 if case["dtype"] == "bf16" else 8) / 4e14


def draw(rng):
    """Another case of the same ranges: sizes spread over their logarithm, odd ones among them."""
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    largest = max(map(_cost, listed()))
    while True:
        dtype, d = rng.choice([("bf16", 128)] * 5 + [("bf16", 64)] * 3 + [("f32", 64), ("f32", 128)])
        hkv, g = rng.choice([(4, 7), (2, 7), (8, 8), (2, 2), (8, 4), (4, 8), (1, 12), (3, 5), (8, 1), (1, 16)])
        batch = rng.choice([1, 1, 1, 2, 3, 4, 8, 16, 33])
        common = dict(dtype=dtype, d=d, hq=hkv * g, hkv=hkv, qkv=rng.random() < 0.5)
        top = log_int(1, 16910)
        lens = [max(1, round(top * rng.uniform(0.3, 1.0))) for _ in range(batch)]
        lens[rng.randrange(batch)] = top
        if rng.random() < 0.4:
            rot = rng.choice([d] * 3 + list(range(16, d, 16)))
            pairs = rot // 2
            axes = [pairs] if rng.random() < 0.7 or pairs < 16 else [pairs - 2 * (pairs * 3 // 8), pairs * 3 // 8, pairs * 3 // 8]
            c = _rope(None, [1] * batch if rng.random() < 0.3 else lens, rot=rot, axes=axes, layout=rng.choice(["half", "half", "interleaved"]),
                      norm=rng.random() < 0.5, factor=rng.choice([1.0, 1.0, 4.0, 8.0, 32.0]), start=rng.choice([0, 0, log_int(1, 1_000_000)]), **common)
        else:
            kind = rng.choice(["prompt"] * 3 + ["piece", "token"])
            q_lens = lens if kind == "prompt" else [1] * batch if kind == "token" else [min(n, log_int(2, 2048)) for n in lens]
            c = _attn(None, q_lens, lens, packed=rng.random() < 0.5, **common)
            if kind != "prompt":
                c["qkv"] = False
        del c["name"]
        if _cost(c) <= largest:
            return c


def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device=gen.device, dtype=torch.float32)


def _buffers(case, q, k, v):
    """q, k, v in the case's memory order."""
    dt = _type(case)
    if not case["qkv"]:
        return q.to(dt), k.to(dt), v.to(dt)
    both = torch.cat([q.to(dt), k.to(dt), v.to(dt)], dim=1).transpose(1, 2).contiguous().transpose(1, 2)
    hq, hkv = case["hq"], case["hkv"]
    return both[:, :hq], both[:, hq:hq + hkv], both[:, hq + hkv:]


def _frequencies(rot, factor):
    """Turns of the position per pair, in radians: theta^(-2i / rot); with a factor the pairs of fewer than one turn in 32768
    positions are slowed down by it, those of more than 32 turns stay, and the ones between go over linearly."""
    f = [THETA ** (-2.0 * i / rot) for i in range(rot // 2)]
    if factor == 1.0:
        return f
    share = [min(1.0, max(0.0, (x * 32768 / (2 * math.pi) - 1.0) / 31.0)) for x in f]
    return [x * s + x / factor * (1.0 - s) for x, s in zip(f, share)]


def _positions(case, device):
    """[axes][B][tokens], -1 behind a sequence.  Three axes: 14 tokens of text, then an image of rows of 60, then text again."""
    tokens = max(_ints(case["lens"]))
    t = torch.arange(tokens, device=device)
    lens = torch.tensor(_ints(case["lens"]), device=device)[:, None]
    if len(_ints(case["axes"])) == 1:
        p = t[None, None, :].expand(1, len(_ints(case["lens"])), -1) + case["start"]
    else:
        image = (t >= 14) & (t < max(14, tokens - 128))
        row, col = (t - 14) // 60, (t - 14) % 60
        after = t - torch.clamp(image.sum() - 60, min=0)
        flat = torch.where(t < 14, t, after)
        p = torch.stack([torch.where(image, 14, flat), torch.where(image, 14 + row, flat), torch.where(image, 14 + col, flat)])
        p = p[:, None, :].expand(-1, len(_ints(case["lens"])), -1) + case["start"]
    return torch.where(t[None, None, :] < lens[None], p, -1).to(torch.int32).contiguous()


def _rope_inputs(case, seed):
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(seed)
    B, T, d, hq, hkv = len(_ints(case["lens"])), max(_ints(case["lens"])), case["d"], case["hq"], case["hkv"]
    # projections: heads of differing size, a few large elements as trained models have
    size = 0.5 + 1.5 * torch.rand((1, hq + 2 * hkv, 1, d), generator=gen, device=gen.device)
    x = _randn(gen, B, hq + 2 * hkv, T, d) * size
    q, k, v = _buffers(case, x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:])
    weights = [(1.0 + 0.2 * _randn(gen, d)).to(_type(case)) for _ in range(2)]
    return q, k, v, weights


def _attn_inputs(case, seed):
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(seed)
    d, hq, hkv = case["d"], case["hq"], case["hkv"]
    B, nq, nk = len(_ints(case["q_lens"])), max(_ints(case["q_lens"])), max(_ints(case["kv_lens"]))
    if case["packed"]:
        B, nq, nk = 1, sum(_ints(case["q_lens"])), sum(_ints(case["kv_lens"]))
    # queries lean to a direction that a share of the keys has: peaked rows, as attention over images has
    u = _randn(gen, B, hkv, 1, d)
    u /= u.norm(dim=-1, keepdim=True)
    lean = 3.0 * (torch.rand((B, hkv, nk, 1), generator=gen, device=gen.device) < 0.05)
    q = _randn(gen, B, hq, nq, d) + 0.15 * d * u.repeat_interleave(hq // hkv, dim=1)
    k = _randn(gen, B, hkv, nk, d) + lean * u
    v = _randn(gen, B, hkv, nk, d)
    return _buffers(case, q, k, v)


def _spans(case):
    """(batch row, first query, queries, first key, keys) of every sequence."""
    out, q0, k0 = [], 0, 0
    for b, (n, m) in enumerate(zip(_ints(case["q_lens"]), _ints(case["kv_lens"]))):
        out.append((0, q0, n, k0, m) if case["packed"] else (b, 0, n, 0, m))
        q0, k0 = q0 + n, k0 + m
    return out


def prepare(case, seed):
    if case["op"] == "rope":
        q, k, v, (qw, kw) = _rope_inputs(case, seed)
        B, T, d = q.shape[0], q.shape[2], case["d"]
        st = dict(case=case, q=q, k=k, v=v, qw=qw if case["norm"] else None, kw=kw if case["norm"] else None,
                  positions=_positions(case, q.device),
                  freqs=torch.tensor(_frequencies(case["rot"], case["factor"]), dtype=torch.float64, device=q.device),
                  scale=0.1 * math.log(case["factor"]) + 1.0,
                  # outputs as scoring, compaction and decode take them; zero where padding is left as it is
                  out=[torch.zeros((B, x.shape[1], T, d), dtype=x.dtype, device=x.device) for x in (q, k, v)])
        if own:
            import paper_2503_23956_amd as A
            st["call"] = A.prepare_rope(q, k, v, *st["out"], positions=st["positions"], freqs=st["freqs"], axis_pairs=_ints(case["axes"]),
                                        layout=A.AIR_ROPE_HALF if case["layout"] == "half" else A.AIR_ROPE_INTERLEAVED,
                                        q_weight=st["qw"], k_weight=st["kw"], eps=1e-6, scale=st["scale"])
        return st
    q, k, v = _attn_inputs(case, seed)
    out = torch.zeros((q.shape[0], q.shape[2], case["hq"], case["d"]), dtype=q.dtype, device=q.device).transpose(1, 2)
    st = dict(case=case, q=q, k=k, v=v, out=out)
    if own:
        import paper_2503_23956_amd as A
        st["call"] = A.prepare_prompt_attn(q, k, v, out, spans=_spans(case))
    return st


def _plain_rope(st):
    case = st["case"]
    rot, pairs = case["rot"], case["rot"] // 2
    axis = torch.repeat_interleave(torch.arange(len(_ints(case["axes"]))), torch.tensor(_ints(case["axes"]))).to(st["q"].device)
    angle = st["positions"][axis].permute(1, 2, 0).double() * st["freqs"]  # [B][token][pair]
    angle = torch.remainder(angle, 2 * math.pi)
    cos = (torch.cos(angle).float() * st["scale"])[:, None]
    sin = (torch.sin(angle).float() * st["scale"])[:, None]
    real = (st["positions"][0] >= 0)[:, None, :, None]

    def rotated(x, w):
        y = x.float()
        if w is not None:
            y = y * torch.rsqrt(y.square().mean(dim=-1, keepdim=True) + 1e-6) * w.float()
        half = case["layout"] == "half"
        a, b = (y[..., :pairs], y[..., pairs:rot]) if half else (y[..., 0:rot:2], y[..., 1:rot:2])
        ra, rb = a * cos - b * sin, a * sin + b * cos
        r = torch.cat([ra, rb], dim=-1) if half else torch.stack([ra, rb], dim=-1).flatten(-2)
        return torch.where(real, torch.cat([r, y[..., rot:]], dim=-1), 0.0).to(x.dtype)

    return [rotated(st["q"], st["qw"]), rotated(st["k"], st["kw"]), torch.where(real, st["v"], 0.0).contiguous()]


def _plain_attn(st):
    case = st["case"]
    d, hq, hkv = case["d"], case["hq"], case["hkv"]
    g = hq // hkv
    out = torch.zeros_like(st["out"])
    for b, q0, n, k0, m in _spans(case):
        k = st["k"][b, :, k0:k0 + m].float().transpose(1, 2).contiguous()
        v = st["v"][b, :, k0:k0 + m].float().contiguous()
        rows = max(1, int(2 ** 29 / (hq * m)))  # query rows at a time: 2 GB of logits
        for r0 in range(0, n, rows):
            r1 = min(n, r0 + rows)
            q = st["q"][b, :, q0 + r0:q0 + r1].float().reshape(hkv, g * (r1 - r0), d)
            s = (q @ k).view(hkv, g, r1 - r0, m) / math.sqrt(d)
            last = torch.arange(r0, r1, device=s.device) + (m - n)
            s = s.masked_fill(torch.arange(m, device=s.device)[None, :] > last[:, None], -math.inf)
            p = torch.exp(s - s.amax(dim=-1, keepdim=True))
            o = (p.view(hkv, g * (r1 - r0), m) @ v).view(hkv, g, r1 - r0, d) / p.sum(dim=-1, keepdim=True)
            out[b, :, q0 + r0:q0 + r1] = o.view(hq, r1 - r0, d).to(out.dtype)
    return out


def run(st):
    if own:
        import paper_2503_23956_amd as A
        if st["case"]["op"] == "rope":
            A.air_rope(prepared=st["call"])
        else:
            A.air_prompt_attn(prepared=st["call"])
        return st["out"]
    return _plain_rope(st) if st["case"]["op"] == "rope" else _plain_attn(st)


def work(case):
    """rope: every element of q, k, v read and written once, the positions once; a square and a product per element where
    normalised and six operations per rotated pair.  attn: q, k, v read and the outputs written once; two products of d
    per head and pair of a query and a key that it sees."""
    e, d, hq, hkv = 2 if case["dtype"] == "bf16" else 4, case["d"], case["hq"], case["hkv"]
    if case["op"] == "rope":
        n = sum(_ints(case["lens"]))
        return {"bytes": n * (2.0 * (hq + 2 * hkv) * d * e + 4 * len(_ints(case["axes"]))),
                "flops": n * (hq + hkv) * ((4.0 * d if case["norm"] else 0.0) + 3.0 * case["rot"])}
    seen = sum(n * (m - n) + n * (n + 1) / 2 for n, m in zip(_ints(case["q_lens"]), _ints(case["kv_lens"])))
    return {"bytes": 2.0 * d * e * (sum(_ints(case["q_lens"])) * hq + sum(_ints(case["kv_lens"])) * hkv), "flops": 4.0 * d * hq * seen}


def exact(case, seed):
    """The operators' definitions in fp64, a head at a time."""
    if case["op"] == "rope":
        q, k, v, (qw, kw) = _rope_inputs(case, seed)
        pos = _positions(case, q.device)
        freqs = _frequencies(case["rot"], case["factor"])
        gain = 0.1 * math.log(case["factor"]) + 1.0
        tables, pair = [], 0
        for axis, count in enumerate(_ints(case["axes"])):
            for _ in range(count):
                turn = torch.exp(1j * (pos[axis].double() * freqs[pair]).to(torch.complex128))
                tables.append(gain * turn)
                pair += 1
        turn = torch.stack(tables, dim=-1)  # [B][token][pair]
        pad = pos[0] < 0
        rot, out = case["rot"], []
        for x, w in ((q, qw), (k, kw), (v, None)):
            y = x.double()
            if x is not v:
                if case["norm"]:
                    y = y / (y.pow(2).sum(dim=-1, keepdim=True) / case["d"] + 1e-6).sqrt() * w.double()
                first, second = ((slice(0, rot // 2), slice(rot // 2, rot)) if case["layout"] == "half"
                                 else (slice(0, rot, 2), slice(1, rot, 2)))
                z = torch.complex(y[..., first], y[..., second]) * turn[:, None]
                y = y.clone()
                y[..., first], y[..., second] = z.real, z.imag
            out.append(y.masked_fill(pad[:, None, :, None], 0.0))
        return out
    q, k, v = _attn_inputs(case, seed)
    g = case["hq"] // case["hkv"]
    shape = (q.shape[0], q.shape[2], case["hq"], case["d"])
    out = torch.zeros(shape, dtype=torch.float64, device=q.device).transpose(1, 2)
    for b, q0, n, k0, m in _spans(case):
        for h in range(case["hq"]):
            kh, vh = (x[b, h // g, k0:k0 + m].double() for x in (k, v))
            for r in range(0, n, 4096):
                qh = q[b, h, q0 + r:q0 + min(n, r + 4096)].double()
                s = qh @ kh.t().contiguous() * case["d"] ** -0.5
                behind = torch.ones_like(s, dtype=torch.bool).triu_(diagonal=m - n + r + 1)
                out[b, h, q0 + r:q0 + r + len(qh)] = torch.softmax(s.masked_fill_(behind, -math.inf), dim=1) @ vh
    return out
