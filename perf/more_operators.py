"""Operators of a cache that is generated into: rows of K and V held in 4 bits (`air_quant_append`, `air_quant_read`), attention that
reads them and leaves what every slot was attended to (`air_quant_attn`), and eviction by those weights (`air_evict`), beside their plain forms.

Tensors are indexed [B][head][token or slot][d].  Fields of a case: op; dtype and d; hq query heads over hkv KV heads; group: elements
of a row that share a step; `held`: slots of every sequence that hold a token before the call.

A group of a row is held as  lo = its least element, rounded down to bf16;  step = (greatest - lo) / 15, rounded up to bf16 (0 below
2^-120);  code = round((x - lo) / step), where the difference, the division by 15 and the quotient are each rounded to fp32.  It
stands for lo + step code.

store: `lens` rows of every sequence go behind those held, and are read back.  token_major: K and V are views of one projection's
output [B][token][2 hkv][d].
attn: q_lens queries of every sequence (rows behind a shorter one's are padding, left as they are) over the slots held; append: their own keys
and values go into the cache first; causal: query t of n sees all but the last n - 1 - t slots, else all; weigh: the sum of the
probabilities that a KV head's queries give a slot is added to the slot's weight.
evict: sequences with more than `limit` slots keep `keep` of them: the tokens at the `first` lowest and `recent` highest positions, then those of the
largest weights, ties to the lower slot.  Slots in front of `keep` that are given up take, in order, the tokens kept behind it.  rows: the cache holds
K and V as they are; else in 4 bits, and what is kept is read back.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False  # True: `run` calls the library; False: the operators in elementary torch operations


def _text(numbers):
    """A list of whole numbers as a case holds it."""
    return " ".join(map(str, numbers))


def _ints(text):
    return [int(x) for x in text.split()]


def _store(name, lens, held=None, **kw):
    return dict(dict(name=name, op="store", dtype="bf16", d=128, hkv=4, group=32, lens=_text(lens), held=_text(held or [0] * len(lens)),
                     token_major=False), **kw)


def _attn(name, q_lens, held, **kw):
    return dict(dict(name=name, op="attn", dtype="bf16", d=128, hq=28, hkv=4, group=32, q_lens=_text(q_lens), held=_text(held), append=True,
                     causal=True, weigh=False), **kw)


def _evict(name, held, keep, limit, **kw):
    return dict(dict(name=name, op="evict", dtype="bf16", d=128, hkv=4, group=32, held=_text(held), keep=keep, limit=limit, first=4, recent=64,
                     rows=False), **kw)


RAGGED = [2574, 2391, 2702, 2433, 2811, 2320, 2575, 2499, 2640, 2350, 2777, 2512, 2603, 2448, 2699, 2361]


def listed():
    return [
        # One generated token of sixteen sequences: launch latency.
        _store("store-step-16", [1] * 16, RAGGED),
        # The prompt of one large image, 7B geometry, as the projection leaves it.
        _store("store-image-7b", [7432], token_major=True),
        # Two long prompts of a 72B geometry.
        _store("store-long-72b", [16910, 16001], hkv=8, group=64),
        # One token over the whole prompt's cache: latency, and one pass over K and V.
        _attn("attn-token", [1], [7432]),
        # A step of eight sequences of differing lengths, small model with heads of 64 elements, weights for a later eviction.
        _attn("attn-step-d64", [1] * 8, [7432, 1601, 257, 4000, 33, 901, 6000, 2500], d=64, hq=14, hkv=2, weigh=True),
        # A step of sixteen long sequences, 72B geometry: bound by reading the cache.
        _attn("attn-step-72b", [1] * 16, [16910, 16001, 15007, 16500, 16384, 14001, 16777, 15555] * 2, hq=64, hkv=8, weigh=True),
        # Full-precision check of a small model: the last 32 tokens of two prompts weigh the slots in front of a first eviction.
        _attn("attn-window-f32", [32, 17], [656, 131], dtype="f32", d=64, hq=4, hkv=2, append=False, causal=False, weigh=True),
        # A piece of 500 tokens behind a prompt that is held already.
        _attn("attn-piece-7b", [500], [7432], group=64),
        # Windows of 64 queries over eight long prompts, 72B geometry, to weigh their slots: the largest.
        _attn("attn-window-72b", [64] * 8, [16910, 16001, 15007, 16500, 16384, 14001, 16777, 15555], hq=64, hkv=8, append=False, weigh=True),
        # A serving step: sixteen sequences, those that have grown by 64 tokens behind 2304 give up 64.
        _evict("evict-step-16", [2368, 2331, 2368, 2304, 2350, 2368, 2310, 2367] * 2, 2304, 2367, rows=True),
        # After the prompt of one large image: a tenth stays, read back from 4 bits.
        _evict("evict-image-7b", [7432], 743, 743),
        # Two long prompts of a 72B geometry cut to half.
        _evict("evict-long-72b", [16910, 16001], 8192, 8192, hkv=8, group=64),
    ]


def _cost(case):
    w = work(case)
    return w["bytes"] / 4e12 + w["flops"] * (1 if case["dtype"] == "bf16" else 8) / 2e14


def draw(rng):
    """Another case of the same ranges: sizes spread over their logarithm, odd ones among them."""
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["store", "attn", "attn", "evict"])
    largest = max(_cost(c) for c in listed() if c["op"] == op)
    while True:
        dtype, d = rng.choice([("bf16", 128)] * 5 + [("bf16", 64)] * 3 + [("f32", 64), ("f32", 128)])
        hkv, g = rng.choice([(4, 7), (2, 7), (8, 8), (2, 2), (8, 4), (4, 8), (1, 12), (3, 5), (8, 1), (1, 16)])
        batch = rng.choice([1, 1, 1, 2, 3, 4, 8, 16, 33])
        common = dict(dtype=dtype, d=d, hkv=hkv, group=rng.choice([32, 64]))
        top = log_int(1, 16910)
        held = [max(1, round(top * rng.uniform(0.3, 1.0))) for _ in range(batch)]
        held[rng.randrange(batch)] = top
        if op == "store":
            lens = [1] * batch if rng.random() < 0.3 else held
            c = _store(None, lens, [0] * batch if rng.random() < 0.5 else [rng.randint(0, 500) for _ in range(batch)],
                       token_major=rng.random() < 0.5, **common)
        elif op == "attn":
            n = rng.choice([1, 1, 1, log_int(2, 64), log_int(2, 512)])
            c = _attn(None, [max(1, round(n * rng.uniform(0.5, 1.0))) for _ in range(batch)], held, hq=hkv * g, append=rng.random() < 0.5,
                      causal=rng.random() < 0.7, weigh=rng.random() < 0.5, **common)
            if not c["append"]:  # a call without rows of its own has at most as many queries as slots
                c["q_lens"] = _text([min(a, b) for a, b in zip(_ints(c["q_lens"]), held)])
        else:
            keep = max(1, round(top * rng.uniform(0.05, 0.95)))
            first = rng.randint(0, min(8, keep // 4))
            c = _evict(None, held, keep, rng.randint(keep, max(keep, top - 1)), first=first, recent=rng.randint(0, (keep - first) // 2),
                       rows=rng.random() < 0.5, **common)
        del c["name"]
        if _cost(c) <= largest:
            return c


# ---- inputs ------------------------------------------------------------------------------------------------------------------
def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device=gen.device, dtype=torch.float32)


def _device_ints(numbers, device):
    return torch.tensor(numbers, dtype=torch.int32, device=device)


def _rows(gen, case, n):
    """Keys with channels of differing size and offset, as trained models have them, and values; in the case's type."""
    shape, d = (len(_ints(case["held"])), case["hkv"], n, case["d"]), case["d"]
    size = 0.5 + 1.5 * torch.rand((1, case["hkv"], 1, d), generator=gen, device=gen.device)
    offset = 3.0 * _randn(gen, 1, case["hkv"], 1, d) * (torch.rand((1, case["hkv"], 1, d), generator=gen, device=gen.device) < 0.05)
    return (_randn(gen, *shape) * size + offset).to(_type(case)), _randn(gen, *shape).to(_type(case))


def _slots(case):
    """Slots of the case's cache: what it takes after the call, and a few more."""
    new = case["lens"] if case["op"] == "store" else case["q_lens"] if case["op"] == "attn" and case["append"] else ""
    return max(_ints(case["held"])) + max(_ints(new), default=0) + 5


def _inputs(case, seed):
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(seed)
    held, hkv = _ints(case["held"]), case["hkv"]
    B, slots = len(held), _slots(case)
    x = {}
    if case["op"] == "store":
        k, v = _rows(gen, case, max(_ints(case["lens"])))
        if case["token_major"]:
            both = torch.cat([k, v], dim=1).transpose(1, 2).contiguous().transpose(1, 2)
            k, v = both[:, :hkv], both[:, hkv:]
        return dict(k=k, v=v)
    x["held_k"], x["held_v"] = _rows(gen, case, max(held))
    # what a slot was attended to until now: heavy-tailed, some never
    weights = torch.exp(2.0 * _randn(gen, B, hkv, slots))
    x["weights"] = weights * (torch.rand(weights.shape, generator=gen, device=gen.device) < 0.95)
    order = torch.arange(slots, device=gen.device)
    if case["op"] == "evict":  # slots of an earlier eviction hold later tokens than their neighbours
        swapped = torch.argsort(order + 40.0 * torch.rand((B, hkv, slots), generator=gen, device=gen.device), dim=-1)
        x["positions"] = swapped.to(torch.int32)
        return x
    x["positions"] = order.to(torch.int32).expand(B, hkv, -1).contiguous()
    n = max(_ints(case["q_lens"]))
    # queries lean to a direction that a share of the keys has: peaked rows, as attention over images has
    lean = _randn(gen, B, hkv, 1, case["d"])
    lean /= lean.norm(dim=-1, keepdim=True)
    q = _randn(gen, B, case["hq"], n, case["d"]) + 0.15 * case["d"] * lean.repeat_interleave(case["hq"] // hkv, dim=1)
    x["q"] = q.to(_type(case)).transpose(1, 2).contiguous().transpose(1, 2)
    toward = 3.0 * (torch.rand((B, hkv, max(held), 1), generator=gen, device=gen.device) < 0.05)
    x["held_k"] = (x["held_k"].float() + toward * lean).to(_type(case))
    if case["append"]:
        x["k"], x["v"] = _rows(gen, case, n)
    return x


def prepare(case, seed):
    x = _inputs(case, seed)
    dev, held, dt = torch.device("cuda:0"), _ints(case["held"]), _type(case)
    B, hkv, d, slots, group = len(held), case["hkv"], case["d"], _slots(case), case["group"]
    st = dict(case=case, x=x, lens=_device_ints(held, dev))
    if case["op"] == "store":
        n = max(_ints(case["lens"]))
        st["counts"] = _device_ints(_ints(case["lens"]), dev)
        st["out"] = [torch.zeros((B, hkv, n, d), dtype=dt, device=dev) for _ in range(2)]
    elif case["op"] == "attn":
        n = max(_ints(case["q_lens"]))
        st["counts"] = _device_ints(_ints(case["q_lens"]), dev)
        st["out"] = torch.zeros((B, n, case["hq"], d), dtype=dt, device=dev).transpose(1, 2)
    else:
        st["lens_out"] = torch.zeros_like(st["lens"])
        if case["rows"]:
            st["rows"] = [torch.zeros((B, hkv, slots, d), dtype=dt, device=dev) for _ in range(2)]
            for to, rows in zip(st["rows"], (x["held_k"], x["held_v"])):
                to[:, :, :rows.shape[2]] = rows
        else:
            st["out"] = [torch.zeros((B, hkv, case["keep"], d), dtype=dt, device=dev) for _ in range(2)]
    if own:
        import paper_2503_23956_amd as A
        if not case.get("rows"):
            st["cache"] = A.QuantCache(B, hkv, slots, d, A.AIR_BF16 if case["dtype"] == "bf16" else A.AIR_F32, group=group, device=dev)
            if case["op"] != "store":
                A.air_quant_append(st["cache"], x["held_k"], x["held_v"], lens=torch.zeros_like(st["lens"]), counts=st["lens"])
        if case["op"] == "store":
            st["call"] = A.prepare_quant_append(st["cache"], x["k"], x["v"], lens=st["lens"], counts=st["counts"])
            st["read"] = A.prepare_quant_read(st["cache"], *st["out"], starts=st["lens"], counts=st["counts"])
        elif case["op"] == "attn":
            st["call"] = A.prepare_quant_attn(st["cache"], x["q"], st["out"], lens=st["lens"], counts=st["counts"], k=x.get("k"), v=x.get("v"),
                                              causal=case["causal"], weights=x["weights"] if case["weigh"] else None,
                                              positions=x["positions"] if case["append"] else None,
                                              first_positions=st["lens"] if case["append"] else None, max_len=slots)
        else:
            planes = st["rows"] if case["rows"] else st["cache"].planes
            st["call"] = A.prepare_evict(planes, x["weights"], positions=x["positions"], lens=st["lens"], lens_out=st["lens_out"],
                                         keep=case["keep"], limit=case["limit"], first=case["first"], recent=case["recent"])
            if not case["rows"]:
                st["read"] = A.prepare_quant_read(st["cache"], *st["out"], starts=None, counts=st["lens_out"])
    elif not case.get("rows"):
        # the plain cache: two codes a byte, lo and step of every group
        st["planes"] = [torch.zeros((B, hkv, slots, n), dtype=t, device=dev)
                        for n, t in ((d // 2, torch.uint8), (d // group, torch.bfloat16), (d // group, torch.bfloat16)) * 2]
        if case["op"] != "store":
            for i, rows in enumerate((x["held_k"], x["held_v"])):
                for to, part in zip(st["planes"][3 * i:], _packed(rows, group)):
                    to[:, :, :rows.shape[2]] = part
    return st


# ---- plain forms ---------------------------------------------------------------------------------------------------------------
def _packed(x, group):
    """(codes, two a byte; lo; step) of rows."""
    y = x.float().unflatten(-1, (-1, group))
    least = y.amin(dim=-1)
    bits = least.view(torch.int32)
    lo = torch.where((bits < 0) & (bits & 0xFFFF != 0), (bits & -0x10000) + 0x10000, bits & -0x10000).view(torch.float32)
    width = y.amax(dim=-1) - lo
    step = ((width / torch.full_like(width, 15.0)).view(torch.int32) + 0xFFFF & -0x10000).view(torch.float32)  # (a division, not a product with 1 / 15)
    step = torch.where(step < 2.0 ** -120, 0.0, step)
    share = (y - lo[..., None]) / step[..., None]
    code = torch.where(step[..., None] > 0, torch.round(share), 0.0).clamp(0, 15).flatten(-2).to(torch.uint8)
    return code[..., 0::2] | code[..., 1::2] << 4, lo.to(torch.bfloat16), step.to(torch.bfloat16)


def _unpacked(codes, lo, step):
    """What the codes stand for, in fp32."""
    c = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2).float().unflatten(-1, (lo.shape[-1], -1))
    return (lo.float()[..., None] + step.float()[..., None] * c).flatten(-2)


def _put(planes, k, v, lens, counts, group):
    """Rows t < counts of k and v into slots lens + t."""
    t = torch.arange(k.shape[2], device=k.device)
    b, t = torch.nonzero(t[None, :] < counts[:, None], as_tuple=True)
    at = lens[b].long() + t
    for i, rows in enumerate((k, v)):
        for to, part in zip(planes[3 * i:], _packed(rows, group)):
            to.transpose(1, 2)[b, at] = part.transpose(1, 2)[b, t]
    return b, t, at


def _plain_store(st):
    x, case = st["x"], st["case"]
    b, t, at = _put(st["planes"], x["k"], x["v"], st["lens"], st["counts"], case["group"])
    for i, out in enumerate(st["out"]):
        out.transpose(1, 2)[b, t] = _unpacked(*(p.transpose(1, 2)[b, at] for p in st["planes"][3 * i:3 * i + 3])).to(out.dtype)
    return {"k": st["out"][0], "v": st["out"][1]}


def _plain_attn(st):
    x, case = st["x"], st["case"]
    hkv, d, n = case["hkv"], case["d"], max(_ints(case["q_lens"]))
    g, B = case["hq"] // hkv, len(_ints(case["held"]))
    lens = st["lens"]
    if case["append"]:
        b, t, at = _put(st["planes"], x["k"], x["v"], lens, st["counts"], case["group"])
        x["positions"].transpose(1, 2)[b, at] = (lens[b] + t).to(torch.int32)[:, None]
        if case["weigh"]:
            x["weights"].transpose(1, 2)[b, at] = 0.0
        lens = lens + st["counts"]
    k, v = (_unpacked(*st["planes"][3 * i:3 * i + 3]) for i in range(2))
    slot, t = torch.arange(k.shape[2], device=k.device), torch.arange(n, device=k.device)
    seen = lens[:, None].expand(-1, n)
    if case["causal"]:
        seen = seen - st["counts"][:, None] + t + 1
    real = t < st["counts"][:, None]  # [B][n]
    hidden = (slot >= seen[..., None]) | ~real[..., None]  # [B][n][slot]
    held = slot < lens[:, None]
    v = torch.where(held[:, None, :, None], v, 0.0)
    s = (x["q"].float().reshape(B, hkv, g * n, d) @ k.transpose(-1, -2)).view(B, hkv, g, n, -1) / math.sqrt(d)
    s = s.masked_fill(hidden[:, None, None], -math.inf)
    p = torch.exp(s - s.amax(dim=-1, keepdim=True).clamp(min=-1e30))
    p = p / p.sum(dim=-1, keepdim=True).clamp(min=1e-30)
    out = (p.view(B, hkv, g * n, -1) @ v).view(B, hkv * g, n, d)
    st["out"].copy_(torch.where(real[:, None, :, None], out, st["out"].float()))
    got = {"out": st["out"]}
    if case["weigh"]:
        x["weights"] += p.sum(dim=(2, 3))
        got["weights"] = x["weights"]
    if case["append"]:
        got["positions"] = x["positions"]
    return got


def _plain_evict(st):
    x, case = st["x"], st["case"]
    keep, lens = case["keep"], st["lens"]
    weights, positions = x["weights"], x["positions"]
    slot = torch.arange(weights.shape[2], device=weights.device)
    over = (lens > case["limit"])[:, None, None]
    held = (slot < lens[:, None])[:, None]
    last = torch.where(held, positions, -1).amax(dim=-1, keepdim=True)
    safe = (positions < case["first"]) | (positions > last - case["recent"])
    key = torch.where(held, torch.where(safe, math.inf, weights), -math.inf)
    order = torch.sort(key, dim=-1, descending=True, stable=True).indices
    kept = torch.zeros_like(held.expand_as(key)).scatter(-1, order[..., :keep], True)
    hole, moved = ~kept & (slot < keep) & over, kept & (slot >= keep) & over
    b, h, to = torch.nonzero(hole, as_tuple=True)
    source = torch.nonzero(moved, as_tuple=True)  # as many, in the same order of sequences, heads and slots
    for plane in [weights, positions] + (st["rows"] if case["rows"] else st["planes"]):
        plane[b, h, to] = plane[source]
    st["lens_out"].copy_(torch.where(lens > case["limit"], keep, lens))
    got = {"lens": st["lens_out"], "weights": weights, "positions": positions}
    if case["rows"]:
        return dict(got, k=st["rows"][0], v=st["rows"][1])
    real = (torch.arange(keep, device=lens.device) < st["lens_out"][:, None])[:, None, :, None]
    for i, out in enumerate(st["out"]):
        out.copy_(torch.where(real, _unpacked(*(p[:, :, :keep] for p in st["planes"][3 * i:3 * i + 3])), out.float()))
    return dict(got, k=st["out"][0], v=st["out"][1])


def run(st):
    op = st["case"]["op"]
    if not own:
        return {"store": _plain_store, "attn": _plain_attn, "evict": _plain_evict}[op](st)
    import paper_2503_23956_amd as A
    x = st["x"]
    if op == "store":
        A.air_quant_append(prepared=st["call"])
        A.air_quant_read(prepared=st["read"])
        return {"k": st["out"][0], "v": st["out"][1]}
    if op == "attn":
        A.air_quant_attn(prepared=st["call"])
        got = {"out": st["out"]}
        if st["case"]["weigh"]:
            got["weights"] = x["weights"]
        if st["case"]["append"]:
            got["positions"] = x["positions"]
        return got
    A.air_evict(prepared=st["call"])
    got = {"lens": st["lens_out"], "weights": x["weights"], "positions": x["positions"]}
    if st["case"]["rows"]:
        return dict(got, k=st["rows"][0], v=st["rows"][1])
    A.air_quant_read(prepared=st["read"])
    return dict(got, k=st["out"][0], v=st["out"][1])


def work(case):
    """store: rows of K and V read, their codes and steps written and read, the values written.  attn: codes and steps of the slots read once,
    queries (and new rows) read and outputs written, weights read and written; two products of d per query head, query and slot that it
    sees.  evict: weights and positions of the sequences that give up slots read; of rows that move, as many as a random choice has on average,
    each read and written; what is kept in 4 bits read and its values written."""
    e, d, hkv = 2 if case["dtype"] == "bf16" else 4, case["d"], case["hkv"]
    packed, plain = 2 * hkv * (d / 2 + 4 * d / case["group"]), 2 * hkv * d * e  # bytes of a token, K and V
    held = _ints(case["held"])
    if case["op"] == "store":
        n = sum(_ints(case["lens"]))
        return {"bytes": 2.0 * n * (packed + plain), "flops": 2.0 * n * hkv * d * 6}
    if case["op"] == "attn":
        q = _ints(case["q_lens"])
        n = [h + c if case["append"] else h for h, c in zip(held, q)]
        seen = sum(c * m - (c * (c - 1) / 2 if case["causal"] else 0) for c, m in zip(q, n))
        return {"bytes": sum(n) * (packed + (8.0 * hkv if case["weigh"] else 0)) + sum(q) * (2.0 * case["hq"] * d * e + (plain if case["append"] else 0)),
                "flops": 4.0 * d * case["hq"] * seen}
    size, total = plain if case["rows"] else packed, 0.0
    for h in held:
        if h > case["limit"]:
            total += 8.0 * h * hkv + 2.0 * (size + 8 * hkv) * case["keep"] * (h - case["keep"]) / h
        if not case["rows"]:
            total += min(h, case["keep"] if h > case["limit"] else h) * (packed + plain)
    return {"bytes": total + 8.0 * len(held), "flops": sum(h for h in held if h > case["limit"]) * 4.0 * hkv}


# ---- the definitions in fp64 ---------------------------------------------------------------------------------------------------
def _values(x, group):
    """What rows stand for once they are held in 4 bits: fp64, from the definition, its roundings to fp32 and bf16 included."""
    y = x.double().unflatten(-1, (x.shape[-1] // group, group))

    def eight_bits(z, toward):
        part, power = torch.frexp(z)
        return torch.ldexp(toward(part * 256.0), power - 8)

    lo = eight_bits(y.min(dim=-1, keepdim=True).values, torch.floor)
    step = eight_bits(((y.max(dim=-1, keepdim=True).values - lo).float().double() / 15.0).float().double(), torch.ceil)
    step = step * (step >= 2.0 ** -120)
    share = ((y - lo).float().double() / torch.where(step > 0, step, 1.0)).float().double()
    return (lo + step * torch.clamp(torch.round(share), 0, 15)).flatten(-2)


def _exact_evict(case, x):
    weights, positions = x["weights"].double().cpu().numpy().copy(), x["positions"].cpu().numpy().copy()
    held, keep = _ints(case["held"]), case["keep"]
    B, hkv, slots = weights.shape
    new = np.array([keep if n > case["limit"] else n for n in held], dtype=np.int32)
    rows = [torch.zeros((B, hkv, slots, case["d"]), dtype=torch.float64, device=x["held_k"].device) for _ in range(2)]
    for to, r in zip(rows, (x["held_k"], x["held_v"])):
        to[:, :, :r.shape[2]] = r.double() if case["rows"] else _values(r, case["group"])
    for b, n in enumerate(held):
        for h in range(hkv) if n > case["limit"] else ():
            w, pos = weights[b, h, :n], positions[b, h, :n]
            safe = (pos < case["first"]) | (pos > pos.max() - case["recent"])
            best = np.lexsort((np.arange(n), -w, ~safe))[:keep]  # protected first, then by weight, then by slot
            into = np.setdiff1d(np.arange(keep), best)
            come = np.sort(best[best >= keep])
            weights[b, h, into], positions[b, h, into] = weights[b, h, come], positions[b, h, come]
            i, j = (torch.from_numpy(a).to(rows[0].device) for a in (into, come))
            for r in rows:
                r[b, h, i] = r[b, h, j]
    if not case["rows"]:
        rows = [r[:, :, :keep].clone() for r in rows]
        for b, n in enumerate(new):
            for r in rows:
                r[b, :, n:] = 0.0
    dev = rows[0].device
    return {"lens": torch.from_numpy(new).to(dev), "weights": torch.from_numpy(weights).to(dev), "positions": torch.from_numpy(positions).to(dev),
            "k": rows[0], "v": rows[1]}


def exact(case, seed):
    """The operators' definitions in fp64, a head at a time."""
    x = _inputs(case, seed)
    held, hkv, d = _ints(case["held"]), case["hkv"], case["d"]
    if case["op"] == "evict":
        return _exact_evict(case, x)
    if case["op"] == "store":
        out = [_values(x[name], case["group"]) for name in ("k", "v")]
        for b, n in enumerate(_ints(case["lens"])):
            for o in out:
                o[b, :, n:] = 0.0
        return {"k": out[0], "v": out[1]}
    q, counts, g = x["q"], _ints(case["q_lens"]), case["hq"] // hkv
    weights, positions = x["weights"].double(), x["positions"].clone()
    out = torch.zeros((q.shape[0], q.shape[2], case["hq"], d), dtype=torch.float64, device=q.device).transpose(1, 2)
    for b, (n, c) in enumerate(zip(held, counts)):
        for h in range(hkv):
            k, v = (x[name][b, h, :n] for name in ("held_k", "held_v"))
            if case["append"]:
                k, v = (torch.cat([r, x[name][b, h, :c]]) for r, name in ((k, "k"), (v, "v")))
                weights[b, h, n:n + c] = 0.0
                positions[b, h, n:n + c] = torch.arange(n, n + c, device=q.device)
            k, v = _values(k, case["group"]), _values(v, case["group"])
            for i in range(h * g, h * g + g):
                s = q[b, i, :c].double() @ k.t().contiguous() * d ** -0.5
                if case["causal"]:
                    s.masked_fill_(torch.ones_like(s, dtype=torch.bool).triu_(diagonal=len(k) - c + 1), -math.inf)
                p = torch.softmax(s, dim=1)
                out[b, i, :c] = p @ v
                weights[b, h, :len(k)] += p.sum(dim=0)
    got = {"out": out}
    if case["weigh"]:
        got["weights"] = weights
    if case["append"]:
        got["positions"] = positions
    return got
