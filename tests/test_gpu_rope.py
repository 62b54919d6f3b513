"""air_rope against its formulas in fp64, with bounds derived from the roundings it makes."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _plain(x, w, pos, freqs, axis_pairs, half, eps, scale):
    """fp64 rows and, per element, a bound on the error of computing them in fp32 with one rounding to x's type."""
    import torch

    y = x.double().cpu()
    d = y.shape[-1]
    rel = torch.zeros(())
    if w is not None:
        y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + eps) * w.double().cpu()
        # d fused sums, the mean's factor, eps, root, division and two products, each half a step of 2^-23
        rel = torch.tensor((d / 2 + 8) * 2.0 ** -24)
    pairs = sum(axis_pairs)
    out, err = y.clone(), rel * y.abs()
    if pairs:
        axis = np.repeat(np.arange(len(axis_pairs)), axis_pairs)
        angle = pos.double().cpu()[axis].permute(1, 2, 0) * freqs.double().cpu()
        cos, sin = torch.cos(angle)[:, None] * scale, torch.sin(angle)[:, None] * scale
        first, second = (slice(0, pairs), slice(pairs, 2 * pairs)) if half else (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2))
        a, b = y[..., first], y[..., second]
        out[..., first], out[..., second] = a * cos - b * sin, a * sin + b * cos
        # the fraction of a turn is rounded to 2^-25 (2 pi 2^-25 < 2^-22 rad), sine and cosine to 4 units of 2^-24 and times scale;
        # products and their sum to three more; fp64 angles of up to 2^21 rad: 2^-31
        each = scale * (2.0 ** -22 + 8 * 2.0 ** -24) + rel
        e = (a.abs() + b.abs()) * each
        err[..., first], err[..., second] = e, e
    step = 2.0 ** -8 if x.dtype == torch.bfloat16 else 2.0 ** -24
    return out, 1.01 * err + (out.abs() + err) * step + 1e-38


def _check(got, want, err, name):
    import torch

    far = (got.double().cpu() - want).abs()
    worst = (far - err).max().item()
    assert bool((far <= err).all()), f"{name}: {worst} above its bound"


def _inputs(B, T, hq, hkv, d, dtype, order, seed):
    """q, k, v as views of one packed buffer, of a token-major or of a head-major one."""
    import torch

    g = torch.Generator(device="cuda:0").manual_seed(seed)
    x = torch.randn((B, T, hq + 2 * hkv, d), generator=g, device="cuda:0").to(dtype)
    if order == "head":
        x = x.transpose(1, 2).contiguous()
    else:
        x = x.transpose(1, 2)
    return x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("half", [True, False])
@pytest.mark.parametrize("pairs", [(0,), (8,), (16,), (24,), (32,), (5, 11), (1, 6, 9), (8, 12, 12)])
def test_against_fp64(dtype, d, half, pairs):
    import torch

    import paper_2503_23956_amd as A

    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    if d == 128 and pairs == (32,):
        pairs = (64,)
    for B, T, hq, hkv, norm, order, start in ((1, 1, 5, 5, True, "packed", 700_001), (2, 33, 7, 1, False, "token", 0), (3, 43, 6, 3, True, "head", 12)):
        q, k, v = _inputs(B, T, hq, hkv, d, dt, order, 7 * T + d)
        g = torch.Generator(device="cuda:0").manual_seed(5)
        pos = torch.randint(0, 5000, (len(pairs), B, T), generator=g, device="cuda:0", dtype=torch.int32) + start
        freqs = torch.tensor(A.air_rope_frequencies(sum(pairs), 1e4)[0], device="cuda:0")
        qw, kw = ((1 + 0.3 * torch.randn(d, generator=g, device="cuda:0")).to(dt) for _ in range(2)) if norm else (None, None)
        outs = [torch.full((B, x.shape[1], T, d), math.nan, dtype=dt, device="cuda:0") for x in (q, k, v)]
        A.air_rope(q, k, v, *outs, positions=pos if sum(pairs) else None, freqs=freqs if sum(pairs) else None, axis_pairs=pairs,
                   layout=A.AIR_ROPE_HALF if half else A.AIR_ROPE_INTERLEAVED, q_weight=qw, k_weight=kw, eps=1e-5, scale=1.2)
        torch.cuda.synchronize()
        for x, w, o, name in ((q, qw, outs[0], "q"), (k, kw, outs[1], "k")):
            want, err = _plain(x, w, pos, freqs, pairs, half, 1e-5, 1.2)
            _check(o, want, err, f"{name} {B, T, hq, hkv, norm, order}")
        assert torch.equal(outs[2], v)


def test_padding_rows_are_left_as_they_are():
    import torch

    import paper_2503_23956_amd as A

    B, T, d = 3, 70, 128
    q, k, v = _inputs(B, T, 4, 2, d, torch.bfloat16, "token", 3)
    lens = [70, 1, 0]
    pos = torch.full((1, B, T), -1, dtype=torch.int32, device="cuda:0")
    for b, n in enumerate(lens):
        pos[0, b, :n] = torch.arange(n)
    freqs = torch.tensor(A.air_rope_frequencies(64, 1e4)[0], device="cuda:0")
    q, k, v = (x.clone() for x in (q, k, v))
    for x in (q, k, v):
        for b, n in enumerate(lens):
            x[b, :, n:] = math.nan
    outs = [torch.full_like(x, 42.0) for x in (q, k, v)]
    A.air_rope(q, k, v, *outs, positions=pos, freqs=freqs, axis_pairs=(64,))
    torch.cuda.synchronize()
    for x, o in zip((q, k, v), outs):
        for b, n in enumerate(lens):
            assert bool((o[b, :, n:] == 42.0).all()) and not bool(torch.isnan(o[b, :, :n]).any())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens", [1, 200])
def test_in_place_and_parts_of_the_call_give_the_same_bits(dtype, tokens):
    import torch

    import paper_2503_23956_amd as A

    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    for half in (A.AIR_ROPE_HALF, A.AIR_ROPE_INTERLEAVED):
        q, k, v = _inputs(2, tokens, 6, 3, 64, dt, "packed", 11)
        pos = torch.arange(2 * tokens, dtype=torch.int32, device="cuda:0").view(2, tokens)
        kw = dict(positions=pos, freqs=torch.tensor(A.air_rope_frequencies(24, 1e4)[0], device="cuda:0"), axis_pairs=(24,), layout=half)
        outs = [torch.zeros_like(x) for x in (q, k, v)]
        A.air_rope(q, k, v, *outs, **kw)
        alone = [torch.zeros_like(x) for x in (q, k, v)]
        A.air_rope(q, q_out=alone[0], **kw)
        A.air_rope(k=k, k_out=alone[1], **kw)
        A.air_rope(v=v, v_out=alone[2], **kw)
        A.air_rope(q, k, **kw)  # in place, inside one packed buffer
        torch.cuda.synchronize()
        for a, b, c in zip(outs, alone, (q, k, v)):
            assert torch.equal(a, b) and torch.equal(a, c)


def test_far_positions_turn_as_exactly_as_near_ones():
    """A whole number of turns further the same rotation: with a frequency of 2 pi / 64 positions p and p + 64 n agree."""
    import torch

    import paper_2503_23956_amd as A

    x = torch.randn(1, 1, 64, 64, device="cuda:0").expand(1, 1, 64, 64).contiguous()
    freqs = torch.full((32,), 2 * math.pi / 64, dtype=torch.float64, device="cuda:0")
    near = torch.arange(64, dtype=torch.int32, device="cuda:0").view(1, 64)
    outs = [torch.empty_like(x) for _ in range(2)]
    for o, add in zip(outs, (0, 64 * 30_000_000)):
        A.air_rope(x, q_out=o, positions=near + add, freqs=freqs, axis_pairs=(32,))
    # 1.9e9 positions are 1.9e8 rad: fp64 angles are good to 1.9e8 * 2^-52 = 4.2e-8 rad, the rest is the bound of the rotation
    bound = (x[..., :32].abs() + x[..., 32:].abs()) * (2 * 2.0 ** -22 + 16 * 2.0 ** -24 + 1e-7)
    far = (outs[0] - outs[1]).abs()
    assert bool((far <= torch.cat([bound, bound], -1)).all())


def test_graph_replays_and_other_streams():
    import torch

    import paper_2503_23956_amd as A

    q, k, v = _inputs(4, 1, 8, 2, 128, torch.bfloat16, "packed", 1)
    pos = torch.tensor([[5], [70], [-1], [900]], dtype=torch.int32, device="cuda:0")
    freqs = torch.tensor(A.air_rope_frequencies(64, 1e6)[0], device="cuda:0")
    outs = [torch.zeros((4, x.shape[1], 1, 128), dtype=x.dtype, device="cuda:0") for x in (q, k, v)]
    call = A.prepare_rope(q, k, v, *outs, positions=pos, freqs=freqs, axis_pairs=(64,))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        A.air_rope(prepared=call)
    want = [torch.zeros_like(o) for o in outs]
    side = torch.cuda.Stream()
    for step in range(4):
        q.copy_(torch.randn_like(q))
        pos += 1
        if step == 2:
            pos[2] = 17  # the slot is taken up
        g.replay()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            A.air_rope(q, k, v, *want, positions=pos, freqs=freqs, axis_pairs=(64,))
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert torch.equal(o, w)
        assert bool((outs[0][2] == 0).all()) == (step < 2 and int(pos[2]) < 0)
        if int(pos[2]) >= 0 and step < 2:
            pos[2] = -1000  # still empty
            for o, w in zip(outs, want):
                o[2] = 0
                w[2] = 0


def test_calls_without_work_and_broadcast_sources():
    import torch

    import paper_2503_23956_amd as A

    q, k, v = _inputs(2, 9, 4, 2, 64, torch.bfloat16, "token", 2)
    freqs = torch.tensor(A.air_rope_frequencies(32, 1e4)[0], device="cuda:0")
    pos = torch.arange(18, dtype=torch.int32, device="cuda:0").view(2, 9)
    none = torch.zeros((2, 0), dtype=torch.int32, device="cuda:0")
    A.air_rope(q[:, :, :0], k[:, :, :0], v[:, :, :0], positions=none, freqs=freqs, axis_pairs=(32,))
    wide = k[:1, :1, :1].expand(2, 4, 9, 64)  # one row for all
    kw = dict(positions=pos, freqs=freqs, axis_pairs=(32,))
    outs = [torch.zeros((2, 4, 9, 64), dtype=q.dtype, device="cuda:0") for _ in range(2)]
    A.air_rope(wide, q_out=outs[0], **kw)
    A.air_rope(wide.contiguous(), q_out=outs[1], **kw)
    torch.cuda.synchronize()
    assert torch.equal(*outs)
    with pytest.raises(A.AirError):  # in place: the rows of the destination would overlap
        A.air_rope(wide, **kw)


def test_as_many_rows_as_a_call_takes():
    import torch

    import paper_2503_23956_amd as A

    n, tail = 2 ** 27, 5000  # 17 GB
    x = torch.empty((1, 1, n, 64), dtype=torch.bfloat16, device="cuda:0")
    x[:, :, n - tail:] = torch.randn((1, 1, tail, 64), device="cuda:0").bfloat16()
    pos = torch.full((1, n), -1, dtype=torch.int32, device="cuda:0")
    pos[0, n - tail:] = torch.arange(tail, dtype=torch.int32, device="cuda:0")
    freqs = torch.tensor(A.air_rope_frequencies(32, 1e4)[0], device="cuda:0")
    few = x[:, :, n - tail:].clone()
    few_pos = pos[:, n - tail:].contiguous()
    A.air_rope(x, positions=pos, freqs=freqs, axis_pairs=(32,))
    A.air_rope(few, positions=few_pos, freqs=freqs, axis_pairs=(32,))
    torch.cuda.synchronize()
    assert torch.equal(x[:, :, n - tail:], few)
    more = torch.empty((1, 1, 1, 64), dtype=torch.bfloat16, device="cuda:0").expand(1, 1, n + 1, 64)
    with pytest.raises(A.AirError):
        A.air_rope(more, q_out=more)


@pytest.mark.parametrize("tokens", [1, 70])
def test_as_many_heads_as_a_call_takes(tokens):
    """Heads are independent: the same rows whether 16384 heads are one call's or eight calls'."""
    import torch

    import paper_2503_23956_amd as A

    q, k, v = (torch.randn((1, 16384, tokens, 64), device="cuda:0").bfloat16() for _ in range(3))
    pos = torch.arange(tokens, dtype=torch.int32, device="cuda:0").view(1, tokens) + 5
    kw = dict(positions=pos, freqs=torch.tensor(A.air_rope_frequencies(32, 1e4)[0], device="cuda:0"), axis_pairs=(32,))
    outs = [torch.zeros_like(x) for x in (q, k, v)]
    A.air_rope(q, k, v, *outs, **kw)
    parts = [torch.zeros_like(x) for x in (q, k, v)]
    for i in range(0, 16384, 2048):
        A.air_rope(*(x[:, i:i + 2048] for x in (q, k, v)), *(x[:, i:i + 2048] for x in parts), **kw)
    torch.cuda.synchronize()
    for a, b in zip(outs, parts):
        assert torch.equal(a, b)
    assert torch.equal(outs[2], v)
