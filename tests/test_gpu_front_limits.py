"""What air_rope and air_prompt_attn promise at the edges of their arguments, on the GPU."""
import math

import pytest

from test_front_limits import MIXED
from test_gpu_prompt import KINDS, _check, _run, _tensors

pytestmark = pytest.mark.gpu


def test_outputs_expanded_over_the_batch_are_refused():
    import torch

    import paper_2503_23956_amd as A

    q = torch.randn((2, 4, 3, 64), device="cuda:0").bfloat16()
    k = torch.randn((2, 2, 3, 64), device="cuda:0").bfloat16()
    out = torch.full((1, 4, 3, 64), 42.0, device="cuda:0").bfloat16()
    with pytest.raises(A.AirError, match="two sequences overlap"):
        A.air_prompt_attn(q, k, k, out.expand(2, 4, 3, 64))
    with pytest.raises(A.AirError, match="two sequences overlap"):
        A.air_prompt_attn(q[:1], k[:1], k[:1], out, spans=[(0, 0, 2, 0, 2), (0, 1, 2, 1, 2)])
    skew = out.as_strided((1, 4, 3, 64), (768, 64, 64, 1))  # head 1 of a token is head 0 of the next
    with pytest.raises(A.AirError, match="output rows overlap"):
        A.air_prompt_attn(q[:1], k[:1], k[:1], skew)
    with pytest.raises(A.AirError, match="rows of a destination overlap"):
        A.air_rope(q[:1], q_out=skew)
    torch.cuda.synchronize()
    assert bool((out == 42.0).all())


def test_prepared_calls_called_directly():
    import torch

    import paper_2503_23956_amd as A

    q = torch.randn((1, 8, 5, 128), device="cuda:0").bfloat16()
    k, v = (torch.randn((1, 2, 5000, 128), device="cuda:0").bfloat16() for _ in range(2))
    for spans in ([(0, 0, 5, 0, 5000)], [(0, 0, 5, 0, 5)]):  # with splits and without
        want, out = torch.zeros_like(q), torch.zeros_like(q)
        A.air_prompt_attn(q, k, v, want, spans=spans)
        call = A.prepare_prompt_attn(q, k, v, out, spans=spans)
        assert (call.workspace_bytes > 0) == (spans[0][4] == 5000)
        call()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        out.zero_()
        ws = torch.empty(max(1, call.workspace_bytes), dtype=torch.uint8, device="cuda:0")
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        call(side.cuda_stream, ws)
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    with pytest.raises(A.AirError, match="needs its workspace"):
        A.prepare_prompt_attn(q, k, v, out)(side.cuda_stream)
    turn = A.prepare_rope(q)
    turn()
    with pytest.raises(A.AirError, match="takes no workspace"):
        turn(workspace=ws)


def _without(q, k, v, n, m, low, high):
    """Attention in fp64 of n queries behind m - n keys, without the keys low .. high - 1, and its bound (the roundings as test_gpu_prompt
    counts them: logits of d products in fp32, exp2 to 2^-22, sums of m terms, bf16 probabilities and outputs)."""
    import torch

    d, g = q.shape[3], q.shape[1] // k.shape[1]
    at = torch.arange(m, device=q.device)
    use = (at[None, :] <= torch.arange(n, device=q.device)[:, None] + (m - n)) & ((at < low) | (at >= high))[None, :]
    want, bound = [], []
    for h in range(q.shape[1]):
        qs, ks, vs = q[0, h, :n].double(), k[0, h // g].double(), v[0, h // g].double()
        s = (qs @ ks.T.contiguous() * d ** -0.5).masked_fill(~use, -math.inf)
        p = torch.softmax(s, dim=1).nan_to_num(0.0)
        dot = (qs.abs() @ ks.abs().T.contiguous() * d ** -0.5).masked_fill(~use, 0.0).amax(1, keepdim=True)
        rel = 2 * (torch.expm1(dot * ((d + 8) * 2.0 ** -24)) + 2.0 ** -22 + (m + 64) * 2.0 ** -24)
        step = 2.0 ** -24
        if q.dtype == torch.bfloat16:
            rel, step = rel + 2.0 ** -8, 2.0 ** -8
        o, a = p @ vs, p @ vs.abs() * rel
        want.append(o)
        bound.append(a * 1.01 + (o.abs() + a) * step + 1e-37)
    return torch.stack(want), torch.stack(bound)


@pytest.mark.parametrize("dtype,d", KINDS)
@pytest.mark.parametrize("hq,hkv,n,m", [(4, 2, 1, 40), (4, 2, 3, 700), (28, 4, 1, 6000), (8, 2, 70, 3000), (28, 4, 200, 333), (28, 4, 900, 900), (28, 4, 3000, 3100)])
@pytest.mark.parametrize("key", [-math.inf, -3e4])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_visible_values_that_are_not_finite(dtype, d, hq, hkv, n, m, key, bad):
    """At keys that weigh nothing, whole tiles, waves and splits of them: their columns are not finite, wherever the keys lie; nothing else changes."""
    import torch

    import paper_2503_23956_amd as A

    q, k, v = _tensors(1, n, m, hq, hkv, d, dtype, n + m + d, order="token")
    q = q.abs()
    spans = [(0, 0, n, 0, m)]
    seen = torch.arange(n, device=q.device) + (m - n)  # last key of a row
    # (first and last such key, keys of them whose value is not finite)
    for low, high, at in ((0, m * 2 // 3, (0, m // 3)), (m // 5, m // 2, (m // 5 + 1,)), (max(1, m - 2), m, (m - 1,)), (max(1, m - 1 - n // 2), m, (max(1, m - 1 - n // 2),))):
        k2, v2 = k.clone(), v.clone()
        k2[:, :, low:high] = key
        want, bound = _without(q, k, v, n, m, low, high)
        for column, i in zip((5, d - 2), at):
            v2[:, :, i, column] = bad
        got = _run(A, q, k2, v2, spans)[0].double()
        some = torch.zeros((n, d), dtype=torch.bool, device=q.device)  # rows and columns that such a value reaches
        for column, i in zip((5, d - 2), at):
            some[:, column] |= seen >= i
        # a query element of 0 meets a key of -inf: 0 x inf, the logit is no number, and the row is none
        none = (q[0, :, :n] == 0).any(-1, keepdim=True) & (seen[:, None] >= low) & math.isinf(key)
        assert bool(torch.isnan(got[none.expand_as(got)]).all())
        zero = ((seen[:, None] < high) & (low == 0) & ~none).expand_as(got)  # rows of nothing but such keys
        if math.isinf(key):
            assert bool((got[zero] == 0).all())
        some = some.expand_as(got) & ~zero & ~none
        assert not bool(torch.isfinite(got[some]).any()), (low, high, at)
        assert bool(((got - want).abs() <= bound)[~some & ~zero & ~none].all()), (low, high, at)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv,n,m", [(7, 1, 1, 2), (28, 4, 1, 5), (28, 4, 1, 40), (8, 2, 4, 700), (28, 4, 1, 7432), (16, 1, 2, 3000), (14, 2, 3, 33)])
def test_probabilities_of_single_tokens_keep_16_bits(d, hq, hkv, n, m):
    """Elements whose values cancel show the roundings of the probabilities: 2^-16 of each, not the 2^-8 of bf16."""
    import torch

    import paper_2503_23956_amd as A

    q, k, v = _tensors(1, n, m, hq, hkv, d, "bf16", n + m + d, order="token")
    got = _run(A, q, k, v, [(0, 0, n, 0, m)])[0].double()
    g = hq // hkv
    qs, ks, vs = q[0].double(), k[0].double().repeat_interleave(g, dim=0), v[0].double().repeat_interleave(g, dim=0)
    behind = torch.arange(m, device=q.device)[None, :] > torch.arange(n, device=q.device)[:, None] + (m - n)
    s = (qs @ ks.transpose(1, 2).contiguous() * d ** -0.5).masked_fill(behind, -math.inf)
    dot = (qs.abs() @ ks.abs().transpose(1, 2).contiguous() * d ** -0.5).masked_fill(behind, 0.0).amax(-1, keepdim=True)
    p = torch.softmax(s, dim=-1)
    want, size = p @ vs, p @ vs.abs()
    # two bf16 terms, 16 bits: p = 2^e (1 + ...) less its first 8 bits is below 2^(e - 7), half a step there at most 2^(e - 16); logits in fp32 (d products and the factor), exp2 to 2^-22, sums of m terms;
    # both in the sum of the probabilities too; bf16 rounds the output
    rel = 2 * (torch.expm1(dot * ((d + 8) * 2.0 ** -24)) + 2.0 ** -22 + (m + 64) * 2.0 ** -24) + 2.0 ** -16
    bound = size * rel * 1.01 + (want.abs() + size * rel) * 2.0 ** -8
    far = (got - want).abs() - bound
    assert bool((far <= 0).all()), f"{far.max().item()} above its bound, {int((far > 0).sum())} elements"


@pytest.mark.parametrize("low,high", [(0, 5000), (10 ** 6, 10 ** 6 + 5000), (2 ** 30, 2 ** 31 - 1)])
def test_angles_at_any_position(low, high):
    """Cosine and sine of position x frequency, against the fraction of a turn in whole numbers: 2 pi to 200 bits."""
    import random
    from fractions import Fraction

    import numpy as np
    import torch

    import paper_2503_23956_amd as A

    rng = random.Random(low)
    inverse = Fraction("0.159154943091895335768883763372514362034459645740456448747667344058896797634226535090113802766253085956")  # 1 / (2 pi)
    scaled = int(inverse * 2 ** 300)
    T, pairs = 4000, 32
    pos = [rng.randint(low, high) for _ in range(T - 2)] + [low, high]
    freqs = [1.0, 0.5, 8.0, 2 * math.pi / 64] + [rng.uniform(0.5, 1.0) for _ in range(pairs - 4)]
    turns = np.empty((T, pairs))
    for j, f in enumerate(freqs):
        top, bottom = f.as_integer_ratio()
        mod = bottom << 300
        for i, p in enumerate(pos):
            turns[i, j] = float(Fraction(p * top * scaled % mod, mod))
    q = torch.zeros((1, 1, T, 64), device="cuda:0")
    q[..., :pairs] = 1.0  # the first of every pair: the result is (cos, sin)
    A.air_rope(q, positions=torch.tensor([[pos]], dtype=torch.int32, device="cuda:0"), freqs=torch.tensor(freqs, dtype=torch.float64, device="cuda:0"),
               axis_pairs=(pairs,))
    torch.cuda.synchronize()
    got = q[0, 0].double().cpu().numpy()
    # the rest of a turn to 2^-28 of one (2 pi 2^-28 rad); sine and cosine to 4 units of 2^-24; products with 1 and 0 are exact
    bound = 2 * math.pi * 2.0 ** -28 + 4 * 2.0 ** -24
    far = np.maximum(abs(got[:, :pairs] - np.cos(2 * math.pi * turns)), abs(got[:, pairs:] - np.sin(2 * math.pi * turns)))
    assert far.max() <= bound, (far.max(), bound)


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("dtype,d,hq,hkv,pairs,rows,split", MIXED)
def test_mixed_calls_of_every_kernel(dtype, d, hq, hkv, pairs, rows, split, packed):
    """Sequences in rows of a padded batch or behind each other with gaps; what lies behind a sequence's keys is no number."""
    import torch

    import paper_2503_23956_amd as A

    nq, nk = max(n for n, _ in pairs), max(m for _, m in pairs)
    if packed:
        spans, q0, k0 = [], 2, 1
        for n, m in pairs:
            spans.append((0, q0, n, k0, m))
            q0, k0 = q0 + n + 3, k0 + m + 2
        q, k, v = _tensors(1, q0, k0, hq, hkv, d, dtype, d + hq + rows, order="head")
    else:
        spans = [(b, 0, n, 0, m) for b, (n, m) in enumerate(pairs)]
        q, k, v = _tensors(len(pairs), nq, nk, hq, hkv, d, dtype, d + hq + rows, order="token")
    used = torch.zeros((k.shape[0], k.shape[2]), dtype=torch.bool, device=k.device)
    for b, _, _, k0, m in spans:
        used[b, k0:k0 + m] = True
    for x in (k, v):
        x.masked_fill_(~used[:, None, :, None], math.nan)
    tile, splits = A.air_prompt_plan(A.prepare_prompt_attn(q, k, v, torch.empty_like(q), spans=spans))
    assert (tile, splits > 1) == (rows, split)
    _check(q, k, v, spans, _run(A, q, k, v, spans))
