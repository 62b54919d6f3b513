"""air_quant_attn where magnitudes lie far apart: a slot that takes nearly all of a row beside many that share the rest, values of every size beside
each other, logits far beyond those of trained models, rows that are not numbers.  Bounds are relative to what the output is made of: sum p |v|."""
import math

import pytest

from quant_util import unpacked

pytestmark = pytest.mark.gpu


def _ints(x):
    import torch

    return torch.tensor(x, dtype=torch.int32, device="cuda:0")


def _randn(seed, *shape):
    import torch

    return torch.randn(shape, generator=torch.Generator(device="cuda:0").manual_seed(seed), device="cuda:0")


def _formula(cache, q, n, scale, head=0):
    """A KV head's rows (one query head each) over n slots that all of them see, fp64: sizes of the logits' sums, probabilities, values."""
    (kl, ks, kstep), (vl, vs, _) = ([y[:1, head:head + 1] for y in x] for x in unpacked(cache))
    k, v = (kl + ks)[0, 0, :n], (vl + vs)[0, 0, :n]
    x = q[0, head].double()
    s = x @ k.t().contiguous() * scale
    size = x.abs() @ (kl.abs() + ks + 32.0 * kstep)[0, 0, :n].t().contiguous() * scale
    return size, s.softmax(-1), v


def _logit_error(size, d, terms):
    """How far a probability may be off, relative: sums of 2 d products of exact numbers and the factor, a rounding of 2^-24 each of the sum of
    magnitudes (32 steps where codes have 16 added); K in one fp16 term (2^-11 of magnitudes) or two; the same in the sum."""
    import torch

    return 2 * torch.expm1(size * ((2 * d + 16) * 2.0 ** -24 + 2.0 ** (-11 if terms == 1 else -21)))


def _floor(p):
    """What a probability may lose beside its 11 bits: 2^-18 of the greatest among the 32 slots it is read with, at most 2^-31 of the row's greatest,
    and never more than itself."""
    import torch

    pad = (-p.shape[-1]) % 32
    near = torch.nn.functional.pad(p, (0, pad)).unflatten(-1, (-1, 32)).amax(-1).repeat_interleave(32, -1)[..., :p.shape[-1]]
    top = p.amax(-1, keepdim=True)
    return torch.minimum(p, torch.minimum(2.0 ** -31 * top, torch.maximum(2.0 ** -18 * near, 2.0 ** -91 * top)))


# ---- probabilities ---------------------------------------------------------------------------------------------------------------
def _check_out(got, size, p, val, group, terms, bits=11):
    """Outputs against sum p v: 11 bits of a probability, of their sum and of a value, 2^-15 of the greatest of a value's group, the floor."""
    want, a = p @ val, p @ val.abs()
    great = val.abs().unflatten(-1, (-1, group)).amax(-1).repeat_interleave(group, -1)
    off = _logit_error(size, val.shape[-1], terms)
    bound = (p * off) @ val.abs() + a * off.amax(-1, keepdim=True) + 3 * 2.0 ** -bits * a + p @ great * 2.0 ** -15 + _floor(p) @ val.abs()
    bound = bound * 1.01 + (want.abs() + bound) * 2.0 ** -8
    far = (got.double() - want).abs()
    assert bool((far <= bound).all()), f"{(far / bound).max().item()} of the bound, {(far / a).max().item()} of sum p |v|"


def _check_weights(w, size, p, d):
    exact = _logit_error(size, d, 2)
    want, rows = p.sum(0), p.shape[0]
    bound = (p * (exact + exact.amax(-1, keepdim=True) + 2.0 ** -21 + (p.shape[1] + 64) * 2.0 ** -23)).sum(0) + want * (rows + 8) * 2.0 ** -24
    far = (w.double() - want).abs()
    assert bool((far <= bound).all()), f"weights {(far / bound).max().item()} of the bound"


@pytest.mark.parametrize("above", [18, 25, 26, 40, 75])
@pytest.mark.parametrize("rows", [4, 20, 48, 300])
@pytest.mark.parametrize("d,group", [(64, 32), (128, 64)])
@pytest.mark.parametrize("weigh", [False, True])
def test_a_slot_far_above_the_others(d, group, rows, above, weigh):
    """One slot `above` (base 2) higher than the others' mean, its value 0: the output is what the others share, however little that is.  So many
    heads that every one is read in one piece."""
    import torch

    import paper_2503_23956_amd as A

    n, H, scale, lift = 4033, 256, 0.05, 16.0
    cache = A.QuantCache(1, H, n, d, group=group)
    k, v = 0.5 * _randn(1, 1, H, n, d), _randn(2, 1, H, n, d) + 1.0
    k[..., 0] = 0.0
    at = [0, n - 1] + [(977 * h) % n for h in range(2, H)]
    for h, x in enumerate(at):
        k[0, h, x], v[0, h, x] = 0.0, 0.0
        k[0, h, x, 0] = above * math.log(2.0) / (scale * lift)
    A.air_quant_append(cache, k.bfloat16(), v.bfloat16())
    q = _randn(3, 1, H, rows, d)
    q[..., 0] = lift
    q = q.bfloat16()
    out, w = torch.empty_like(q), torch.zeros((1, H, n), device="cuda:0")
    A.air_quant_attn(cache, q, out, lens=_ints([n]), causal=False, scale=scale, weights=w if weigh else None)
    for h in (0, 1, 100):
        size, p, val = _formula(cache, q, n, scale, h)
        _check_out(out[0, h], size, p, val, group, 2 if weigh else 1)
        if weigh:
            _check_weights(w[0, h], size, p, d)


@pytest.mark.parametrize("above", [26, 30])
def test_a_slot_far_above_a_quarter_of_a_million(above):
    """An even rest of 2^18 slots behind one slot, in one piece (the launch goes by a small max_len)."""
    import torch

    import paper_2503_23956_amd as A

    n, d, T = 1 << 18, 64, 40960
    cache = A.QuantCache(1, 1, n, d)
    k, v = torch.zeros((1, 1, n, d), device="cuda:0"), 1.0 + 0.25 * _randn(4, 1, 1, n, d)
    k[0, 0, 5, 0] = above * math.log(2.0)
    v[0, 0, 5] = 0.0
    A.air_quant_append(cache, k.bfloat16(), v.bfloat16())
    q = torch.zeros((1, 1, T, d), dtype=torch.bfloat16, device="cuda:0")
    q[..., 0] = 1.0
    out = torch.empty_like(q)
    A.air_quant_attn(cache, q, out, lens=_ints([n]), causal=False, scale=1.0, max_len=160)
    size, p, val = _formula(cache, q[:, :, :1], n, 1.0)
    want, a = p @ val, p @ val.abs()
    off = _logit_error(size, d, 1).amax()
    bound = a * (2 * off + 3 * 2.0 ** -11 + 2.0 ** -14) + _floor(p) @ val.abs() + a * (n + 64) * 2.0 ** -24
    bound = bound * 1.01 + (want.abs() + bound) * 2.0 ** -8
    assert bool(((out[0, 0].double() - want).abs() <= bound).all()), f"{out[0, 0, 0, :4].tolist()} for {want[0, :4].tolist()}"


@pytest.mark.parametrize("rows", [48, 300])
@pytest.mark.parametrize("weigh", [False, True])
def test_logits_that_rise_and_fall(rows, weigh):
    """Every other stretch of 96 slots lies 30 (base 2) lower, with values of 0 in the upper ones: references go up and down by the hundred."""
    import torch

    import paper_2503_23956_amd as A

    n, d, room, scale = 6000, 128, 70000, 0.05
    cache = A.QuantCache(1, 1, n + room, d)
    k, v = 0.5 * _randn(5, 1, 1, n, d), _randn(6, 1, 1, n, d)
    low = (torch.arange(n, device="cuda:0") // 96) % 2 == 1
    k[..., 0] = torch.where(low, -30.0 * math.log(2.0) / (scale * 16.0), 0.0)
    v[:, :, ~low] = 0.0
    A.air_quant_append(cache, k.bfloat16(), v.bfloat16())
    q = _randn(7, 1, 1, rows, d)
    q[..., 0] = 16.0
    q = q.bfloat16()
    out, w = torch.empty_like(q), torch.zeros((1, 1, n + room), device="cuda:0")
    A.air_quant_attn(cache, q, out, lens=_ints([n]), causal=False, scale=scale, weights=w if weigh else None)
    size, p, val = _formula(cache, q, n, scale)
    _check_out(out[0, 0], size, p, val, 32, 2 if weigh else 1)
    if weigh:
        _check_weights(w[0, 0, :n], size, p, d)


# ---- values ----------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("below", [10, 16, 20, 23, 30, 100])
@pytest.mark.parametrize("rows", [4, 20, 48, 300])
@pytest.mark.parametrize("d,group", [(64, 32), (64, 64), (128, 32), (128, 64)])
@pytest.mark.parametrize("weighs", [False, True])
@pytest.mark.parametrize("pieces", [1, 2])
def test_values_beside_larger_ones(below, rows, d, group, weighs, pieces):
    """A slot of ordinary values, at which no row looks, or which weighs 2^-below, beside others 2^-below as large; in every group of columns the same at
    another size.  A row looks at few slots.  Read in one piece (many heads) or many."""
    import torch

    import paper_2503_23956_amd as A

    n, H, room, scale = (1500, 256, 0, 0.5) if pieces == 1 else (1500, 1, 70000, 0.5)
    cache = A.QuantCache(1, H, n + room, d, group=group)
    k, v = 0.5 * _randn(1, 1, H, n, d), _randn(2, 1, H, n, d) * 2.0 ** -below
    k[..., 0] = 0.0
    k[:, :, 700, 0] = -below * math.log(2.0) / (scale * 16.0) if weighs else -4000.0
    v[:, :, 700] *= 2.0 ** below
    for g in range(d // group):
        v[..., g * group:(g + 1) * group] *= 10.0 ** (3 * g)
    A.air_quant_append(cache, k.bfloat16(), v.bfloat16())
    q = _randn(3, 1, H, rows, d)
    q[..., 0] = 16.0
    q = q.bfloat16()
    out, w = torch.empty_like(q), torch.zeros((1, H, n + room), device="cuda:0")
    A.air_quant_attn(cache, q, out, lens=_ints([n]), causal=False, scale=scale, weights=w)
    for h in (0, H // 2):
        size, p, val = _formula(cache, q, n, scale, h)
        # (the slot's own logit is far from the others': its error, larger than theirs, is not that of their probabilities)
        size[:, 700] = torch.where(p[:, 700] > 2.0 ** -126, size[:, 700], 0.0)
        _check_out(out[0, h], size, p, val, group, 2, 11 if below < 24 else 8)


# ---- keys ------------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("rows", [4, 20, 48, 300])
@pytest.mark.parametrize("size", [-20, -8, -7, -6, -5, 0, 10, 11, 12, 40])
def test_weights_of_small_and_large_keys(rows, size):
    """Equal keys lo + 8 step = 2^size (1 + 255 2^-19), whose low bits lie 2^-19 and less below: the rows' logits are 600 (base 2), and every slot has its share.
    K has 22 bits; sums are rounded to 24 sixteen times (products of two terms) and six times (by group)."""
    import torch

    import paper_2503_23956_amd as A

    n, d, room = 40, 128, 70000
    cache = A.QuantCache(1, 1, n + room, d)
    for p in cache.planes[:2]:
        p.fill_(0x88)
    for p in cache.planes[2:]:
        p[..., ::2], p[..., 1::2] = 2.0 ** size, 255 * 2.0 ** (size - 22)
    q = torch.full((1, 1, rows, d), 2304.0 * 2.0 ** (-6 - size), device="cuda:0").bfloat16()
    w = torch.zeros((1, 1, n + room), device="cuda:0")
    A.air_quant_attn(cache, q, None, lens=_ints([n]), causal=False, weights=w)
    want = rows / n
    bound = math.log(2.0) * 600 * (2.0 ** -22 + 22 * 2.0 ** -24) + 2.0 ** -21 + (n + rows + 72) * 2.0 ** -24
    far = (w[0, 0, :n].double() - want).abs().max().item() / want
    assert far <= bound, f"{far} off, {bound} allowed"
    assert not bool(w[0, 0, n:].any())


# ---- logits of any size ----------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("d,group", [(64, 32), (64, 64), (128, 32), (128, 64)])
@pytest.mark.parametrize("rows", [1, 6, 20, 48, 300])
@pytest.mark.parametrize("size", [1e2, 3e3, 1e6, 1e9])
@pytest.mark.parametrize("pieces", [1, 2])
def test_equal_logits_share_a_row_at_any_size(d, group, rows, size, pieces):
    """Equal keys of any elements: equal logits, so that the slots share a row equally however large these are, in the outputs and in the weights: sums
    of as many terms, and a product with one over the sum."""
    import torch

    import paper_2503_23956_amd as A

    n, H, room = (300, 32, 9000) if pieces == 1 else (300, 1, 70000)
    cache = A.QuantCache(1, H, n + room, d, group=group)
    k, v = _randn(1, 1, H, 1, d).bfloat16().expand(1, H, n, d), _randn(2, 1, H, n, d).bfloat16()
    A.air_quant_append(cache, k, v)
    q = (size * _randn(3, 1, H, rows, d)).bfloat16()
    out, w = torch.empty_like(q), torch.zeros((1, H, n + room), device="cuda:0")
    A.air_quant_attn(cache, q, out, lens=_ints([n]), causal=False, weights=w)
    far = (w[:, :, :n].double() * n / rows - 1.0).abs().max().item()
    assert far <= (n + rows + 72) * 2.0 ** -24 + 2.0 ** -21, f"weights {far} off"
    assert not bool(w[:, :, n:].any())
    _, (vl, vs, _) = unpacked(cache)
    val = (vl + vs)[:, :, :n]
    want, a = val.mean(2, keepdim=True), val.abs().mean(2, keepdim=True)
    assert bool(((out.double() - want).abs() <= a * 3 * 2.0 ** -11 + 2.0 ** -8 * want.abs() + 1e-6).all())


@pytest.mark.parametrize("d,group", [(64, 32), (128, 64)])
@pytest.mark.parametrize("rows", [1, 20, 48, 300])
@pytest.mark.parametrize("size", [30.0, 1e3, 1e5, 1e7])
@pytest.mark.parametrize("causal", [False, True])
def test_weights_of_a_row_add_up_to_one_at_any_size(d, group, rows, size, causal):
    import torch

    import paper_2503_23956_amd as A

    n, room = 2000, 70000
    cache = A.QuantCache(1, 1, n + room, d, group=group)
    A.air_quant_append(cache, _randn(1, 1, 1, n, d).bfloat16(), _randn(2, 1, 1, n, d).bfloat16())
    q = (size * _randn(3, 1, 1, rows, d)).bfloat16()
    w = torch.zeros((1, 1, n + room), device="cuda:0")
    A.air_quant_attn(cache, q, None, lens=_ints([n]), causal=causal, weights=w)
    far = abs(w.double().sum().item() / rows - 1.0)
    # the sums of 2000 probabilities, their factor, and weights of up to `rows` terms
    assert far <= (n + rows + 72) * 2.0 ** -24 + 2.0 ** -20, f"{far} off"


# ---- rows that are not numbers ---------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,d,group", [("bf16", 64, 32), ("bf16", 128, 64), ("f32", 64, 64), ("f32", 128, 32)])
@pytest.mark.parametrize("T,bad", [(2, 0), (8, 0), (8, 3), (12, 5), (60, 0), (60, 31), (300, 150)])
@pytest.mark.parametrize("room", [0, 70000])
def test_a_row_of_nan_weighs_only_slots_that_it_sees(dtype, d, group, T, bad, room):
    import torch

    import paper_2503_23956_amd as A

    n = 400
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    cache = A.QuantCache(1, 1, n + room, d, A.AIR_BF16 if dtype == "bf16" else A.AIR_F32, group=group)
    A.air_quant_append(cache, _randn(1, 1, 1, n, d).to(dt), _randn(2, 1, 1, n, d).to(dt))
    q = _randn(3, 1, 1, T, d).to(dt)
    q[0, 0, bad, 1] = math.nan
    out, w = torch.empty_like(q), torch.zeros((1, 1, n + room), device="cuda:0")
    A.air_quant_attn(cache, q, out, lens=_ints([n]), causal=True, weights=w)
    seen = n - T + 1 + bad  # slots that the row sees
    assert bool(w[0, 0, :seen].isnan().all()) and not bool(w[0, 0, seen:].isnan().any())
    assert bool(out[0, 0, bad].isnan().all()) and not bool(out[0, 0, :bad].isnan().any()) and not bool(out[0, 0, bad + 1:].isnan().any())
    # what the others give to the slots that it does not see
    q2, w2 = q.clone(), torch.zeros_like(w)
    q2[0, 0, bad] = 0.0
    A.air_quant_attn(cache, q2, None, lens=_ints([n]), causal=True, weights=w2)
    assert torch.equal(w[0, 0, seen:], w2[0, 0, seen:])


# ---- scales ----------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("scale", [1.5e-45, 1e-42, 1e-38, 1e-30, 1e30, 1e38])
@pytest.mark.parametrize("rows", [1, 8, 20, 48, 300])
@pytest.mark.parametrize("room", [0, 70000])
@pytest.mark.parametrize("q_size", [1e-12, 1.0, 1e12])
def test_scales_at_the_ends_of_their_range(scale, rows, room, q_size):
    """Logits that all vanish, of rows that see all slots, some or none: the mean of what they see; and logits of 0 at any scale."""
    import torch

    import paper_2503_23956_amd as A

    n, d = 200, 128
    cache = A.QuantCache(1, 1, n + room, d)
    k, v = _randn(1, 1, 1, n, d), _randn(2, 1, 1, n, d) + 1.0
    q = q_size * _randn(3, 1, 1, rows, d)
    if scale * q_size > 1e-10:  # keys of 0
        k.zero_()
    A.air_quant_append(cache, k.bfloat16(), v.bfloat16())
    q = q.bfloat16()
    out, w = torch.empty_like(q), torch.zeros((1, 1, n + room), device="cuda:0")
    A.air_quant_attn(cache, q, out, lens=_ints([n]), causal=True, scale=scale, weights=w)
    _, (vl, vs, _) = unpacked(cache)
    val = (vl + vs)[0, 0, :n]
    seen = (torch.arange(rows, device="cuda:0") + 1 + n - rows).clamp(min=0)
    p = (torch.arange(n, device="cuda:0") < seen[:, None]).double() / seen[:, None].clamp(min=1)
    want, a = p @ val, p @ val.abs()
    assert bool(((out[0, 0].double() - want).abs() <= a * (3 * 2.0 ** -11 + 2.0 ** -8) + 1e-6).all())
    assert bool(((w[0, 0, :n].double() - p.sum(0)).abs() <= p.sum(0) * ((n + rows + 72) * 2.0 ** -24 + 2.0 ** -20)).all())
