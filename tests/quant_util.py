"""The 4-bit format and the attention over it in fp64, from their definitions in include/aircache.h."""
import math


def values_of(x, group):
    """What rows (any float type, [..., d]) stand for once held: fp64, every rounding of the definition in its place."""
    import torch

    y = x.double().unflatten(-1, (-1, group))

    def bf16_next_to(z, up):  # z: values of fp32; the nearest bf16, or its neighbour on the other side of z
        near = z.float().bfloat16()
        wrong = near.double() < z if up else near.double() > z
        bits = near.view(torch.int16) + torch.where((z < 0) != up, 1, -1).to(torch.int16)
        return torch.where(wrong, bits.view(torch.bfloat16), near).double()

    low, high = y.amin(-1, keepdim=True), y.amax(-1, keepdim=True)
    fine = torch.isfinite(y).all(-1, keepdim=True) & (y.abs().amax(-1, keepdim=True) < 2.0 ** 126)
    low, high = torch.where(fine, low, 0.0), torch.where(fine, high, 0.0)
    lo = bf16_next_to(low, False)
    step = bf16_next_to(((high - lo).float().double() / torch.full_like(high, 15.0)).float().double(), True)
    step = torch.where(step < 2.0 ** -120, 0.0, step)
    share = ((y - lo).float().double() / torch.where(step > 0, step, 1.0)).float().double()
    code = torch.where(step > 0, torch.round(share).clamp(0, 15), 0.0)
    return torch.where(fine, lo + step * torch.nan_to_num(code), math.nan).flatten(-2), torch.where(fine, step, math.nan).expand_as(y).flatten(-2)


def unpacked(cache):
    """(lo, step code, step) of K and of V, fp64 [B][H][capacity][d], out of the cache's memory as the header lays it out."""
    import torch

    out, d = [], cache.head_dim
    for i, (codes, scales) in enumerate(zip(cache.planes[:2], cache.planes[2:])):
        c = torch.stack([codes & 15, codes >> 4], dim=-1)  # [..., byte, half]
        if i == 0:
            p = torch.arange(d // 8, device=codes.device)
            byte = (d // 8 * (p % 4) + 4 * (p // 4))[:, None] + torch.arange(4, device=codes.device)
            c = c[..., byte, :].flatten(-2)[..., [0, 4, 1, 5, 2, 6, 3, 7]].flatten(-2)  # [..., p, element]
        else:
            c = c.flatten(-2)
        pair = scales.double().unflatten(-1, (-1, 2))
        lo, step = (pair[..., j].repeat_interleave(cache.group, dim=-1) for j in range(2))
        out.append((lo, step * c.double(), step))
    return out


def attention(cache, q, held, counts, causal, scale=None, weigh=True, wide=False):
    """(out, its bound, weights, their bound) of every sequence, fp64: lists over the batch of [Hq][count][d] and [H][held].

    Bounds: a logit is a sum of d products step q code and as many q lo, each exact or rounded to fp32, whose sums round once per term (bf16:
    codes have 16 added, and taken off again: 16 step q twice more); the exponent and the power of two (2^-22); sums of `held` terms; the factor
    p step keeps 15 bits (bf16: a first term cut off, 2^-7, the rest rounded, 2^-8) or 24; outputs are rounded once.

    bf16 calls of 33 rows and more, where they are large (the bound holds for both ways): V and the probabilities, and with these their sum, are rounded to fp16 (half a step 2^-11; probabilities below
    2^-14 of a reference that is at most 2^8 above the largest by 2^-25) or, where values have no ordinary magnitude (`wide`), to bf16 (2^-8);
    without weights, K in fp16 (2^-11, and 2^-25 of rows of at least 2^-6), with them in two such terms."""
    import torch

    d, H = cache.head_dim, cache.n_kv_heads
    g = q.shape[1] // H
    scale = scale or d ** -0.5
    half = 2.0 ** -8 if q.dtype == torch.bfloat16 else 2.0 ** -24
    (klo, kst, kstep), (vlo, vst, _) = unpacked(cache)
    extra = 32.0 * kstep if q.dtype == torch.bfloat16 else 0.0 * kstep
    result = []
    for b, (n, c) in enumerate(zip(held, counts)):
        qs = q[b, :, :c].double()
        kl, ks, vl, vs, ke = (x[b, :, :n].repeat_interleave(g, dim=0) for x in (klo, kst, vlo, vst, extra))
        t = lambda x: x.transpose(1, 2).contiguous()  # noqa: E731
        s = qs @ t(kl + ks) * scale
        size = qs.abs() @ t(kl.abs() + ks + ke) * scale
        seen = torch.ones((c, n), dtype=torch.bool, device=q.device)
        if causal:
            seen = torch.arange(n, device=q.device)[None] <= torch.arange(c, device=q.device)[:, None] + (n - c)
        s, size = s.masked_fill(~seen, -math.inf), size.masked_fill(~seen, 0.0)
        top = s.amax(-1, keepdim=True) if n else s.new_zeros((*s.shape[:2], 1))
        p = torch.exp(s - torch.where(torch.isinf(top) & (top < 0), 0.0, top))
        p = p.masked_fill(~seen, 0.0)
        p = p / p.sum(-1, keepdim=True).clamp(min=1e-300)
        off = size.amax(-1, keepdim=True) * ((2 * d + 16) * 2.0 ** -24) + size.amax(-1, keepdim=True) * 2.0 ** -22 if n else p.sum(-1, keepdim=True)
        if n and q.dtype == torch.bfloat16 and q.shape[2] * g >= 33:
            dot = (qs.abs() @ t((kl + ks).abs()) * scale).masked_fill(~seen, 0.0)
            least = qs.abs().sum(-1, keepdim=True) * (kl + ks).abs().amax((1, 2), keepdim=True) * scale * 2.0 ** -19
            off = off + (dot.amax(-1, keepdim=True) * 2.0 ** -11 + least) * (2.0 ** -11 if weigh else 1.0)
        rel = 2 * (torch.expm1(off) + 2.0 ** -22 + (n + 64) * 2.0 ** -24)
        vl_seen = torch.where(torch.isfinite(vl), vl, 0.0) if not bool(seen.all()) else vl
        o, a = p @ (vl_seen + vs), p @ (vl_seen.abs() + vs)
        low = half > 2.0 ** -20  # bf16
        many = low and q.shape[2] * g >= 33
        err = a * (rel + (3 * 2.0 ** (-8 if wide else -11) if many else 2.0 ** -15 if low else 2.0 ** -22))
        if many and n and not wide:
            err = err + (vl_seen.abs() + vs).amax(1, keepdim=True) * (2 * n * 2.0 ** -25) + n * 2.0 ** -25
        bound = err * 1.01 + (o.abs() + err) * half + 1e-37
        w = p.reshape(H, g * c, n).sum(1)
        wb = (p * rel).reshape(H, g * c, n).sum(1) * 1.01 + w * (g * c + 8) * 2.0 ** -24 + 1e-37
        result.append((o, bound, w, wb))
    return result
