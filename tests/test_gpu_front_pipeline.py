"""From the projections of a prompt to decoded tokens: rotation, prompt attention, scoring, budgets, compaction, and for every new
token rotation and decode attention, as a serving program calls them; eager and with the step recorded into a HIP graph."""
import math

import numpy as np
import pytest

import synth
from oracle import aircache_oracle as O

pytestmark = pytest.mark.gpu

L, HQ, HKV, D, STEPS = 2, 14, 2, 128, 5


def _rotated(x, w, pos, freqs, eps=1e-6):
    """[head][token][d] in fp64: norm with weight w, pairs (i, i + d / 2), one position axis per third of the pairs."""
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w
    axis = np.repeat(np.arange(3), AXES)
    angle = pos[axis].T * freqs
    c, s = np.cos(angle), np.sin(angle)
    a, b = y[..., : D // 2], y[..., D // 2:]
    return np.concatenate([a * c - b * s, a * s + b * c], -1)


AXES = (16, 24, 24)


@pytest.mark.parametrize("graph", [False, True])
def test_prompt_to_decoded_tokens(graph):
    import torch

    import paper_2503_23956_amd as A

    dev = torch.device("cuda:0")
    seqs = [synth.configs.Seq(14 + 400 + 40, 14, 400, 14 + 400, 40), synth.configs.Seq(14 + 333 + 25, 14, 333, 14 + 333, 25)]
    B, S = len(seqs), max(s.seq_len for s in seqs)
    gen = torch.Generator(device="cuda:0").manual_seed(3)
    freqs_host, _ = A.air_rope_frequencies(D // 2, 1e6)
    freqs = torch.tensor(freqs_host, device=dev)
    # positions: text counts on, image tokens have a row and a column of 20; -1 behind a sequence
    pos = np.full((3, B, S + STEPS), -1, dtype=np.int32)
    for b, s in enumerate(seqs):
        t = np.arange(s.seq_len)
        img = (t >= s.vis_start) & (t < s.text_start)
        flat = np.where(t < s.vis_start, t, t - s.vis_len + 20)
        r, c = (t - s.vis_start) // 20, (t - s.vis_start) % 20
        pos[:, b, : s.seq_len] = [np.where(img, 14, flat), np.where(img, 14 + r, flat), np.where(img, 14 + c, flat)]
    prompt_pos = torch.tensor(pos[:, :, :S], device=dev).contiguous()
    qw, kw = ((1 + 0.2 * torch.randn(D, generator=gen, device=dev)).bfloat16() for _ in range(2))
    f64 = lambda t: t.double().cpu().numpy()  # noqa: E731

    cfg = A.make_config(n_layers=L, n_q_heads=HQ, n_kv_heads=HKV, head_dim=D, batch=B, max_vis_len=400, max_nonvis_len=54, max_window=40,
                        max_decode_steps=STEPS, dtype=A.AIR_BF16, alpha=0.9, retention=0.25, device_steps=int(graph))
    cache = A.AirCache(cfg, dev)
    q, k, v, attn = [], [], [], []
    for _ in range(L):
        qkv = torch.randn((B, S, HQ + 2 * HKV, D), generator=gen, device=dev).bfloat16()
        for b, s in enumerate(seqs):
            qkv[b, s.seq_len:] = math.nan
        parts = [x.transpose(1, 2) for x in (qkv[:, :, :HQ], qkv[:, :, HQ:HQ + HKV], qkv[:, :, HQ + HKV:])]
        outs = [torch.zeros((B, x.shape[1], S, D), dtype=x.dtype, device=dev) for x in parts]
        A.air_rope(*parts, *outs, positions=prompt_pos, freqs=freqs, axis_pairs=AXES, q_weight=qw, k_weight=kw)
        o = torch.zeros((B, S, HQ, D), dtype=torch.bfloat16, device=dev).transpose(1, 2)
        A.air_prompt_attn(*outs, o, spans=[(b, 0, s.seq_len, 0, s.seq_len) for b, s in enumerate(seqs)])
        for x, out, w in zip(parts, outs, (qw, kw, None)):  # rotation: one rounding of the fp64 result, but for ties
            for b, s in enumerate(seqs):
                raw = f64(x[b, :, : s.seq_len])
                want = raw if w is None else _rotated(raw, f64(w), pos[:, b, : s.seq_len], freqs_host)
                got = f64(out[b, :, : s.seq_len])
                assert np.abs(got - want).max() <= np.abs(want).max() * 2.0 ** -8 and not out[b, :, s.seq_len:].any()
        for b, s in enumerate(seqs):  # attention of the rotated tensors
            n = s.seq_len
            for h in range(HQ):
                qq, kk, vv = f64(outs[0][b, h, :n]), f64(outs[1][b, h * HKV // HQ, :n]), f64(outs[2][b, h * HKV // HQ, :n])
                logit = qq @ kk.T / math.sqrt(D) + np.triu(np.full((n, n), -np.inf), 1)
                p = np.exp(logit - logit.max(1, keepdims=True))
                p /= p.sum(1, keepdims=True)
                # probabilities and outputs rounded to bf16, logits of at most 40 in fp32
                bound = (p @ np.abs(vv)) * (2.0 ** -8 + 1e-4) + np.abs(p @ vv) * 2.0 ** -8 + 1e-6
                assert (np.abs(f64(o[b, h, :n]) - p @ vv) <= bound).all()
        q.append(outs[0]), k.append(outs[1]), v.append(outs[2]), attn.append(o)
    # text queries as scoring wants them: row j = text token j of the sequence
    n_text = max(s.n_text for s in seqs)
    text = []
    for l in range(L):
        t = torch.zeros((B, HQ, n_text, D), dtype=torch.bfloat16, device=dev)
        for b, s in enumerate(seqs):
            t[b, :, : s.n_text] = q[l][b, :, s.text_start:s.seq_len]
        text.append(t)
    cache.air_score(0, L, text, k, v, seqs)
    cache.air_budget()
    cache.air_select_compact(0, L, k, v)

    # decode: one packed projection a layer, rotated into the dense tensors that the decode attention takes
    new = torch.zeros((L, B, HQ + 2 * HKV, D), dtype=torch.bfloat16, device=dev)
    qn, kn, vn = (torch.zeros((L, B, h, D), dtype=torch.bfloat16, device=dev) for h in (HQ, HKV, HKV))
    out = torch.zeros_like(qn)
    step_pos = torch.zeros((3, L * B, 1), dtype=torch.int32, device=dev)
    rows = [x.view(L * B, -1, 1, D) for x in (qn, kn, vn)]
    flat = new.view(L * B, HQ + 2 * HKV, 1, D)
    parts = [flat[:, :HQ], flat[:, HQ:HQ + HKV], flat[:, HQ + HKV:]]
    call = A.prepare_rope(*parts, *rows, positions=step_pos, freqs=freqs, axis_pairs=AXES, q_weight=qw, k_weight=kw)

    def step():
        A.air_rope(prepared=call)
        cache.air_decode_attn(0, L, qn, kn, vn, out)

    if graph:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
    added = []
    for t in range(STEPS):
        new.copy_(torch.randn(new.shape, generator=gen, device=dev))
        for b, s in enumerate(seqs):
            step_pos.view(3, L, B)[:, :, b] = s.seq_len - s.vis_len + 20 + t
        if graph:
            g.replay()
        else:
            step()
        torch.cuda.synchronize()
        added.append((kn.clone(), vn.clone()))
        for l in range(L):
            idx = cache.air_get_indices(l)
            bud = cache.air_get_budgets()
            for b, s in enumerate(seqs):
                p3 = np.full((3, 1), s.seq_len - s.vis_len + 20 + t)
                want_q = _rotated(f64(new[l, b, :HQ, None]), f64(qw), p3, freqs_host)[:, 0]
                assert np.abs(f64(qn[l, b]) - want_q).max() <= np.abs(want_q).max() * 2.0 ** -8
                seg = O.Segments(s.seq_len, s.vis_start, s.vis_len, s.win_start, s.win_len)
                for h in range(HKV):
                    kc, vc = O.compact(f64(k[l][b, h, : s.seq_len]), f64(v[l][b, h, : s.seq_len]), seg, idx[b, h, : bud[b, l]])
                    kc = np.concatenate([kc] + [f64(a[0][l, b, h])[None] for a in added])
                    vc = np.concatenate([vc] + [f64(a[1][l, b, h])[None] for a in added])
                    g0 = h * (HQ // HKV)
                    want = O.decode_attn(f64(qn[l, b, g0:g0 + HQ // HKV]), kc, vc)
                    np.testing.assert_allclose(f64(out[l, b, g0:g0 + HQ // HKV]), want, atol=2e-2)
    cache.close()
